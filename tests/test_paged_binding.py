"""The binding of the paged calls: the structs they are given, and the compiled checks behind them."""
import ctypes

import pytest
import torch

from paper_2507_08143_b200 import binding as B


def _cache():
    k = torch.zeros(4, 16, 128, dtype=torch.bfloat16)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)
    return B.PagedCache(k, k.clone(), i32(1, 2, 3, 2), mass=torch.zeros(4, 16), positions=i32(4, 16))


def test_calls_refuse_other_structs():
    """Every struct goes to the library by address: one of another kind would be read as what it is not."""
    c, shape, i32 = _cache(), B.Shape(1, 2, 128, 48, [4, 0, 3]), lambda *s: torch.zeros(*s, dtype=torch.int32)
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)
    q, n = bf(3, 4, 128), i32(1, 2, 3)
    for cache, opt in ((c, B.options()), (c, c), (c, c.c), (c, None), (shape, B.decode_options(2, 20)), (c.c, B.decode_options(2, 20)),
                       (None, B.decode_options(2, 20))):
        with pytest.raises(TypeError):
            B.paged_attention(cache, 0, opt, q, n, bf(3, 4, 128), bf(100))
    kv = bf(1, 2, 7, 128)
    for cache, s in ((c, c), (c, shape.c), (c, B.options()), (shape, shape), (None, shape)):
        with pytest.raises(TypeError):
            B.paged_fill(cache, s, kv, kv, [2, 0, 3])
    for cache in (shape, c.c, None):
        with pytest.raises(TypeError):
            B.paged_evict(cache, n, n, n, 32)
    for cache, opt in ((c, B.options()), (shape, B.decode_options(2, 20)), (c, c)):
        with pytest.raises((TypeError, ctypes.ArgumentError)):
            B.paged_attention_workspace_bytes(cache, opt)
