"""Calls of the paged cache at the edges of what the header allows."""
import numpy as np
import pytest
import torch

from tests import helpers as H
from tests.test_gpu_paged import make_cache, pools_of, run_attention, run_evict, same_bits

pytestmark = pytest.mark.gpu


def test_fill_of_nothing_across_heads():
    from paper_2507_08143_b200 import binding as B
    _, cache, len_d = make_cache([[[4, -1], [0, 9]]], 8, 2, 8)
    before = pools_of(cache)
    empty = torch.empty(1, 2, 0, 128, dtype=torch.bfloat16, device="cuda")
    out, st = torch.full_like(len_d, 9), torch.full_like(len_d, 9)
    B.paged_fill(cache, B.Shape(1, 2, 128, 48, [0, 0]), empty, empty, [0, 0], idx=torch.empty(1, 0, dtype=torch.int32, device="cuda"),
                 head_offsets=torch.zeros(1, 2, 3, dtype=torch.int32, device="cuda"), lengths=len_d, lengths_out=out, status=st)
    assert torch.equal(out, len_d) and not st.any()
    same_bits(pools_of(cache), before, "nothing")


def test_evict_window_that_begins_below_the_least_position():
    """next_position - recent below -2^31: every token is recent, so the lowest slots stay and nothing moves."""
    from paper_2507_08143_b200 import binding as B
    _, cache, len_d = make_cache([[[50]]], 16, 0, 3)
    before = pools_of(cache)
    out, budgets = torch.zeros_like(len_d), torch.full_like(len_d, 20)
    nxt = torch.tensor([-2 ** 31 + 5], dtype=torch.int32, device="cuda")
    B.paged_evict(cache, len_d, budgets, out, 50, recent=10, next_position=nxt)
    assert int(out) == 20
    same_bits(pools_of(cache), before, "nothing moves")
