"""Precision of the attention over the paged cache where its terms cancel: the softmax weights must not lose more than two bf16
terms leave out, whatever the values are that they multiply."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from tests import helpers as H
from tests.test_gpu_paged import make_cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("g,append", [(1, False), (4, True), (8, True), (16, True), (20, False)])
def test_attention_weights_keep_their_bits(g, append):
    """Nearly equal weights against values of either sign: many results are far smaller than the sum of |p v| that a rounding
    of the weights scales with.  Bound, relative to that sum:
      scores     eight accumulations of 16 products, each dropping at most 2^-23 of the largest partial sum per summand, and 2
                 further roundings: dy = (8 * 17 + 2) * 2^-23 * mag, mag the largest scale * sum |q||k|; twice (weight and sum)
      weights    2 * 2^-22 of the exponentials, (n / 8 + 64) * 2^-24 of their sum in fp32
      product    the weight, in [2^e, 2^(e+1)), in two bf16 terms: the first cut off, the second, below 2^(e-7), rounded to a step of
                 at most 2^(e-15), so by at most 2^(e-16): 2^-16 of the weight in all (rounding the first term gives less); 17
                 summands per 16 tokens and term, and at most 16 joins: (n / 16 + 16) * 2 * 17 * 2^-23
    and the result is rounded once to bf16: 2^-8 of itself."""
    from paper_2507_08143_b200 import binding as B
    scale, q_scale = 128 ** -0.5, 0.1
    lengths = np.array([[[3, 12, 33, 40], [700, 17, 5, 1]]], np.int32)
    _, heads, batch = lengths.shape
    host, cache, len_d = make_cache(lengths, 16, 1, 50 + g)
    gen = torch.Generator().manual_seed(g)
    q = (q_scale * torch.randn(batch, heads * g, 128, generator=gen)).bfloat16()
    kn, vn = torch.randn(batch, heads, 128, generator=gen).bfloat16(), torch.randn(batch, heads, 128, generator=gen).bfloat16()
    opt = B.decode_options(g, 701, scale=scale)
    out = torch.empty(batch, heads * g, 128, dtype=torch.bfloat16, device="cuda")
    new = dict(k_new=kn.cuda(), v_new=vn.cuda()) if append else {}
    B.paged_attention(cache, 0, opt, q.cuda(), len_d, out, B.alloc_paged_attention_workspace(cache, opt), **new)
    new = dict(k_new=H.bits(kn), v_new=H.bits(vn)) if append else {}
    ref, _, _, info = po.attention(host, 0, H.bits(q), lengths, np.float64(np.float32(scale)), **new)
    got = out.float().cpu().numpy().astype(np.float64)
    for (h, b), (at, p, pv, mag) in info.items():
        rows, n = slice(h * g, (h + 1) * g), len(at)
        rel = 2 * (8 * 17 + 2) * 2.0 ** -23 * mag + 2 * 2.0 ** -22 + (n / 8 + 64) * 2.0 ** -24
        rel += 2.0 ** -16 + (n / 16 + 16) * 2 * 17 * 2.0 ** -23
        tol = 1.01 * rel * pv + 2.0 ** -8 * np.abs(ref[b, rows]) + 1e-30
        err = np.abs(got[b, rows] - ref[b, rows])
        assert np.all(err <= tol), f"(h={h}, b={b}, n={n}): {np.max(err / tol):.2f} of the bound"


@pytest.mark.parametrize("n", [1, 2, 20])
def test_attention_of_infinite_values_is_infinite(n):
    """Weights that one term holds exactly (all scores are equal: every weight is 1 before the division) leave nothing for the
    second, which must not make 0 * inf of an infinite value."""
    from paper_2507_08143_b200 import binding as B
    host, cache, len_d = make_cache([[[n]]], 16, 1, 60)
    at = po.slot_of(host, (0, 0, 0), n - 1)
    cache.tensors[1][at][3], cache.tensors[1][at][4] = float("inf"), float("-inf")
    q = torch.zeros(1, 3, 128, dtype=torch.bfloat16, device="cuda")
    opt = B.decode_options(3, n)
    out = torch.empty_like(q)
    B.paged_attention(cache, 0, opt, q, len_d, out, B.alloc_paged_attention_workspace(cache, opt))
    o = out.float().cpu()
    assert torch.all(o[..., 3] == float("inf")) and torch.all(o[..., 4] == float("-inf"))
    assert torch.isfinite(o[..., :3]).all() and torch.isfinite(o[..., 5:]).all()
