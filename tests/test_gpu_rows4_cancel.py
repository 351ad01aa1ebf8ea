"""Attention over rows in 4 bits whose values lie on both sides of 0: over a long context little is left of what is summed, and rows of one
token come out as they are held, wherever their least value and step are."""
import numpy as np
import pytest
import torch

from oracle import rows_oracle as ro
from oracle.compactor_oracle import bf16_bits_to_f64
from tests import helpers as H

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads, g, softcap", [(16, 4, 0.0), (16, 12, 0.0), (16, 3, 30.0)])
def test_outputs_of_a_long_context_are_the_nearest_bf16(heads, g, softcap):
    """Before it is rounded to bf16 an output is off by little more than the weights' two terms make it: each weight by at most 2^-16 of itself, on either
    side, which over the tokens adds up to less than 2^-16 sqrt(sum p^2 v^2); as much again is left to the sums in fp32.  An output that is off by that much
    rounds to another bf16 than the exact one with a probability of at most twice that over the step between two bf16, 2^-8 of its power of
    two.  Sums of steps and of least values apart from each other, each of one sign, are ten times further off."""
    from paper_2507_08143_b200 import binding as B
    gen = torch.Generator(device="cuda").manual_seed(12)
    page, n = 64, 131072
    per = n // page
    table = torch.randperm(heads * per, generator=gen, device="cuda").to(torch.int32).view(1, heads, 1, per)
    pools = [torch.empty(heads * per, page, 80, dtype=torch.uint8, device="cuda") for _ in range(2)]
    cache = B.PagedCache4(*pools, table)
    lengths = torch.zeros(1, heads, 1, dtype=torch.int32, device="cuda")
    for h in range(heads):                                   # (one at a time: the pools are what is large)
        x = [torch.randn(1, 1, n, 128, generator=gen, device="cuda").bfloat16() for _ in range(2)]
        B.paged_fill(B.PagedCache4(*pools, table[:, h:h + 1].contiguous()), B.Shape(1, 1, 128, 48, [n]), *x, [n])
    lengths.fill_(n)
    q = torch.randn(1, heads * g, 128, generator=gen, device="cuda").bfloat16()
    opt = B.decode_options(g, n, softcap=softcap)
    out = torch.empty_like(q)
    B.paged_attention(cache, 0, opt, q, lengths, out, B.alloc_paged_attention_workspace(cache, opt))
    other, allowed = 0, 0.0
    for h in range(heads):
        def values(pool):
            rows = pool[table[0, h, 0].long()].flatten(0, 1)
            par = rows[:, 64:].contiguous().view(torch.bfloat16).double().view(-1, 4, 2)
            codes = torch.stack([rows[:, :64] & 15, rows[:, :64] >> 4], -1).flatten(1).double().view(-1, 4, 32)
            return (par[..., 1:] + par[..., :1] * codes).flatten(1)
        k, v = values(pools[0]), values(pools[1])
        y = float(np.float32(128 ** -0.5)) * (q[0, h * g:(h + 1) * g].double() @ k.T)
        p = torch.softmax(softcap * torch.tanh(y / softcap) if softcap else y, 1)
        want = p @ v
        off = 2 * 2.0 ** -16 * torch.sqrt(p.square() @ v.square())
        step = torch.exp2(torch.floor(torch.log2(want.abs())) - 7)
        nearest = torch.from_numpy(bf16_bits_to_f64(ro.f64_to_bf16_bits(want.cpu().numpy()))).cuda()
        other += int((out[0, h * g:(h + 1) * g].double() != nearest).sum())
        allowed += float((2 * off / step).clamp(max=1).sum())
    print(f"{other} of {q.numel()} are not the nearest ({100 * other / q.numel():.2f} %), {100 * allowed / q.numel():.2f} % allowed")
    assert other <= allowed, f"{other} of {q.numel()}, {allowed:.0f} allowed"


@pytest.mark.parametrize("g", [1, 9])
def test_a_row_of_one_token_is_what_it_is_held_as(g):
    """Its weight is 1, so that the output is the value rounded once, to the bit: least values far above the step, far below it, of either sign, and
    steps at the ends of their range."""
    from paper_2507_08143_b200 import binding as B
    rng = np.random.default_rng(5)
    rows = []
    for offset in (0.0, 1.0, -3.0, 2.0 ** 9, -2.0 ** 12, 2.0 ** 20):
        for scale in (1.0, 2.0 ** -6, 2.0 ** -30, 2.0 ** -118, 2.0 ** 118):
            for x in (rng.standard_normal(128), rng.random(128), -rng.random(128), rng.random(128) ** 8 + 2.0 ** -25, np.zeros(128)):
                rows.append(offset * (scale if scale > 1 else 1.0) * (2.0 ** -20 if scale > 1 else 1.0) + scale * x)
    bits = ro.f64_to_bf16_bits(np.array(rows))
    batch = len(rows)
    v = torch.from_numpy(bf16_bits_to_f64(bits)).bfloat16().cuda().view(batch, 1, 128)
    table = torch.arange(batch, dtype=torch.int32, device="cuda").view(1, 1, batch, 1)
    pool = lambda: torch.zeros(batch, 8, 80, dtype=torch.uint8, device="cuda")
    cache = B.PagedCache4(pool(), pool(), table)
    k, q = torch.randn(batch, 1, 128, device="cuda").bfloat16(), torch.randn(batch, g, 128, device="cuda").bfloat16()
    opt = B.decode_options(g, 8)
    out = torch.empty_like(q)
    B.paged_attention(cache, 0, opt, q, torch.zeros(1, 1, batch, dtype=torch.int32, device="cuda"), out, B.alloc_paged_attention_workspace(cache, opt), k_new=k,
                      v_new=v)
    want = bf16_bits_to_f64(ro.f64_to_bf16_bits(ro.values4(ro.hold4(bits))))
    assert np.isfinite(want).all()
    got = out.double().cpu().numpy()
    for j in range(g):
        np.testing.assert_array_equal(got[:, j], want)


@pytest.mark.parametrize("g", [5, 12])
def test_a_channel_of_zeros_among_others_of_one_sign_stays_zero(g):
    """Its code is that of the least (or the greatest) value in every row, or it is the least value 0 itself: both sums that it is made of are each other's opposites,
    product by product."""
    from paper_2507_08143_b200 import binding as B
    gen = torch.Generator(device="cuda").manual_seed(6)
    heads, page, n = 3, 16, 20011
    per = -(-n // page)
    table = torch.randperm(heads * per, generator=gen, device="cuda").to(torch.int32).view(1, heads, 1, per)
    pools = [torch.empty(heads * per, page, 80, dtype=torch.uint8, device="cuda") for _ in range(2)]
    cache = B.PagedCache4(*pools, table)
    lengths = torch.zeros(1, heads, 1, dtype=torch.int32, device="cuda")
    k = torch.randn(1, heads, n, 128, generator=gen, device="cuda").bfloat16()
    v = torch.randn(1, heads, n, 128, generator=gen, device="cuda").abs().bfloat16()
    v[..., 0::8] = 0
    v[..., 64:96] = torch.where(torch.arange(32, device="cuda") % 8 == 0, 0.0, 100.0)
    B.paged_fill(cache, B.Shape(1, heads, 128, 48, [n]), k, v, [n], lengths_out=lengths)
    q = torch.randn(1, heads * g, 128, generator=gen, device="cuda").bfloat16()
    opt = B.decode_options(g, n)
    out = torch.empty_like(q)
    B.paged_attention(cache, 0, opt, q, lengths, out, B.alloc_paged_attention_workspace(cache, opt))
    assert not out[..., 0::8].any()
    others = out[..., torch.arange(128, device="cuda") % 8 != 0]
    assert torch.all(others > 0.5)
