"""Attention over long units in 4 bits, whose second kernel is laid out for many weights: against 64 bits on the GPU, two runs alike."""
import numpy as np
import pytest
import torch

from oracle import rows_oracle as ro
from tests import helpers as H

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens, heads, g", [([131071], 2, 5), ([40000, 90001, 0, 700], 4, 4), ([70000], 1, 12)])
@pytest.mark.parametrize("accumulate", [True, False])
def test_attention4_of_long_units(lens, heads, g, accumulate):
    from paper_2507_08143_b200 import binding as B
    gen = torch.Generator(device="cuda").manual_seed(9)
    page, batch = 64, len(lens)
    per = [-(-(n + 1) // page) for n in lens]
    table = torch.full((1, heads, batch, max(per)), -1, dtype=torch.int32, device="cuda")
    ids = torch.randperm(heads * sum(per), generator=gen, device="cuda").to(torch.int32)
    at = 0
    for h in range(heads):
        for b in range(batch):
            table[0, h, b, : per[b]] = ids[at: at + per[b]]
            at += per[b]
    pool = lambda: torch.full((ids.numel(), page, 80), 255, dtype=torch.uint8, device="cuda")
    cache = B.PagedCache4(pool(), pool(), table, mass=torch.zeros(ids.numel(), page, device="cuda"))
    lengths = torch.zeros(1, heads, batch, dtype=torch.int32, device="cuda")
    x = [torch.randn(1, heads, sum(lens), 128, generator=gen, device="cuda").bfloat16() for _ in range(2)]
    B.paged_fill(cache, B.Shape(1, heads, 128, 48, lens), *x, lens, lengths_out=lengths)
    q = torch.randn(batch, heads * g, 128, generator=gen, device="cuda").bfloat16()
    opt = B.decode_options(g, max(lens) + 1, accumulate=accumulate)
    ws = B.alloc_paged_attention_workspace(cache, opt)
    got = []
    for _ in range(2):
        cache.tensors[3].zero_()
        out, lse = torch.empty_like(q), torch.empty(batch, heads * g, device="cuda")
        B.paged_attention(cache, 0, opt, q, lengths, out, ws, lse_out=lse)
        got.append((out, lse, cache.tensors[3].clone()))
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(*got))
    out, lse, mass = got[0]
    start = np.concatenate([[0], np.cumsum(lens)])
    for h in range(heads):
        for b, n in enumerate(lens):
            rows = slice(h * g, (h + 1) * g)
            if n == 0:
                assert torch.all(out[b, rows] == 0) and torch.all(lse[b, rows] == float("-inf"))
                continue
            (ks, kl), (vs, vl) = ([torch.from_numpy(y).cuda() for y in ro.values4(ro.hold4(H.bits(t[0, h, start[b]: start[b] + n])), True)] for t in x)
            qq, scale = q[b, rows].double(), float(np.float32(128 ** -0.5))
            y = scale * (qq @ (ks + kl).T)
            mag = float((scale * (qq.abs() @ (ks.abs() + kl.abs()).T)).max())
            p = torch.softmax(y, 1)
            # as in the other tests of these rows: 161 2^-23 of the largest sum for a score; weights; two terms 2^-16; sums over n tokens; bf16
            dy = 161 * 2.0 ** -23 * mag
            rel = 2 * dy + 2 * 2.0 ** -22 + (n / 8 + 64) * 2.0 ** -24
            tol = (rel + 2.0 ** -16 + (n / 16 + 17) * 17 * 2.0 ** -23) * 1.01 * (p @ (vs.abs() + vl.abs())) + 2.0 ** -8 * (p @ (vs + vl)).abs()
            assert torch.all((out[b, rows].double() - p @ (vs + vl)).abs() <= tol)
            want = torch.logsumexp(y, 1)
            assert torch.all((lse[b, rows].double() - want).abs() <= dy + rel + 2.0 ** -22 * want.abs())
            if accumulate:
                w = mass[table[0, h, b, : per[b]].long()].flatten()[:n].double()
                assert torch.all((w - p.sum(0)).abs() <= (1.01 * rel + (g + 2) * 2.0 ** -24) * p.sum(0))


@pytest.mark.parametrize("page", [8, 16, 32])
@pytest.mark.parametrize("append", [True, False])
def test_attention4_of_long_units_with_pages_that_are_none(page, append):
    """Every warp goes through more than 32 pages of a unit, one in thirty of which is none: rows of random codes, steps and least values."""
    from paper_2507_08143_b200 import binding as B
    gen = torch.Generator(device="cuda").manual_seed(page)
    heads, g, n = 8, 3, 150003
    per = -(-(n + 1) // page)
    pools = []
    for _ in range(2):
        pool = torch.randint(0, 256, (heads * per, page, 80), generator=gen, device="cuda", dtype=torch.uint8)
        s = (torch.randint(8, 16, (heads * per, page, 4), generator=gen, device="cuda") / 64.0)          # four significant bits
        lo = torch.randn(heads * per, page, 4, generator=gen, device="cuda").bfloat16() - 1
        pool[..., 64:] = torch.stack([s.bfloat16(), lo], -1).flatten(2).contiguous().view(torch.uint8)
        pools.append(pool)
    table = torch.randperm(heads * per, generator=gen, device="cuda").to(torch.int32).view(1, heads, 1, per)
    lost = torch.rand(1, heads, 1, per, generator=gen, device="cuda") < 1 / 30
    lost[..., -1] = False
    bad = torch.where(torch.rand(lost.shape, generator=gen, device="cuda") < 0.5, -1, heads * per).to(torch.int32)
    mass = torch.zeros(heads * per, page, device="cuda")
    cache = B.PagedCache4(*pools, torch.where(lost, bad, table).contiguous(), mass=mass)
    lengths = torch.full((1, heads, 1), n, dtype=torch.int32, device="cuda")
    q = (torch.randn(1, heads * g, 128, generator=gen, device="cuda") / 8).bfloat16()
    new = [torch.randn(1, heads, 128, generator=gen, device="cuda").bfloat16() for _ in range(2)] if append else [None, None]
    opt = B.decode_options(g, n + 1, accumulate=True)
    out, lse, status = torch.empty_like(q), torch.empty(1, heads * g, device="cuda"), torch.zeros(1, heads, 1, dtype=torch.int32, device="cuda")
    B.paged_attention(cache, 0, opt, q, lengths, out, B.alloc_paged_attention_workspace(cache, opt), k_new=new[0], v_new=new[1], lse_out=lse, status=status)
    assert torch.all(status == 8)                            # COMPACTOR_STATUS_PAGE
    assert not mass[table[lost].long()].any()                # nothing is written where no page is
    total, scale = n + append, float(np.float32(128 ** -0.5))
    for h in range(heads):
        def values(pool):                                    # of the rows as they are held now, the new token's among them
            rows = pool[table[0, h, 0].long()].flatten(0, 1)[:total]
            par = rows[:, 64:].contiguous().view(torch.bfloat16).double().view(-1, 4, 2)
            codes = torch.stack([rows[:, :64] & 15, rows[:, :64] >> 4], -1).flatten(1).double().view(-1, 4, 32)
            sc, lo = par[..., :1] * codes, par[..., 1:].expand_as(codes)
            return (sc + lo).flatten(1), (sc.abs() + lo.abs()).flatten(1)
        (k, ka), (v, va) = values(pools[0]), values(pools[1])
        rows, there = slice(h * g, (h + 1) * g), ~lost[0, h, 0].repeat_interleave(page)[:total]
        qq = q[0, rows].double()
        y = (scale * (qq @ k.T)).masked_fill(~there, float("-inf"))
        dy = 161 * 2.0 ** -23 * float((scale * (qq.abs() @ ka.T)).max())                 # as above
        p = torch.softmax(y, 1)
        rel = 2 * dy + 2 * 2.0 ** -22 + (total / 8 + 64) * 2.0 ** -24
        tol = (rel + 2.0 ** -16 + (total / 16 + 17) * 17 * 2.0 ** -23) * 1.01 * (p @ va) + 2.0 ** -8 * (p @ v).abs()
        assert torch.all((out[0, rows].double() - p @ v).abs() <= tol)
        want = torch.logsumexp(y, 1)
        assert torch.all((lse[0, rows].double() - want).abs() <= dy + rel + 2.0 ** -22 * want.abs())
        w = mass[table[0, h, 0].long()].flatten()[:total].double()
        assert torch.all((w - p.sum(0)).abs() <= (1.01 * rel + (g + 2) * 2.0 ** -24) * p.sum(0))
