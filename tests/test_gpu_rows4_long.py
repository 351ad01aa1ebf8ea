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
