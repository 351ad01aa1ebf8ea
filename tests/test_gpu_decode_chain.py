"""The operators around the paged cache as they are used together: norms with rotation of a prefill, its compression, the kept rows into pages
(of bf16 or in 4 bits), key bounds, and decoding steps that choose pages, attend to them and append, captured in one graph; and the calls that
the other tests do not make: queries at the ends of the range, workspaces between guard bands, the largest sizes."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from oracle import rows_oracle as ro
from tests import helpers as H
from tests.test_gpu_paged import attention_bounds, make_cache
from tests.test_gpu_rows4 import attention4_bounds, make_cache4, run_attention4

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("four", [False, True])
def test_prefill_compression_and_decoding_steps_in_a_graph(four):
    from paper_2507_08143_b200 import binding as B
    layers, heads, g, page, pages, steps = 2, 2, 4, 16, 5, 4
    seqlens, keep = [300, 190, 0], [150, 40, 0]
    T, batch, qh = sum(seqlens), 3, heads * g
    gen = torch.Generator(device="cuda").manual_seed(5)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda").bfloat16()
    freq = (10000.0 ** (-torch.arange(64, device="cuda", dtype=torch.float64) / 64)).float()
    qw, kw = rand(128).abs() + 0.5, rand(128).abs() + 0.5
    pos = torch.cat([torch.arange(n) for n in seqlens]).to(torch.int32).cuda()
    # ---- prefill: keys before and after the rotation, scores by the ones, pages with the others
    k_plain, k = (torch.empty(layers, heads, T, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    qkv = rand(layers, T, qh + 2 * heads, 128)
    v = qkv[:, :, qh + heads:].transpose(1, 2)
    q_all = torch.empty(layers, qh, T, 128, dtype=torch.bfloat16, device="cuda")
    for l in range(layers):
        B.norm_rope(qkv[l, :, :qh], qkv[l, :, qh:qh + heads], pos, freq, q_all[l].transpose(0, 1), k[l].transpose(0, 1), k_plain_out=k_plain[l].transpose(0, 1),
                    q_weight=qw, k_weight=kw)
    shape = B.Shape(layers, heads, 128, 48, seqlens)
    idx = torch.empty(layers, heads, sum(keep), dtype=torch.int32, device="cuda")
    dense = [torch.empty(layers, heads, sum(keep), 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    B.compress(shape, k_plain, k, v, B.make_sketch(1, 128, 48).cuda(), keep, idx, *dense, B.alloc_workspace(shape))
    room = max(keep) + steps
    n_pages = layers * heads * batch * -(-room // page)
    table = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32).view(layers, heads, batch, -1)
    pool = lambda: torch.zeros(n_pages, page, 80, dtype=torch.uint8, device="cuda") if four else torch.zeros(n_pages, page, 128, dtype=torch.bfloat16, device="cuda")
    Cache = B.PagedCache4 if four else B.PagedCache
    kp, vp, mass = pool(), pool(), torch.zeros(n_pages, page, device="cuda")
    positions = torch.zeros(n_pages, page, dtype=torch.int32, device="cuda")
    cache = Cache(kp, vp, table, mass=mass, positions=positions)
    lengths = torch.tensor([0, 0, -1], dtype=torch.int32, device="cuda").expand(layers, heads, batch).contiguous()
    B.paged_fill(cache, shape, k, v, keep, idx=idx, lengths=lengths, lengths_out=lengths)
    bounds = torch.zeros(n_pages, 2, 128, dtype=torch.bfloat16, device="cuda")
    B.paged_bounds(cache, lengths, bounds, room)
    back = [torch.empty_like(d) for d in dense]
    B.paged_read(cache, B.Shape(layers, heads, 128, 48, keep), lengths, *back)
    for d, b in zip(dense, back):
        if four:
            np.testing.assert_array_equal(H.bits(b), ro.f64_to_bf16_bits(ro.values4(ro.hold4(H.bits(d))).astype(np.float32)))
        else:
            assert torch.equal(d, b)
    # ---- a step, all layers: norm and rotation of the new rows, choice, attention; lengths and positions go on
    position = torch.tensor(seqlens, dtype=torch.int32, device="cuda")
    new = rand(layers, batch, qh + 2 * heads, 128)
    qr, kr = torch.empty(layers, batch, qh, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(layers, batch, heads, 128, dtype=torch.bfloat16, device="cuda")
    out, lse = torch.empty_like(qr), torch.empty(layers, batch, qh, device="cuda")
    chosen = [torch.zeros(1, heads, batch, pages, dtype=torch.int32, device="cuda") for _ in range(layers)]
    short = [torch.zeros(1, heads, batch, dtype=torch.int32, device="cuda") for _ in range(layers)]
    few = [Cache(kp, vp, c, mass=mass, positions=positions) for c in chosen]
    opt = B.decode_options(g, pages * page, accumulate=True)
    ws, ws_select = B.alloc_paged_attention_workspace(few[0], opt), B.alloc_paged_select_workspace(cache, room)

    def step():
        for l in range(layers):
            B.norm_rope(new[l, :, :qh], new[l, :, qh:qh + heads], position, freq, qr[l], kr[l], q_weight=qw, k_weight=kw)
            B.paged_select(cache, l, g, qr[l], lengths, bounds, chosen[l], short[l], ws_select, room, k_new=kr[l])
            B.paged_attention(few[l], 0, opt, qr[l], short[l], out[l], ws, k_new=kr[l], v_new=new[l, :, qh + heads:], new_positions=position, lse_out=lse[l])
        lengths.add_(1).sub_((lengths == 0).to(torch.int32))              # (-1 stays)
        position.add_(1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    state = [t.clone() for t in (kp, vp, mass, positions, bounds, lengths, position)]
    with torch.cuda.stream(side):
        step()                                                           # warm-up, undone
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for t, s in zip((kp, vp, mass, positions, bounds, lengths, position), state):
        t.copy_(s)
    # ---- the same in 64 bits, from the rows that the norm kernel made
    bits = (lambda t: t.cpu().numpy()) if four else H.bits
    host = dict(k=bits(kp).copy(), v=bits(vp).copy(), mass=mass.cpu().numpy().copy(), positions=positions.cpu().numpy().copy(), table=table.cpu().numpy())
    hb = H.bits(bounds)
    weights = host["mass"].astype(np.float64)
    for s in range(steps):
        new.normal_(generator=gen)
        n, at = lengths.cpu().numpy().copy(), position.cpu().numpy().copy()
        graph.replay()
        torch.cuda.synchronize()
        for l in range(layers):
            want, want_len, hb = ro.select(host, l, g, H.bits(qr[l]), n, hb, pages, 1, 1, H.bits(kr[l]), room)
            np.testing.assert_array_equal(chosen[l][0].cpu().numpy(), want)
            np.testing.assert_array_equal(short[l][0].cpu().numpy(), want_len)
            att = ro.attention4 if four else po.attention
            ref, ref_lse, after, info = att(dict(host, table=want[None]), 0, H.bits(qr[l]), want_len[None], np.float64(np.float32(128 ** -0.5)),
                                            k_new=H.bits(kr[l]), v_new=H.bits(new[l, :, qh + heads:]), new_positions=at, accumulate=True)
            weights += after["mass"] - host["mass"]
            host = dict(after, table=host["table"], mass=host["mass"])
            o, ls = out[l].double().cpu().numpy(), lse[l].double().cpu().numpy()
            assert set(info) == {(h, b) for h in range(heads) for b in range(batch) if n[l, h, b] >= 0}
            for (h, b), (slots, p, pv, mag) in info.items():
                r = slice(h * g, (h + 1) * g)
                dy, rel, tol = attention4_bounds(g, pv, ref[b, r], mag, 0.0, len(slots)) if four else attention_bounds(g, p, pv, ref[b, r], mag, 128 ** -0.5, 0.0, len(slots))
                assert np.all(np.abs(o[b, r] - ref[b, r]) <= tol) and np.all(np.abs(ls[b, r] - ref_lse[b, r]) <= dy + rel + 2.0 ** -22 * np.abs(ref_lse[b, r]))
        np.testing.assert_array_equal(bits(kp), host["k"])
        np.testing.assert_array_equal(bits(vp), host["v"])
    assert lengths.cpu().numpy().tolist() == [[[150 + steps, 40 + steps, -1]] * heads] * layers
    np.testing.assert_allclose(mass.cpu().numpy(), weights, atol=steps * g * 1e-4)
    # ---- and back to the budget, bounds once more
    budgets = torch.where(lengths > 0, lengths - steps, lengths)
    B.paged_evict(cache, lengths, budgets, lengths, room)
    B.paged_bounds(cache, lengths, bounds, room)
    host = dict(k=bits(kp), v=bits(vp), mass=mass.cpu().numpy(), positions=positions.cpu().numpy(), table=table.cpu().numpy())
    want = ro.bounds(host, list(np.ndindex(layers, heads, batch)), lengths.cpu().numpy(), hb)
    live = np.unique(host["table"][:, :, :2, : 40 // page])
    np.testing.assert_array_equal(H.bits(bounds)[live] & 0x7FFF, want[live] & 0x7FFF)


@pytest.mark.parametrize("q_scale", [0.0, 1e-30, 1e-6, 1e6, 1e15])
def test_attention4_queries_of_any_size(q_scale):
    """Scores far apart are a choice of one token, scores of 0 the mean of all; both exact at any size of the queries."""
    from paper_2507_08143_b200 import binding as B
    for g in (2, 12):
        host, cache, len_d = make_cache4([[[100, 33]]], 16, 1, 21)
        q = (q_scale * torch.randn(2, g, 128, generator=torch.Generator().manual_seed(3))).bfloat16()
        opt = B.decode_options(g, 200)
        out, lse = torch.empty(2, g, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(2, g, device="cuda")
        B.paged_attention(cache, 0, opt, q.cuda(), len_d, out, B.alloc_paged_attention_workspace(cache, opt), lse_out=lse)
        ref, ref_lse, _, info = ro.attention4(host, 0, H.bits(q), np.array([[[100, 33]]], np.int32), np.float64(np.float32(128 ** -0.5)))
        for b in range(2):
            at, p, pv, mag = info[(0, b)]
            if q_scale > 1e3:                                             # (the second best is far behind)
                assert np.sort(p, 1)[:, -2].max() < 1e-30
                pv, mag = np.abs(ref[b]), 0.0
            dy, rel, tol = attention4_bounds(g, pv, ref[b], mag, 0.0, len(at))
            assert np.all(np.abs(out[b].double().cpu().numpy() - ref[b]) <= tol)
            if q_scale < 1e3:
                assert np.all(np.abs(lse[b].double().cpu().numpy() - ref_lse[b]) <= dy + rel + 2.0 ** -22 * np.abs(ref_lse[b]))


def test_attention4_scales_at_the_ends_of_the_range():
    from paper_2507_08143_b200 import binding as B
    _, cache, len_d = make_cache4([[[50, 0]]], 16, 1, 22)
    q = torch.randn(2, 2, 128).bfloat16().cuda()
    for scale, softcap in ((2e-38, 0.0), (1e30, 0.0), (1e-30, 1e-5), (1e10, 1e5)):
        opt = B.decode_options(2, 51, scale=scale, softcap=softcap)
        out = torch.full((2, 2, 128), 7.0, dtype=torch.bfloat16, device="cuda")
        B.paged_attention(cache, 0, opt, q, len_d, out, B.alloc_paged_attention_workspace(cache, opt))
        assert torch.isfinite(out).all() and torch.all(out[1] == 0)


def test_workspaces_between_guard_bands():
    """No call writes outside the bytes that it asked for."""
    from paper_2507_08143_b200 import binding as B
    lens = np.array([[[500, 0, 77, 1500], [20, 333, -1, 64]]], np.int32)
    for four in (False, True):
        _, cache, len_d = (make_cache4 if four else make_cache)(lens, 16, 1, 30)
        for g in (4, 7, 20):
            for accumulate in (False, True):
                opt = B.decode_options(g, 1501, accumulate=accumulate)
                size = B.paged_attention_workspace_bytes(cache, opt)
                ws = torch.full((size + 8192,), 171, dtype=torch.uint8, device="cuda")
                q = torch.randn(4, 2 * g, 128, device="cuda").bfloat16()
                B.paged_attention(cache, 0, opt, q, len_d, torch.empty_like(q), ws[4096:4096 + size])
                assert torch.all(ws[:4096] == 171) and torch.all(ws[4096 + size:] == 171)
        size = B.paged_select_workspace_bytes(cache, 1501)
        ws = torch.full((size + 8192,), 171, dtype=torch.uint8, device="cuda")
        bounds = torch.randn(cache.n_pages + 2, 2, 128, device="cuda").bfloat16()
        kept = bounds.clone()
        table, short = torch.full((3, 2, 4, 7), 5, dtype=torch.int32, device="cuda"), torch.full((3, 2, 4), 5, dtype=torch.int32, device="cuda")
        q, kn = torch.randn(4, 8, 128, device="cuda").bfloat16(), torch.randn(4, 2, 128, device="cuda").bfloat16()
        B.paged_select(cache, 0, 4, q, len_d, bounds[1:-1], table[1:2], short[1:2], ws[4096:4096 + size], 1501, k_new=kn)
        assert torch.all(ws[:4096] == 171) and torch.all(ws[4096 + size:] == 171)
        assert torch.all(table[0] == 5) and torch.all(table[2] == 5) and torch.all(short[0] == 5) and torch.all(short[2] == 5)
        changed = (bounds != kept).flatten(1).any(1)
        assert not changed[0] and not changed[-1] and int(changed.sum()) <= 7          # one page per unit that has a sequence
        B.paged_bounds(cache, len_d, bounds[1:-1], 1501)
        assert torch.equal(bounds[0], kept[0]) and torch.equal(bounds[-1], kept[-1])


def test_select_of_the_most_pages_a_unit_may_have():
    from paper_2507_08143_b200 import binding as B
    pages = 49152
    table = torch.arange(pages, dtype=torch.int32, device="cuda").view(1, 1, 1, -1)
    pool = torch.zeros(pages, 8, 80, dtype=torch.uint8, device="cuda")
    cache = B.PagedCache4(pool, pool, table)
    gen = torch.Generator(device="cuda").manual_seed(1)
    bounds = torch.randn(pages, 2, 128, generator=gen, device="cuda").bfloat16().sort(1).values
    bounds[20000:30000] = bounds[20000]                                   # ten thousand pages alike
    q = torch.randn(1, 3, 128, generator=gen, device="cuda").bfloat16()
    n = torch.tensor([[[pages * 8]]], dtype=torch.int32, device="cuda")
    ws = B.alloc_paged_select_workspace(cache, pages * 8)
    b, x = bounds.double(), q[0].double()
    score = (torch.where(x[:, None] > 0, b[None, :, 1], b[None, :, 0]) * x[:, None]).sum(-1).amax(0).float()
    alike = int((score > score[20000]).sum())
    for count in (2, 100, alike + 500, 40000, pages - 1, pages):
        score[0] = score[-1] = float("inf")
        want = torch.argsort(score, descending=True, stable=True)[:count].sort().values.to(torch.int32)
        out, short = torch.empty(1, 1, 1, count, dtype=torch.int32, device="cuda"), torch.empty(1, 1, 1, dtype=torch.int32, device="cuda")
        B.paged_select(cache, 0, 3, q, n, bounds, out, short, ws, pages * 8)
        assert torch.equal(out.view(-1), want), count
        assert int(short) == count * 8


def test_random_batches():
    """Every size drawn; both kinds of cache."""
    from paper_2507_08143_b200 import binding as B
    rng = np.random.default_rng(77)
    for case in range(12):
        page, g = int(rng.choice([8, 16, 32, 64])), int(rng.integers(1, 20))
        lens = rng.integers(-1, int(rng.choice([20, 300, 900])), size=(1, int(rng.integers(1, 4)), int(rng.integers(1, 9)))).astype(np.int32)
        lens[0, 0, 0] = abs(int(lens[0, 0, 0]))
        run_attention4(lens, g, page, accumulate=bool(rng.integers(2)), append=bool(rng.integers(2)), softcap=float(rng.choice([0.0, 30.0])), strided=bool(rng.integers(2)),
                       seed=case)
