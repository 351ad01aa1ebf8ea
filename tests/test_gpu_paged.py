"""The paged cache on the GPU: fill, attention of one new token and eviction against the fp64 statements of oracle/paged_oracle.py.

Unused slots of the pools hold not-a-numbers, the page table holds ids outside the pool behind every unit's last page, and
every pool is compared whole, so that a read or write outside a unit's tokens shows."""
import math

import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from tests import helpers as H

pytestmark = pytest.mark.gpu
NAN_BITS = 0x7FC1


def make_cache(lengths, page, room, seed, strided=False, spare=3):
    """A cache whose units can hold lengths + room tokens; values in the first `length` slots, NaN in all others.
    lengths: int array [layers, heads, batch] (negative: no sequence)."""
    lengths = np.asarray(lengths, np.int32)
    rng = np.random.default_rng(seed)
    cap = np.maximum(lengths, 0) + room
    pages = np.maximum(1, -(-cap // page))
    n_pages, max_pages = int(pages.sum()) + spare, int(pages.max()) + 1
    ids = rng.permutation(n_pages)[: pages.sum()]
    table = np.full(lengths.shape + (max_pages,), 0, np.int32)
    table[...] = rng.choice([-1, n_pages, 2 ** 31 - 1, -2 ** 31], size=table.shape)
    at = 0
    for u in np.ndindex(lengths.shape):
        table[u][: pages[u]] = ids[at: at + pages[u]]
        at += pages[u]
    g = torch.Generator().manual_seed(seed)
    pools = []
    for _ in range(2):
        x = torch.full((n_pages, page, 128), float("nan"), dtype=torch.bfloat16)
        pools.append(x)
    mass = torch.full((n_pages, page), float("nan"))
    pos = torch.full((n_pages, page), -7, dtype=torch.int32)
    for u in np.ndindex(lengths.shape):
        for j in range(pages[u]):
            n = min(page, int(lengths[u]) - j * page)
            if n > 0:
                p = int(table[u][j])
                pools[0][p, :n] = torch.randn(n, 128, generator=g).bfloat16()
                pools[0][p, :n, 5] *= 4                                  # a strong channel
                pools[1][p, :n] = torch.randn(n, 128, generator=g).bfloat16()
                mass[p, :n] = torch.rand(n, generator=g) * 3
                pos[p, :n] = torch.arange(j * page, j * page + n, dtype=torch.int32) * 2
    host = dict(k=H.bits(pools[0]), v=H.bits(pools[1]), mass=mass.numpy().copy(), positions=pos.numpy().copy(), table=table)
    if strided:                                                          # K and V interleaved per page, rows with a gap
        both = torch.full((n_pages, 2, page, 144), float("nan"), dtype=torch.bfloat16, device="cuda")
        both[:, 0, :, 8:136] = pools[0].cuda(); both[:, 1, :, 8:136] = pools[1].cuda()
        kd, vd = both[:, 0, :, 8:136], both[:, 1, :, 8:136]
    else:
        kd, vd = pools[0].cuda(), pools[1].cuda()
    from paper_2507_08143_b200 import binding as B
    cache = B.PagedCache(kd, vd, torch.from_numpy(table).cuda(), mass=mass.cuda(), positions=pos.cuda())
    return host, cache, torch.from_numpy(lengths).cuda()


def pools_of(cache):
    k, v, _, mass, pos = cache.tensors
    return dict(k=H.bits(k), v=H.bits(v), mass=mass.cpu().numpy(), positions=pos.cpu().numpy())


def same_bits(got, want, what):
    for name in ("k", "v", "positions"):
        np.testing.assert_array_equal(got[name], want[name], err_msg=f"{what}: {name}")


def attention_bounds(g, p, pv, out, mag, scale, softcap, n):
    """Derived bounds of one (KV head, sequence).  mag: largest scale * sum |q||k|.
    scores: eight accumulations of 16 products; every one may drop a unit of 2^-23 of the largest partial sum for each of its 17
      summands: |dy| <= 8 * 17 * 2^-23 * mag; the cap's derivative is at most 1 and tanhf adds 2^-22 of the cap (2 ulp);
      the scaling to base 2 and the difference to the maximum round once each: 3 * 2^-24 * |y|, |y| <= mag.
    weights: e^dy, ex2 2^-22, and the sum of n terms in fp32 along at most n / 8 + 64 additions: 2^-24 each.
    out: the weights rounded to bf16 (2^-8 each) times |v|, the accumulation over n tokens in fp32 (17 * 2^-23 per 16 tokens), and
      the result rounded once to bf16 (2^-8)."""
    dy = (8 * 17 + 2) * 2.0 ** -23 * mag + (softcap * 2.0 ** -22 if softcap else 0.0)
    rel = 2 * dy + 2 * 2.0 ** -22 + (n / 8 + 64) * 2.0 ** -24
    rel_out = rel + 2.0 ** -8 + (n / 16 + 16) * 17 * 2.0 ** -23
    return dy, rel, rel_out * 1.01 * pv + 2.0 ** -8 * np.abs(out) + 1e-30


def run_attention(lengths, g, page, accumulate=False, softcap=0.0, append=True, strided=False, room=1, seed=0, layer=0, status=True,
                  max_length=None, scale=128 ** -0.5, positions=True, q_scale=1.5):
    from paper_2507_08143_b200 import binding as B
    lengths = np.asarray(lengths, np.int32)
    _, heads, batch = lengths.shape
    host, cache, len_d = make_cache(lengths, page, room, seed, strided)
    gen = torch.Generator().manual_seed(seed + 1)
    q = (q_scale * torch.randn(batch, heads * g, 128, generator=gen)).bfloat16()
    kn, vn = torch.randn(batch, heads, 128, generator=gen).bfloat16(), torch.randn(batch, heads, 128, generator=gen).bfloat16()
    newpos = torch.arange(batch, dtype=torch.int32) + 1000
    limit = int(max(1, lengths.max() + 1)) if max_length is None else max_length
    opt = B.decode_options(g, limit, scale=scale, softcap=softcap, accumulate=accumulate)
    ws = torch.full((max(256, B.paged_attention_workspace_bytes(cache, opt)),), 255, dtype=torch.uint8, device="cuda")   # NaN everywhere
    if strided:                                                          # heads before sequences, rows with a gap
        qd = torch.zeros(heads * g, batch, 136, dtype=torch.bfloat16, device="cuda")[..., :128].transpose(0, 1)
        qd.copy_(q)
        out_all = torch.full((heads * g, batch, 136), 7.0, dtype=torch.bfloat16, device="cuda")
        out = out_all[..., :128].transpose(0, 1)
    else:
        qd, out = q.cuda(), torch.full((batch, heads * g, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((batch, heads * g), 7.0, device="cuda")
    st = torch.full(lengths.shape, 99, dtype=torch.int32, device="cuda") if status else None
    extra = dict(k_new=kn.cuda(), v_new=vn.cuda(), new_positions=newpos.cuda() if positions else None) if append else {}
    B.paged_attention(cache, layer, opt, qd, len_d, out, ws, lse_out=lse, status=st, **extra)
    torch.cuda.synchronize()
    okw = dict(k_new=H.bits(kn), v_new=H.bits(vn), new_positions=newpos.numpy() if positions else None) if append else {}
    ref_out, ref_lse, after, info = po.attention(host, layer, H.bits(q), lengths, np.float64(np.float32(scale)), softcap=softcap,
                                                 accumulate=accumulate, max_length=limit, **okw)
    o, ls = out.float().cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)
    got = pools_of(cache)
    same_bits(got, after, "pools")
    mass_tol = np.zeros_like(after["mass"])
    for h in range(heads):
        for b in range(batch):
            rows = slice(h * g, (h + 1) * g)
            if (h, b) not in info:
                assert np.all(o[b, rows] == 0) and np.all(ls[b, rows] == -np.inf), (h, b)
                continue
            at, p, pv, mag = info[(h, b)]
            dy, rel, tol = attention_bounds(g, p, pv, ref_out[b, rows], mag, scale, softcap, len(at))
            err = np.abs(o[b, rows] - ref_out[b, rows])
            assert np.all(err <= tol), f"out (h={h}, b={b}): {np.max(err / tol):.2f} of the bound"
            lse_tol = dy + rel + 2.0 ** -22 * np.abs(ref_lse[b, rows])
            assert np.all(np.abs(ls[b, rows] - ref_lse[b, rows]) <= lse_tol), f"lse (h={h}, b={b})"
            if accumulate:
                for j, a in enumerate(at):
                    if a is not None:                        # every head's weight, the sum of g of them and the addition
                        mass_tol[a] = (1.01 * rel + (g + 2) * 2.0 ** -24) * p[:, j].sum() + 2.0 ** -24 * abs(after["mass"][a])
    live = ~np.isnan(after["mass"])
    assert np.array_equal(live, ~np.isnan(got["mass"]))
    err = np.abs(got["mass"].astype(np.float64) - after["mass"])[live]
    assert np.all(err <= mass_tol[live]), f"weights: {np.max(err):.3e}"
    if strided:
        pad = out_all[..., 128:].float()
        assert torch.all(pad == 7.0)
    return host, cache, after, st, out, lse


LENGTHS = {
    "one": [[[0]]], "empty": [[[0, -1]]], "tile": [[[15, 16, 17]]], "short": [[[1, 0, -1, 33], [2, 31, 32, 7]]],
    "ragged": [[[700, 3, 0, 129], [-1, 64, 255, 1000]]], "long": [[[9001]]], "two layers": [[[5, 6]], [[40, 0]]],
}


@pytest.mark.parametrize("name", list(LENGTHS))
@pytest.mark.parametrize("append", [True, False])
@pytest.mark.parametrize("accumulate", [True, False])
def test_attention_lengths(name, append, accumulate):
    lengths = np.array(LENGTHS[name], np.int32)
    run_attention(lengths, 4, 16, accumulate=accumulate, append=append, layer=lengths.shape[0] - 1)


@pytest.mark.parametrize("g", [1, 2, 3, 7, 8, 9, 15, 16, 17, 33, 64])
def test_attention_head_layouts(g):
    run_attention([[[37, 0, 210], [16, 90, -1]]], g, 16, accumulate=True, seed=g)
    run_attention([[[400]]], g, 32, accumulate=False, seed=g + 100)


@pytest.mark.parametrize("page", [8, 16, 32, 128, 1024])
def test_attention_page_sizes_and_strides(page):
    run_attention([[[1, 100, 1023, 7], [2 * page, page - 1, page + 1, 3 * page]]], 5, page, accumulate=True, strided=True, seed=page)


@pytest.mark.parametrize("softcap", [0.5, 30.0, 50.0])
def test_attention_capped_scores(softcap):
    run_attention([[[300, 17, 0], [64, 1, 129]]], 3, 16, accumulate=True, softcap=softcap, seed=5, q_scale=6.0)


def test_attention_many_units_and_one_long_one():
    rng = np.random.default_rng(8)
    lengths = rng.integers(-1, 70, size=(1, 4, 130)).astype(np.int32)    # more units than threads of a block
    lengths[0, 2, 77] = 6000
    run_attention(lengths, 2, 16, accumulate=True, seed=8)


def test_attention_without_status_lse_positions():
    run_attention([[[20, 3]]], 2, 8, status=False, positions=False)


def test_attention_length_beyond_the_bound_or_the_pages():
    # 50 + 1 tokens against max_length 40: refused, flagged, its page untouched; its neighbours are served
    _, _, _, st, _, _ = run_attention([[[50, 39, 40, 10]]], 2, 16, accumulate=True, max_length=40)
    assert st.cpu().tolist() == [[[16, 0, 16, 0]]]
    # no page left for the new token
    _, cache, _, st, _, _ = run_attention([[[64, 5]]], 2, 16, room=0, max_length=1000)
    # (the table has one more column than the longest unit needs: the token is attended to, its page is none)
    assert st.cpu().tolist() == [[[8, 0]]]


def test_attention_leaves_out_tokens_on_pages_that_are_none():
    from paper_2507_08143_b200 import binding as B
    for page in (8, 16):
        host, cache, len_d = make_cache([[[100, 40]]], page, 1, 3)
        for tbl in (host["table"], cache.tensors[2]):
            tbl[0, 0, 0, 2] = -5
            tbl[0, 0, 0, 4] = 10 ** 9
        q = torch.randn(2, 4, 128).bfloat16()
        opt = B.decode_options(4, 200, accumulate=True)
        out, lse = torch.empty(2, 4, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(2, 4, device="cuda")
        st = torch.zeros(1, 1, 2, dtype=torch.int32, device="cuda")
        B.paged_attention(cache, 0, opt, q.cuda(), len_d, out, B.alloc_paged_attention_workspace(cache, opt), lse_out=lse, status=st)
        ref, ref_lse, after, info = po.attention(host, 0, H.bits(q), np.array([[[100, 40]]], np.int32), 128 ** -0.5, accumulate=True)
        for b in range(2):
            at, p, pv, mag = info[(0, b)]
            dy, rel, tol = attention_bounds(4, p, pv, ref[b], mag, 128 ** -0.5, 0.0, len(at))
            assert np.all(np.abs(out[b].float().cpu().numpy() - ref[b]) <= tol)
            assert np.all(np.abs(lse[b].cpu().numpy() - ref_lse[b]) <= dy + rel + 2.0 ** -22 * np.abs(ref_lse[b]))
        got = cache.tensors[3].cpu().numpy()
        assert np.array_equal(np.isnan(got), np.isnan(after["mass"]))
        assert np.nanmax(np.abs(got - after["mass"])) < 1e-4
        assert st.cpu().tolist() == [[[8, 0]]]


def test_attention_infinite_and_nan_values_stay_in_their_unit():
    from paper_2507_08143_b200 import binding as B
    host, cache, len_d = make_cache([[[60, 60, 60]]], 16, 1, 4)
    p = host["table"][0, 0, 1, 1]
    cache.tensors[1][p, 3, 9] = float("inf")                              # one value of one unit's V
    p2 = host["table"][0, 0, 2, 0]
    cache.tensors[0][p2, 2] = float("nan")                               # a key of another unit
    q = torch.randn(3, 2, 128).bfloat16().cuda()
    opt = B.decode_options(2, 61)
    out = torch.empty(3, 2, 128, dtype=torch.bfloat16, device="cuda")
    B.paged_attention(cache, 0, opt, q, len_d, out, B.alloc_paged_attention_workspace(cache, opt))
    o = out.float().cpu()
    assert torch.isfinite(o[0]).all() and torch.isnan(o[2]).all()
    assert torch.isinf(o[1, :, 9]).all() and torch.isfinite(o[1, :, :9]).all() and torch.isfinite(o[1, :, 10:]).all()


def test_attention_is_reproducible_and_replays_from_a_graph():
    # a captured call follows lengths, queries and new tokens that change between replays; two runs give the same bits
    from paper_2507_08143_b200 import binding as B
    lens = np.array([[[500, 0, 77, 1500], [20, 333, -1, 64]]], np.int32)
    host, cache, len_d = make_cache(lens, 16, 8, 11)
    g = 4
    q = torch.randn(4, 2 * g, 128, device="cuda").bfloat16()
    kn, vn = torch.randn(4, 2, 128, device="cuda").bfloat16(), torch.randn(4, 2, 128, device="cuda").bfloat16()
    opt = B.decode_options(g, 1600, accumulate=True)
    ws = B.alloc_paged_attention_workspace(cache, opt)
    out, lse = torch.empty_like(q), torch.empty(4, 2 * g, device="cuda")
    start = [t.clone() for t in cache.tensors]

    def call(stream_out, stream_lse, w):
        B.paged_attention(cache, 0, opt, q, len_d, stream_out, w, k_new=kn, v_new=vn, lse_out=stream_lse)
    call(out, lse, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out, lse, ws)
    for step in range(3):
        q.normal_(); kn.normal_(); vn.normal_()
        len_d.copy_(torch.from_numpy(np.where(lens >= 0, lens + step, lens)))
        snap = []
        for replay in (True, False):
            for t, s in zip(cache.tensors, start):
                t.copy_(s)
            if replay:
                graph.replay()
                o, ls = out.clone(), lse.clone()
            else:
                o, ls = torch.empty_like(out), torch.empty_like(lse)
                call(o, ls, torch.full_like(ws, 255))
            torch.cuda.synchronize()
            snap.append([o, ls] + [t.clone() for t in cache.tensors])
        for a, b in zip(*snap):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_attention_on_two_streams_at_once():
    # two layers of one cache, a workspace each, on two streams: as one after the other
    from paper_2507_08143_b200 import binding as B
    lens = np.full((2, 4, 3), 900, np.int32)
    _, cache, len_d = make_cache(lens, 16, 1, 12)
    q = torch.randn(2, 3, 16, 128, device="cuda").bfloat16()
    opt = B.decode_options(4, 901, accumulate=True)
    ws = [B.alloc_paged_attention_workspace(cache, opt) for _ in range(2)]
    out = torch.empty(2, 2, 3, 16, 128, dtype=torch.bfloat16, device="cuda")
    mass0 = cache.tensors[3].clone()
    for l in range(2):
        B.paged_attention(cache, l, opt, q[l], len_d, out[0, l], ws[l])
    torch.cuda.synchronize()
    mass1 = cache.tensors[3].clone()
    cache.tensors[3].copy_(mass0)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for l in range(2):
        with torch.cuda.stream(streams[l]):
            B.paged_attention(cache, l, opt, q[l], len_d, out[1, l], ws[l])
    torch.cuda.synchronize()
    assert torch.equal(out[0], out[1]) and torch.equal(mass1.view(torch.int32), cache.tensors[3].view(torch.int32))


def test_attention_rows_beyond_32_bit_offsets():
    # one pool of 4.3e9 elements, read as K and as V; the pages in use are the last ones
    from paper_2507_08143_b200 import binding as B
    page, n_pages = 1024, 33000
    pool = torch.empty(n_pages, page, 128, dtype=torch.bfloat16, device="cuda")
    assert pool.numel() > 2 ** 32
    table = torch.tensor([[[[n_pages - 1, n_pages - 2]]]], dtype=torch.int32, device="cuda")
    pool[-2:] = torch.randn(2, page, 128, device="cuda").bfloat16()
    cache = B.PagedCache(pool, pool, table)
    q = torch.randn(1, 2, 128, device="cuda").bfloat16()
    opt = B.decode_options(2, 2048)
    out = torch.empty_like(q)
    n = torch.tensor([[[1500]]], dtype=torch.int32, device="cuda")
    B.paged_attention(cache, 0, opt, q, n, out, B.alloc_paged_attention_workspace(cache, opt))
    rows = torch.cat([pool[-1], pool[-2]])[:1500].double()
    p = torch.softmax(q[0].double() @ rows.T * 128 ** -0.5, 1)
    ref = p @ rows
    tol = 2 * 2.0 ** -8 * (p @ rows.abs()) + 2.0 ** -8 * ref.abs()
    assert torch.all((out[0].double() - ref).abs() <= tol)


# ------------------------------------------------------------------------------------------------ fill
def _prefill(layers, heads, seqlens, seed):
    g = torch.Generator().manual_seed(seed)
    T = sum(seqlens)
    return [torch.randn(layers, heads, T, 128, generator=g).bfloat16() for _ in range(2)] + [torch.rand(layers, heads, T, generator=g)]


def run_fill(seqlens, keep, page, layers=2, heads=2, cache_layers=2, first_layer=0, across=False, use_idx=True, held=None, strided=False,
             mass=True, first=True, seed=0, alias=True, room=None, bad_idx=False):
    from paper_2507_08143_b200 import binding as B
    batch = len(seqlens)
    rng = np.random.default_rng(seed)
    held = np.zeros((cache_layers, heads, batch), np.int32) if held is None else np.asarray(held, np.int32)
    host, cache, _ = make_cache(held, page, (max(keep) * (heads if across else 1) if room is None else room), seed, strided)
    k, v, attn = _prefill(layers, heads, seqlens, seed)
    cu, ck = np.concatenate([[0], np.cumsum(seqlens)]), np.concatenate([[0], np.cumsum(keep)])
    rows = {}
    idx = offs = None
    if across:
        idx, offs = np.zeros((layers, heads * sum(keep)), np.int32), np.zeros((layers, batch, heads + 1), np.int32)
        for l in range(layers):
            for b in range(batch):
                pick = np.sort(rng.permutation(heads * seqlens[b])[: heads * keep[b]])
                idx[l, heads * ck[b]: heads * ck[b + 1]] = pick % max(1, seqlens[b])
                offs[l, b, 1:] = np.searchsorted(pick, (np.arange(heads) + 1) * seqlens[b])
                for h in range(heads):
                    rows[l, h, b] = idx[l, heads * ck[b] + offs[l, b, h]: heads * ck[b] + offs[l, b, h + 1]]
    elif use_idx:
        idx = np.zeros((layers, heads, sum(keep)), np.int32)
        for (l, h, b) in np.ndindex(layers, heads, batch):
            pick = np.sort(rng.permutation(seqlens[b])[: keep[b]]).astype(np.int32)
            if bad_idx and keep[b] > 2:
                pick[1], pick[2] = -1, seqlens[b]
            idx[l, h, ck[b]:ck[b + 1]] = pick
            rows[l, h, b] = pick
    else:
        rows = {(l, h, b): np.arange(keep[b]) for (l, h, b) in np.ndindex(layers, heads, batch)}
    fp = rng.integers(0, 1000, batch).astype(np.int32)
    shape = B.Shape(layers, heads, 128, 48, seqlens)
    len_in = torch.from_numpy(held).cuda()
    len_out = len_in if alias else torch.full_like(len_in, -3)
    st = torch.full(held.shape, 99, dtype=torch.int32, device="cuda")
    kd, vd = k.cuda(), v.cuda()
    if strided:                                                          # tokens outside heads, as a model's projection leaves them
        kd = kd.transpose(1, 2).contiguous().transpose(1, 2)
        vd = torch.stack([vd, vd], 3)[:, :, :, 1]
    B.paged_fill(cache, shape, kd, vd, keep, idx=None if idx is None else torch.from_numpy(idx).cuda(),
                 head_offsets=None if offs is None else torch.from_numpy(offs).cuda(), mass_in=attn.cuda() if mass else None,
                 first_position=torch.from_numpy(fp).cuda() if first else None, lengths=len_in, lengths_out=len_out, first_layer=first_layer,
                 status=st)
    torch.cuda.synchronize()
    want, want_len = po.fill(host, first_layer, H.bits(k), H.bits(v), cu, lambda l, h, b: rows[l, h, b], attn.numpy() if mass else None,
                             fp if first else None, held)
    got = pools_of(cache)
    same_bits(got, want, "fill")
    np.testing.assert_array_equal(got["mass"].view(np.uint32), want["mass"].view(np.uint32))
    mine = slice(first_layer, first_layer + layers)
    np.testing.assert_array_equal(len_out.cpu().numpy()[mine], want_len[mine])
    others = np.ones(cache_layers, bool); others[mine] = False
    assert np.all(len_out.cpu().numpy()[others] == (held[others] if alias else -3))
    assert np.all(st.cpu().numpy()[others] == 99)
    return st.cpu().numpy(), got, host


@pytest.mark.parametrize("page", [8, 16, 256])
@pytest.mark.parametrize("across", [False, True])
def test_fill_with_a_selection(page, across):
    run_fill([100, 1, 0, 257, 40], [30, 1, 0, 200, 40], page, across=across, seed=page)
    run_fill([64, 31], [7, 31], page, layers=1, cache_layers=3, first_layer=1, heads=3, across=across, strided=True, alias=False, seed=page + 1)


def test_fill_appends_behind_what_is_held():
    held = np.array([[[5, 0, -1], [16, 15, 3]], [[0, 1, 2], [31, -4, 8]]])
    run_fill([4, 33, 6], [4, 20, 6], 16, held=held, seed=3)
    run_fill([4, 33, 6], [4, 33, 6], 8, held=held, use_idx=False, mass=False, first=False, seed=4)
    run_fill([1, 1, 1], [1, 1, 1], 8, held=held, use_idx=False, seed=5)


def test_fill_skips_bad_rows_and_refuses_units_without_room():
    run_fill([50, 20], [10, 9], 16, bad_idx=True, seed=6)
    held = np.array([[[30, 0], [0, 7]]])                                 # the table has three pages of 16
    st, _, _ = run_fill([40, 40], [40, 33], 16, layers=1, cache_layers=1, held=held, use_idx=False, room=0, seed=7)
    assert st[0, 0, 0] & 16                                              # 30 + 40 tokens do not fit
    assert st[0, 0, 1] == 8                                              # fits the table, but only its first page is one


def test_fill_without_any_tokens():
    from paper_2507_08143_b200 import binding as B
    _, cache, len_d = make_cache([[[4, -1]]], 8, 2, 8)
    before = pools_of(cache)
    empty = torch.empty(1, 1, 0, 128, dtype=torch.bfloat16, device="cuda")
    out = torch.full_like(len_d, 9)
    B.paged_fill(cache, B.Shape(1, 1, 128, 48, [0, 0]), empty, empty, [0, 0], lengths=len_d, lengths_out=out)
    assert out.cpu().tolist() == [[[4, -1]]]
    same_bits(pools_of(cache), before, "nothing")


def test_fill_of_more_sequences_than_one_launch_takes():
    rng = np.random.default_rng(9)
    n = rng.integers(0, 20, 600).tolist()
    run_fill(n, [int(rng.integers(0, x + 1)) for x in n], 8, layers=1, cache_layers=1, heads=1, seed=9)
    run_fill(n, [int(rng.integers(0, x + 1)) for x in n], 8, layers=1, cache_layers=1, heads=2, across=True, seed=10)


# ------------------------------------------------------------------------------------------------ evict
def run_evict(lengths, budgets, page=16, recent=0, seed=0, weights=None, positions=None, max_length=None, layer_range=None, alias=False, strided=False, next_position=None):
    from paper_2507_08143_b200 import binding as B
    lengths, budgets = np.asarray(lengths, np.int32), np.asarray(budgets, np.int32)
    host, cache, len_d = make_cache(lengths, page, 0, seed, strided)
    if weights is not None:
        for u in np.ndindex(lengths.shape):
            for t in range(max(0, int(lengths[u]))):
                host["mass"][po.slot_of(host, u, t)] = weights(u, t)
        cache.tensors[3].copy_(torch.from_numpy(host["mass"]))
    if positions is not None:
        for u in np.ndindex(lengths.shape):
            for t in range(max(0, int(lengths[u]))):
                host["positions"][po.slot_of(host, u, t)] = positions(u, t)
        cache.tensors[4].copy_(torch.from_numpy(host["positions"]))
    nxt = np.full(lengths.shape[2], 2 * max(1, int(lengths.max())), np.int32) if next_position is None else np.asarray(next_position, np.int32)
    bound = int(max(1, lengths.max())) if max_length is None else max_length
    out = len_d if alias else torch.full_like(len_d, -9)
    st = torch.full(lengths.shape, 99, dtype=torch.int32, device="cuda")
    first, count = layer_range or (0, lengths.shape[0])
    B.paged_evict(cache, len_d, torch.from_numpy(budgets).cuda(), out, bound, recent=recent, next_position=torch.from_numpy(nxt).cuda() if recent else None,
                  first_layer=first, layers=count, status=st)
    torch.cuda.synchronize()
    units = [u for u in np.ndindex(lengths.shape) if first <= u[0] < first + count]
    want, want_len = po.evict(host, units, lengths, budgets, recent, nxt, bound)
    got = pools_of(cache)
    same_bits(got, want, "evict")
    np.testing.assert_array_equal(got["mass"].view(np.uint32), want["mass"].view(np.uint32))
    np.testing.assert_array_equal(out.cpu().numpy()[first:first + count], want_len[first:first + count])
    return st.cpu().numpy()


@pytest.mark.parametrize("page", [8, 16, 512])
@pytest.mark.parametrize("recent", [0, 1, 20])
def test_evict_ragged(page, recent):
    lengths = [[[100, 0, 1, -1, 33], [500, 64, 65, 31, 2]], [[7, 1500, 32, 40, 90], [21, 22, 23, 24, 25]]]
    budgets = [[[60, 5, 0, 3, 32], [499, 64, 30, -1, 1]], [[0, 700, 1, 39, 20], [20, 20, 20, 20, 20]]]
    run_evict(lengths, budgets, page, recent, seed=page + recent)


def test_evict_of_a_range_of_layers_in_place():
    lengths = np.full((3, 2, 2), 80, np.int32)
    st = run_evict(lengths, np.full((3, 2, 2), 50), recent=8, layer_range=(1, 1), alias=True, strided=True)
    assert np.all(st[[0, 2]] == 99) and np.all(st[1] == 0)


@pytest.mark.parametrize("n", [33, 5000, 20000])
def test_evict_equal_weights_keep_the_lower_slots(n):
    run_evict([[[n, n, n]]], [[[n // 2, n - 1, 1]]], weights=lambda u, t: 1.0, seed=n)
    run_evict([[[n, n]]], [[[n // 3, n - 2]]], weights=lambda u, t: float(t % 3), seed=n + 1)
    run_evict([[[n]]], [[[n // 2]]], weights=lambda u, t: [0.0, -0.0][t % 2], recent=10, seed=n + 2)


def test_evict_special_weights():
    vals = [float("nan"), float("inf"), 1.0, -1.0, 0.0, 1e-45, -1e-45, float("-inf"), 3e38, -3e38, -float("nan")]
    for b in (1, 3, 30, 60, 90, 109):
        run_evict([[[110]]], [[[b]]], weights=lambda u, t: vals[(t * 7) % 11], seed=b)


def test_evict_recent_window_wider_than_the_budget_and_repeated_positions():
    run_evict([[[50, 50]]], [[[10, 49]]], recent=40, seed=1)
    run_evict([[[50]]], [[[10]]], recent=10, positions=lambda u, t: 99, next_position=[100], seed=2)
    run_evict([[[50]]], [[[10]]], recent=10, positions=lambda u, t: 7 * t % 50, next_position=[50], seed=3)


@pytest.mark.parametrize("n,b", [(40000, 39999), (40000, 20000), (120000, 50000), (262144, 262000)])
def test_evict_long_units_shared_by_a_cluster(n, b):
    rng = np.random.default_rng(n)
    w = rng.exponential(size=n).astype(np.float32)
    run_evict([[[n]]], [[[b]]], page=256, recent=100, weights=lambda u, t: w[t], seed=1)


@pytest.mark.parametrize("alias", [False, True])
def test_evict_of_many_units_some_of_them_long(alias):
    # 48 units, so that long and short ones go their own ways; lengths around the border between them, units at their budget,
    # empty ones and refused ones among them
    rng = np.random.default_rng(4)
    lengths = rng.integers(1, 300, size=(2, 4, 6)).astype(np.int32)
    lengths[0, 0] = [8256, 8257, 20000, 8300, 16513, 9000]
    lengths[1, 2] = [8258, 100, -1, 0, 12000, 31]
    budgets = np.maximum(0, lengths - rng.integers(-2, 200, size=lengths.shape)).astype(np.int32)
    budgets[0, 0] = [8000, 8256, 50, 8300, 9000, 0]
    budgets[1, 2, 4] = -1
    st = run_evict(lengths, budgets, page=32, recent=16, alias=alias, seed=6)
    assert np.all(st == 0)
    lengths[0, 0, 2] = 20001                                             # one token more than the call allows
    st = run_evict(lengths, budgets, page=32, recent=16, alias=alias, seed=7, max_length=20000)
    assert st[0, 0, 2] == 16 and st.sum() == 16


def test_evict_refuses_units_beyond_the_bound_or_with_a_bad_page():
    from paper_2507_08143_b200 import binding as B
    st = run_evict([[[50, 30]]], [[[20, 20]]], max_length=40)
    assert st.tolist() == [[[16, 0]]]
    host, cache, len_d = make_cache([[[50, 50]]], 16, 0, 5)
    before = pools_of(cache)
    for tbl in (host["table"], cache.tensors[2]):
        tbl[0, 0, 0, 3] = 10 ** 8
    out, st = torch.zeros_like(len_d), torch.zeros_like(len_d)
    budgets = torch.tensor([[[20, 20]]], dtype=torch.int32, device="cuda")
    B.paged_evict(cache, len_d, budgets, out, 50, status=st)
    assert out.cpu().tolist() == [[[50, 20]]] and st.cpu().tolist() == [[[8, 0]]]
    got = pools_of(cache)
    for j in range(3):
        p = int(host["table"][0, 0, 0, j])
        np.testing.assert_array_equal(got["k"][p], before["k"][p])


def test_evict_replays_from_a_graph():
    from paper_2507_08143_b200 import binding as B
    lens = np.array([[[300, 45, 0, 80]]], np.int32)
    host, cache, len_d = make_cache(lens, 16, 0, 21)
    budgets = torch.full((1, 1, 4), 60, dtype=torch.int32, device="cuda")
    out = torch.zeros_like(len_d)
    start = [t.clone() for t in cache.tensors]
    B.paged_evict(cache, len_d, budgets, out, 300)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.paged_evict(cache, len_d, budgets, out, 300)
    for n in ([300, 45, 0, 80], [299, 45, 0, 61]):
        for t, s in zip(cache.tensors, start):
            t.copy_(s)
        len_d.copy_(torch.tensor([[n]], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        want, want_len = po.evict(host, list(np.ndindex(1, 1, 4)), np.array([[n]], np.int32), budgets.cpu().numpy())
        same_bits(pools_of(cache), want, "replay")
        np.testing.assert_array_equal(out.cpu().numpy(), want_len)


# ------------------------------------------------------------------------------------------------ the whole path
@pytest.mark.parametrize("across", [False, True])
def test_compress_fill_decode_evict(across):
    """A prefill is compressed, its kept rows go into pages, four tokens are decoded with the weights accumulated, and the
    cache is brought back to its budget: every step against the oracle on the same bits."""
    from paper_2507_08143_b200 import binding as B
    from paper_2507_08143_b200 import inputs
    L, Hh, g, page, m = 2, 2, 4, 16, 48
    w = inputs.Workload("paged", L, Hh, 128, [700, 64, 300], [0.3, 0.5, 0.4], p=0.7, seed=33)
    _, k, v = [t.cuda() if t is not None else None for t in inputs.make_tensors(w, device="cpu")]
    shape = B.Shape(L, Hh, 128, m, w.seqlens)
    keep = [B.keep_count(n, r) for n, r in zip(w.seqlens, w.ratios)]
    phi = inputs.make_sketch_matrix(128, m, 1).cuda()
    q_pre = torch.randn(L, Hh * g, shape.total_tokens, 128, device="cuda").bfloat16()
    opt = B.options(selection=B.SELECT_ACROSS_HEADS if across else B.SELECT_PER_HEAD, q_per_kv=g)
    KK, T = sum(keep), shape.total_tokens
    idx = torch.empty(L, Hh * KK, dtype=torch.int32, device="cuda")
    offs = torch.empty(L, 3, Hh + 1, dtype=torch.int32, device="cuda")
    k_out, v_out = torch.empty(L, Hh * KK, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(L, Hh * KK, 128, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(B.compress_full_workspace_bytes(shape, opt), dtype=torch.uint8, device="cuda")
    B.compress_full(shape, opt, q_pre, k, k, v, phi, keep, idx, k_out, v_out, ws, head_offsets_out=offs)
    attn = torch.empty(L, Hh, T, device="cuda")
    B.attention_scores(shape, q_pre, k, g, attn, B.alloc_workspace(shape), 128 ** -0.5)
    # pages
    units = np.zeros((L, Hh, 3), np.int32)
    host, cache, len_d = make_cache(units, page, Hh * max(keep) + 8, 34)
    B.paged_fill(cache, shape, k, v, keep, idx=idx, head_offsets=offs if across else None, mass_in=attn, lengths=len_d, lengths_out=len_d)
    cu, ck = shape.cu_seqlens, np.concatenate([[0], np.cumsum(keep)])
    idx_h, offs_h = idx.cpu().numpy(), offs.cpu().numpy()

    def rows(l, h, b):
        if across:
            return idx_h[l, Hh * ck[b] + offs_h[l, b, h]: Hh * ck[b] + offs_h[l, b, h + 1]]
        return idx_h.reshape(L, Hh, KK)[l, h, ck[b]:ck[b + 1]]
    host, lens = po.fill(host, 0, H.bits(k), H.bits(v), cu, rows, attn.cpu().numpy())
    same_bits(pools_of(cache), host, "fill")
    np.testing.assert_array_equal(len_d.cpu().numpy(), lens)
    if not across:                                                       # the pages hold what the dense compaction gives
        for b in range(3):
            p, s = po.slot_of(host, (1, 1, b), 3)
            np.testing.assert_array_equal(host["k"][p, s], H.bits(k_out.view(L, Hh, KK, 128))[1, 1, ck[b] + 3])
    budgets = lens.copy()
    # decode
    dopt = B.decode_options(g, Hh * max(keep) + 8, accumulate=True)
    dws = B.alloc_paged_attention_workspace(cache, dopt)
    nxt = torch.tensor(w.seqlens, dtype=torch.int32, device="cuda")
    for step in range(4):
        for l in range(L):
            q = torch.randn(3, Hh * g, 128, device="cuda").bfloat16()
            kn, vn = torch.randn(3, Hh, 128, device="cuda").bfloat16(), torch.randn(3, Hh, 128, device="cuda").bfloat16()
            out = torch.empty_like(q)
            B.paged_attention(cache, l, dopt, q, len_d, out, dws, k_new=kn, v_new=vn, new_positions=nxt)
            ref, _, after, info = po.attention(host, l, H.bits(q), lens, 128 ** -0.5, k_new=H.bits(kn), v_new=H.bits(vn),
                                               new_positions=nxt.cpu().numpy(), accumulate=True)
            got = pools_of(cache)
            same_bits(got, after, f"step {step} layer {l}")
            live = ~np.isnan(after["mass"])
            assert np.max(np.abs(got["mass"] - after["mass"])[live] / np.maximum(1e-3, after["mass"][live])) < 2e-4
            for (h, b), (at, p, pv, mag) in info.items():
                _, _, tol = attention_bounds(g, p, pv, ref[b, h * g:(h + 1) * g], mag, 128 ** -0.5, 0.0, len(at))
                assert np.all(np.abs(out[b, h * g:(h + 1) * g].float().cpu().numpy() - ref[b, h * g:(h + 1) * g]) <= tol)
            host = dict(after, mass=got["mass"].copy())                  # the library's own weights decide what is evicted
        len_d += 1
        nxt += 1
        lens = lens + 1
    # back to the budget
    B.paged_evict(cache, len_d, torch.from_numpy(budgets).cuda(), len_d, Hh * max(keep) + 8, recent=16, next_position=nxt)
    host, lens = po.evict(host, list(np.ndindex(L, Hh, 3)), lens, budgets, 16, nxt.cpu().numpy())
    got = pools_of(cache)
    same_bits(got, host, "evict")
    np.testing.assert_array_equal(got["mass"].view(np.uint32), host["mass"].view(np.uint32))
    np.testing.assert_array_equal(len_d.cpu().numpy(), budgets)


def test_attention_captured_behind_copies_and_memsets():
    # what stands before the call in a graph need not be a kernel: a copy, the clearing of the status words
    from paper_2507_08143_b200 import binding as B
    _, cache, len_d = make_cache([[[100, 7]]], 16, 4, 13)
    q, q2 = torch.randn(2, 4, 128, device="cuda").bfloat16(), torch.randn(2, 4, 128, device="cuda").bfloat16()
    opt = B.decode_options(4, 104)
    ws, out, want = B.alloc_paged_attention_workspace(cache, opt), torch.empty_like(q), torch.empty_like(q)
    st = torch.full((1, 1, 2), 5, dtype=torch.int32, device="cuda")
    B.paged_attention(cache, 0, opt, q2, len_d, want, ws, status=st)
    torch.cuda.synchronize()
    for status in (None, st):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            q.copy_(q2)
            B.paged_attention(cache, 0, opt, q, len_d, out, ws, status=status)
        q.zero_(); out.zero_(); st.fill_(5)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and st.unique().tolist() == [5 if status is None else 0]


@pytest.mark.parametrize("page,heads,lens", [(8, 4, [90001, 120007]), (16, 2, [400003]), (1024, 4, [70000, 131071, 1])])
def test_attention_of_long_contexts_against_torch_in_64_bits(page, heads, lens):
    # every warp walks over many page ids and, where it changes units, over their ends; reference unit by unit on the GPU
    from paper_2507_08143_b200 import binding as B
    batch, g = len(lens), 3
    gen = torch.Generator(device="cuda").manual_seed(page)
    pages = [(n + 1 + page - 1) // page for n in lens]
    n_pages = heads * sum(pages)
    ids = torch.randperm(n_pages, device="cuda", generator=gen).int()
    table = torch.full((1, heads, batch, max(pages)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for h in range(heads):
        for b in range(batch):
            table[0, h, b, :pages[b]] = ids[at:at + pages[b]]
            at += pages[b]
    k = torch.randn(n_pages, page, 128, device="cuda", generator=gen, dtype=torch.bfloat16)
    v = torch.randn(n_pages, page, 128, device="cuda", generator=gen, dtype=torch.bfloat16)
    mass = torch.rand(n_pages, page, device="cuda", generator=gen)
    mass0 = mass.double()
    cache = B.PagedCache(k, v, table, mass=mass)
    q = torch.randn(batch, heads * g, 128, device="cuda", generator=gen).bfloat16()
    kn, vn = torch.randn(batch, heads, 128, device="cuda", generator=gen).bfloat16(), torch.randn(batch, heads, 128, device="cuda", generator=gen).bfloat16()
    lengths = torch.tensor(lens, dtype=torch.int32, device="cuda").expand(1, heads, batch).contiguous()
    opt = B.decode_options(g, max(lens) + 1, accumulate=True)
    out, lse = torch.empty_like(q), torch.empty(batch, heads * g, device="cuda")
    B.paged_attention(cache, 0, opt, q, lengths, out, B.alloc_paged_attention_workspace(cache, opt), k_new=kn, v_new=vn, lse_out=lse)
    for h in range(heads):
        for b, n in enumerate(lens):
            used = table[0, h, b, :pages[b]].long()
            kk, vv = k[used].reshape(-1, 128)[:n + 1].double(), v[used].reshape(-1, 128)[:n + 1].double()
            assert torch.equal(kk[n], kn[b, h].double()) and torch.equal(vv[n], vn[b, h].double())       # appended
            qq = q[b, h * g:(h + 1) * g].double()
            y = qq @ kk.T * 128 ** -0.5
            p = torch.softmax(y, 1)
            ref = p @ vv
            mag = float((qq.abs() @ kk.abs().T).max()) * 128 ** -0.5
            dy, rel, tol = attention_bounds(g, None, (p @ vv.abs()).cpu().numpy(), ref.cpu().numpy(), mag, 128 ** -0.5, 0.0, n + 1)
            assert np.all(np.abs((out[b, h * g:(h + 1) * g].double() - ref).cpu().numpy()) <= tol)
            ref_lse = torch.logsumexp(y, 1)
            assert torch.all((lse[b, h * g:(h + 1) * g].double() - ref_lse).abs() <= dy + rel + 2.0 ** -22 * ref_lse.abs())
            got, want = mass[used].reshape(-1)[:n + 1].double(), mass0[used].reshape(-1)[:n + 1].clone()
            want[n] = 0
            want += p.sum(0)
            # an element of the sum: its own bound, and the rounding of the addition to what was there
            assert torch.all((got - want).abs() <= (1.01 * rel + (g + 2) * 2.0 ** -24) * p.sum(0) + 2.0 ** -24 * want)


def test_attention_of_more_units_than_a_block_keeps_at_hand():
    rng = np.random.default_rng(15)
    lengths = rng.integers(-1, 40, size=(1, 8, 300)).astype(np.int32)    # 2400 units
    lengths[0, 7, 299] = 700
    run_attention(lengths, 1, 8, accumulate=True, seed=15)


@pytest.mark.parametrize("b", [393000, 1000])
def test_evict_of_the_longest_unit(b):
    w = np.random.default_rng(b).exponential(size=393216).astype(np.float32)
    run_evict([[[393216]]], [[[b]]], page=1024, recent=500, weights=lambda u, t: w[t], seed=2)


@pytest.mark.parametrize("seed", range(12))
def test_random_batches(seed):
    # shapes, page sizes, masks and options drawn together
    rng = np.random.default_rng(1000 + seed)
    layers, heads, batch = int(rng.integers(1, 3)), int(rng.integers(1, 6)), int(rng.integers(1, 9))
    page = int(2 ** rng.integers(3, 8))
    top = int(2 ** rng.uniform(0, 11))
    lengths = rng.integers(-1, top + 1, size=(layers, heads, batch)).astype(np.int32)
    run_attention(lengths, int(rng.integers(1, 25)), page, accumulate=bool(rng.integers(2)), softcap=float(rng.choice([0.0, 0.0, 20.0])),
                  append=bool(rng.integers(2)), strided=bool(rng.integers(2)), layer=int(rng.integers(layers)), seed=seed)
    budgets = (lengths * rng.random(lengths.shape) * 1.2).astype(np.int32) - int(rng.integers(0, 2))
    ties = bool(rng.integers(2))
    w = rng.exponential(size=(top + 1,)).astype(np.float32)
    run_evict(lengths, budgets, page=page, recent=int(rng.integers(0, 40)), seed=seed, strided=bool(rng.integers(2)),
              weights=(lambda u, t: float(np.floor(4 * w[t]))) if ties else None, alias=bool(rng.integers(2)))
    seqlens = rng.integers(0, top + 1, size=batch).tolist()
    keep = [int(rng.integers(0, n + 1)) for n in seqlens]
    across = bool(rng.integers(2))
    held = None if across else rng.integers(-1, 30, size=(layers, heads, batch))
    run_fill(seqlens, keep, page, layers=layers, cache_layers=layers, heads=heads, across=across, held=held, use_idx=across or bool(rng.integers(2)),
             mass=bool(rng.integers(2)), strided=bool(rng.integers(2)), alias=bool(rng.integers(2)), seed=seed)


def test_the_steps_of_a_decoding_loop_in_one_graph():
    # attention of every layer, lengths and positions advanced, eviction: captured once, replayed; as the same calls made directly
    from paper_2507_08143_b200 import binding as B
    L, heads, batch, g, page = 2, 3, 4, 2, 16
    lens = np.random.default_rng(3).integers(40, 90, size=(L, heads, batch)).astype(np.int32)
    lens[:, :, 2] = -1

    def start():
        _, cache, len_d = make_cache(lens, page, 20, 77)
        gen = torch.Generator(device="cuda").manual_seed(5)
        rnd = lambda *s: torch.randn(*s, device="cuda", generator=gen).bfloat16()
        st = dict(cache=cache, len=len_d, pos=torch.full((batch,), 200, dtype=torch.int32, device="cuda"), q=rnd(L, batch, heads * g, 128),
                  k=rnd(L, batch, heads, 128), v=rnd(L, batch, heads, 128), out=torch.zeros(L, batch, heads * g, 128, dtype=torch.bfloat16, device="cuda"),
                  budgets=torch.full((L, heads, batch), 60, dtype=torch.int32, device="cuda"), opt=B.decode_options(g, 110, accumulate=True))
        st["ws"] = B.alloc_paged_attention_workspace(cache, st["opt"])
        return st

    def step(s):
        for l in range(L):
            B.paged_attention(s["cache"], l, s["opt"], s["q"][l], s["len"], s["out"][l], s["ws"], k_new=s["k"][l], v_new=s["v"][l], new_positions=s["pos"])
        s["len"].add_((s["len"] >= 0).int())
        s["pos"].add_(1)
        B.paged_evict(s["cache"], s["len"], s["budgets"], s["len"], 110, recent=8, next_position=s["pos"])

    a, b = start(), start()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):                                        # set-up before capture, on a cache of its own
        step(start())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a)
    for i in range(5):
        graph.replay()
        step(b)
    torch.cuda.synchronize()
    assert torch.equal(a["len"], b["len"]) and torch.equal(a["out"], b["out"])
    for x, y in zip(a["cache"].tensors, b["cache"].tensors):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    assert int(a["len"].max()) <= 60 and torch.all(a["len"][:, :, 2] == -1)


def test_evict_of_long_and_short_units_and_fill_in_one_graph():
    # the two launches of an eviction of many ragged units, behind a fill that appends in place: captured, replayed, compared
    from paper_2507_08143_b200 import binding as B
    rng = np.random.default_rng(31)
    lens = rng.integers(100, 400, size=(1, 8, 6)).astype(np.int32)
    lens[0, :, 0] = 8300
    lens[0, 3, 1] = 16600
    host, cache, len_d = make_cache(lens, 32, 5, 31)
    k, v, _ = _prefill(1, 8, [5] * 6, 3)
    shape, kd, vd = B.Shape(1, 8, 128, 48, [5] * 6), k.cuda(), v.cuda()
    budgets = np.maximum(lens - 40, 1)
    bud, lens0, start = torch.from_numpy(budgets).cuda(), len_d.clone(), [t.clone() for t in cache.tensors]

    def calls():
        B.paged_fill(cache, shape, kd, vd, [5] * 6, lengths=len_d, lengths_out=len_d)
        B.paged_evict(cache, len_d, bud, len_d, 16605)
    calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    want, want_len = po.fill(host, 0, H.bits(k), H.bits(v), [5 * b for b in range(7)], lambda l, h, b: np.arange(5), lengths=lens)
    want, want_len = po.evict(want, list(np.ndindex(lens.shape)), want_len, budgets)
    for _ in range(3):
        for t, s in zip(cache.tensors, start):
            t.copy_(s)
        len_d.copy_(lens0)
        graph.replay()
        torch.cuda.synchronize()
        same_bits(pools_of(cache), want, "replay")
        np.testing.assert_array_equal(len_d.cpu().numpy(), want_len)
