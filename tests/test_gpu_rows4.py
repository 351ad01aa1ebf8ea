"""The paged cache with rows held in 4 bits on the GPU: fill, read-back, attention of one new token and eviction against the fp64
statements of oracle/rows_oracle.py.  Unused slots hold bytes that stand for not-a-number, page ids behind a unit's last page lie outside
the pool, and every pool is compared whole."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from oracle import rows_oracle as ro
from oracle.compactor_oracle import bf16_bits_to_f64
from tests import helpers as H
from tests.test_gpu_paged import LENGTHS, _prefill, make_cache

pytestmark = pytest.mark.gpu


def make_cache4(lengths, page, room, seed, strided=False):
    """make_cache with its rows held in 4 bits, and 255s (not a number) in all other slots."""
    from paper_2507_08143_b200 import binding as B
    lengths = np.asarray(lengths, np.int32)
    host, cache, len_d = make_cache(lengths, page, room, seed)
    live = ~np.isnan(host["mass"])
    for name in ("k", "v"):
        rows = np.full(host["mass"].shape + (80,), 255, np.uint8)
        rows[live] = ro.hold4(host[name][live])
        host[name] = rows
    k, v = torch.from_numpy(host["k"]).cuda(), torch.from_numpy(host["v"]).cuda()
    if strided:                                                          # K and V of a page side by side, pages with a gap
        both = torch.full((k.shape[0], 2 * page * 80 + 48), 255, dtype=torch.uint8, device="cuda")
        views = [both[:, i * page * 80:(i + 1) * page * 80].unflatten(1, (page, 80)) for i in range(2)]
        views[0].copy_(k); views[1].copy_(v)
        k, v = views
    return host, B.PagedCache4(k, v, cache.tensors[2], mass=cache.tensors[3], positions=cache.tensors[4]), len_d


def pools4(cache):
    k, v, _, mass, pos = cache.tensors
    return dict(k=k.cpu().numpy(), v=v.cpu().numpy(), mass=mass.cpu().numpy(), positions=pos.cpu().numpy())


def check_pools(got, want, what):
    for name in ("k", "v", "positions"):
        np.testing.assert_array_equal(got[name], want[name], err_msg=f"{what}: {name}")


def attention4_bounds(g, pv, out, mag, softcap, n):
    """Derived bounds of one (KV head, sequence); mag: largest scale * sum |q| (|s c| + |lo|), pv: sum p (|s c| + |lo|).
    scores: nine accumulations of 16 products (exact, but for the last one's sums of 32 query channels: five roundings of 2^-24, and three bf16
      terms of 2^-24 in all), each of which may drop a unit of 2^-23 of the largest partial sum for each of 17 summands; the cap as in the
      attention over bf16 rows; the scaling and the difference to the maximum 3 * 2^-24.
    weights: e^dy, ex2 2^-22, the sum of n terms along at most n / 8 + 64 additions of 2^-24.
    out: two bf16 terms of a weight 2^-16, the sums over n tokens (17 * 2^-23 per 16), once more when the least values' part is added, rounded to bf16 2^-8."""
    dy = (9 * 17 + 6 + 2) * 2.0 ** -23 * mag + (softcap * 2.0 ** -22 if softcap else 0.0)
    rel = 2 * dy + 2 * 2.0 ** -22 + (n / 8 + 64) * 2.0 ** -24
    return dy, rel, (rel + 2.0 ** -16 + (n / 16 + 17) * 17 * 2.0 ** -23) * 1.01 * pv + 2.0 ** -8 * np.abs(out) + 1e-30


def run_attention4(lengths, g, page, accumulate=False, softcap=0.0, append=True, strided=False, room=1, seed=0, layer=0, max_length=None,
                   positions=True, q_scale=1.5, change=None, kn_scale=1.0):
    from paper_2507_08143_b200 import binding as B
    lengths = np.asarray(lengths, np.int32)
    _, heads, batch = lengths.shape
    host, cache, len_d = make_cache4(lengths, page, room, seed, strided)
    if change is not None:
        change(host, cache)
    gen = torch.Generator().manual_seed(seed + 1)
    q = (q_scale * torch.randn(batch, heads * g, 128, generator=gen)).bfloat16()
    kn, vn = ((kn_scale * torch.randn(batch, heads, 128, generator=gen)).bfloat16() for _ in range(2))
    newpos = torch.arange(batch, dtype=torch.int32) + 1000
    limit = int(max(1, lengths.max() + 1)) if max_length is None else max_length
    opt = B.decode_options(g, limit, softcap=softcap, accumulate=accumulate)
    ws = torch.full((max(256, B.paged_attention_workspace_bytes(cache, opt)),), 255, dtype=torch.uint8, device="cuda")
    if strided:
        qd = torch.zeros(heads * g, batch, 136, dtype=torch.bfloat16, device="cuda")[..., :128].transpose(0, 1)
        qd.copy_(q)
        out_all = torch.full((heads * g, batch, 136), 7.0, dtype=torch.bfloat16, device="cuda")
        out = out_all[..., :128].transpose(0, 1)
    else:
        qd, out = q.cuda(), torch.full((batch, heads * g, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((batch, heads * g), 7.0, device="cuda")
    st = torch.full(lengths.shape, 99, dtype=torch.int32, device="cuda")
    extra = dict(k_new=kn.cuda(), v_new=vn.cuda(), new_positions=newpos.cuda() if positions else None) if append else {}
    B.paged_attention(cache, layer, opt, qd, len_d, out, ws, lse_out=lse, status=st, **extra)
    torch.cuda.synchronize()
    okw = dict(k_new=H.bits(kn), v_new=H.bits(vn), new_positions=newpos.numpy() if positions else None) if append else {}
    ref, ref_lse, after, info = ro.attention4(host, layer, H.bits(q), lengths, np.float64(np.float32(128 ** -0.5)), softcap=softcap,
                                              accumulate=accumulate, max_length=limit, **okw)
    o, ls = out.float().cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)
    got = pools4(cache)
    check_pools(got, after, "pools")
    mass_tol = np.zeros_like(after["mass"])
    for h in range(heads):
        for b in range(batch):
            rows = slice(h * g, (h + 1) * g)
            if (h, b) not in info:
                assert np.all(o[b, rows] == 0) and np.all(ls[b, rows] == -np.inf), (h, b)
                continue
            at, p, pv, mag = info[(h, b)]
            if np.isnan(ref[b, rows]).any():
                assert np.array_equal(np.isnan(ref[b, rows]), np.isnan(o[b, rows])), (h, b)
                continue
            dy, rel, tol = attention4_bounds(g, pv, ref[b, rows], mag, softcap, len(at))
            err = np.abs(o[b, rows] - ref[b, rows])
            assert np.all(err <= tol), f"out (h={h}, b={b}): {np.max(err / tol):.2f} of the bound"
            assert np.all(np.abs(ls[b, rows] - ref_lse[b, rows]) <= dy + rel + 2.0 ** -22 * np.abs(ref_lse[b, rows])), f"lse (h={h}, b={b})"
            if accumulate:
                for j, a in enumerate(at):
                    if a is not None:
                        mass_tol[a] = (1.01 * rel + (g + 2) * 2.0 ** -24) * p[:, j].sum() + 2.0 ** -24 * abs(after["mass"][a])
    live = ~np.isnan(after["mass"])
    assert np.array_equal(live, ~np.isnan(got["mass"]))
    err = np.abs(got["mass"].astype(np.float64) - after["mass"])[live]
    assert np.all(err <= mass_tol[live]), f"weights: {np.max(err):.3e}"
    if strided:
        assert torch.all(out_all[..., 128:].float() == 7.0)
    return host, cache, after, st, out, lse


@pytest.mark.parametrize("name", list(LENGTHS))
@pytest.mark.parametrize("append", [True, False])
@pytest.mark.parametrize("accumulate", [True, False])
def test_attention_lengths(name, append, accumulate):
    lengths = np.array(LENGTHS[name], np.int32)
    run_attention4(lengths, 4, 16, accumulate=accumulate, append=append, layer=lengths.shape[0] - 1)


@pytest.mark.parametrize("g", [1, 2, 3, 7, 8, 9, 15, 16, 17, 33, 64])
def test_attention_head_layouts(g):
    run_attention4([[[37, 0, 210], [16, 90, -1]]], g, 16, accumulate=True, seed=g)
    run_attention4([[[400]]], g, 32, accumulate=False, seed=g + 100)


@pytest.mark.parametrize("page", [8, 16, 32, 128, 1024])
def test_attention_page_sizes_and_strides(page):
    run_attention4([[[1, 100, 1023, 7], [2 * page, page - 1, page + 1, 3 * page]]], 5, page, accumulate=True, strided=True, seed=page)


@pytest.mark.parametrize("softcap", [0.5, 50.0])
def test_attention_capped_scores(softcap):
    run_attention4([[[300, 17, 0], [64, 1, 129]]], 3, 16, accumulate=True, softcap=softcap, seed=5, q_scale=6.0)


def test_attention_many_units_and_one_long_one():
    lengths = np.random.default_rng(8).integers(-1, 70, size=(1, 4, 300)).astype(np.int32)       # more units than threads of a block
    lengths[0, 2, 77] = 6000
    run_attention4(lengths, 2, 16, accumulate=True, seed=8)
    run_attention4(lengths[:, :, :40], 10, 8, seed=9)


def test_attention_lengths_beyond_the_bound_and_pages_that_are_none():
    _, _, _, st, _, _ = run_attention4([[[50, 39, 40, 10]]], 2, 16, accumulate=True, max_length=40)
    assert st.cpu().tolist() == [[[16, 0, 16, 0]]]
    _, _, _, st, _, _ = run_attention4([[[64, 5]]], 2, 16, room=0, max_length=1000)      # no page left for the new token
    assert st.cpu().tolist() == [[[8, 0]]]

    def lose(host, cache):
        for tbl in (host["table"], cache.tensors[2]):
            tbl[0, 0, 0, 2] = -5
            tbl[0, 0, 0, 4] = 10 ** 9

    def none_left(host, cache):
        for tbl in (host["table"], cache.tensors[2]):
            tbl[0, 0, 0, :] = -1
    for page in (8, 16):
        _, _, _, st, _, _ = run_attention4([[[100, 40]]], 4, page, accumulate=True, seed=3, change=lose)
        assert st.cpu().tolist() == [[[8, 0]]]
        run_attention4([[[100, 40]]], 4, page, accumulate=True, append=False, seed=3, change=none_left)


def test_attention_values_at_the_ends_of_the_range():
    """Constant groups, steps below and above what is held, groups that are not a number: in one unit each, and in new tokens."""
    def change(host, cache):
        for b, make in enumerate((lambda x: x * 0 + 3, lambda x: x * 2.0 ** -125, lambda x: x * 2.0 ** 60, lambda x: np.where(np.arange(128) == 40, np.inf, x))):
            p = host["table"][0, 0, b, 1]
            x = make(np.random.default_rng(b).standard_normal((16, 128)))
            rows = ro.hold4(ro.f64_to_bf16_bits(x))
            which = "v" if b == 2 else "k"
            host[which][p] = rows
            cache.tensors[0 if which == "k" else 1][int(p)] = torch.from_numpy(rows).cuda()
    run_attention4([[[60, 60, 60, 60, 60]]], 2, 16, seed=4, change=change)
    run_attention4([[[20, 0]]], 2, 16, seed=5, kn_scale=2.0 ** -128)
    run_attention4([[[20, 0]]], 2, 16, seed=6, kn_scale=0.0)


def test_attention_is_as_exact_where_values_cancel():
    """Two halves of a unit whose values are each other's opposites: what is left of the sums is rounded by the weights' terms alone."""
    def change(host, cache):
        for t in range(512):
            a, b = po.slot_of(host, (0, 0, 0), t), po.slot_of(host, (0, 0, 0), t + 512)
            for name, i in (("k", 0), ("v", 1)):
                rows = host[name][a].copy()
                if name == "v":                                          # lo + s c -> -lo - 15 s + s (15 - c)
                    sc, lo = ro.values4(rows, True)
                    x = -(sc + lo)
                    rows = ro.hold4(ro.f64_to_bf16_bits(x))
                host[name][b] = rows
                cache.tensors[i][b[0], b[1]] = torch.from_numpy(rows).cuda()
    run_attention4([[[1024]]], 8, 16, append=False, seed=7, change=change)


def test_attention_is_reproducible_and_replays_from_a_graph():
    from paper_2507_08143_b200 import binding as B
    lens = np.array([[[500, 0, 77, 1500], [20, 333, -1, 64]]], np.int32)
    _, cache, len_d = make_cache4(lens, 16, 8, 11)
    q = torch.randn(4, 8, 128, device="cuda").bfloat16()
    kn, vn = torch.randn(4, 2, 128, device="cuda").bfloat16(), torch.randn(4, 2, 128, device="cuda").bfloat16()
    opt = B.decode_options(4, 1600, accumulate=True)
    ws = B.alloc_paged_attention_workspace(cache, opt)
    out, lse = torch.empty_like(q), torch.empty(4, 8, device="cuda")
    start = [t.clone() for t in cache.tensors]

    def call(o, ls, w):
        B.paged_attention(cache, 0, opt, q, len_d, o, w, k_new=kn, v_new=vn, lse_out=ls)
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
            o, ls = (out, lse) if replay else (torch.empty_like(out), torch.empty_like(lse))
            graph.replay() if replay else call(o, ls, torch.full_like(ws, 255))
            torch.cuda.synchronize()
            snap.append([o.clone(), ls.clone()] + [t.clone() for t in cache.tensors])
        for a, b in zip(*snap):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_attention_on_two_streams_at_once():
    from paper_2507_08143_b200 import binding as B
    _, cache, len_d = make_cache4(np.full((2, 4, 3), 900, np.int32), 16, 1, 12)
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


def test_rows_beyond_32_bit_offsets():
    """A pool of 4.4e9 bytes, used as K and as V; the pages in use are the last ones."""
    from paper_2507_08143_b200 import binding as B
    page, n_pages = 1024, 54000
    pool = torch.empty(n_pages, page, 80, dtype=torch.uint8, device="cuda")
    assert pool.numel() > 2 ** 32
    table = torch.tensor([[[[n_pages - 1, n_pages - 2]]]], dtype=torch.int32, device="cuda")
    cache = B.PagedCache4(pool, pool, table)
    x = torch.randn(1, 1, 1500, 128, device="cuda").bfloat16()
    n = torch.zeros(1, 1, 1, dtype=torch.int32, device="cuda")
    shape = B.Shape(1, 1, 128, 48, [1500])
    B.paged_fill(cache, shape, x, x, [1500], lengths_out=n)
    back = torch.empty(2, 1, 1, 1500, 128, dtype=torch.bfloat16, device="cuda")
    B.paged_read(cache, shape, n, back[0], back[1])
    rows = ro.values4(ro.hold4(H.bits(x)))
    assert np.array_equal(back[0].float().cpu().numpy(), bf16_bits_to_f64(ro.f64_to_bf16_bits(rows.astype(np.float32))))
    assert torch.equal(back[0], back[1])
    q = torch.randn(1, 2, 128, device="cuda").bfloat16()
    opt = B.decode_options(2, 2048)
    out = torch.empty_like(q)
    B.paged_attention(cache, 0, opt, q, n, out, B.alloc_paged_attention_workspace(cache, opt))
    rows = torch.from_numpy(rows[0, 0]).cuda()
    p = torch.softmax(q[0].double() @ rows.T * 128 ** -0.5, 1)
    assert torch.all((out[0].double() - p @ rows).abs() <= 2.0 ** -13 * (p @ rows.abs()) + 2.0 ** -8 * (p @ rows).abs())


# ------------------------------------------------------------------------------------------------ fill and read
def run_fill4(seqlens, keep, page, layers=2, heads=2, cache_layers=2, first_layer=0, across=False, held=None, strided=False, seed=0,
              room=None, scale=1.0, odd=None):
    from paper_2507_08143_b200 import binding as B
    batch = len(seqlens)
    rng = np.random.default_rng(seed)
    held = np.zeros((cache_layers, heads, batch), np.int32) if held is None else np.asarray(held, np.int32)
    host, cache, _ = make_cache4(held, page, (max(keep) * (heads if across else 1) if room is None else room), seed, strided)
    k, v, attn = _prefill(layers, heads, seqlens, seed)
    k, v = (k.float() * scale).bfloat16(), (v.float() * scale).bfloat16()
    if odd is not None:
        odd(k, v)
    cu, ck = np.concatenate([[0], np.cumsum(seqlens)]), np.concatenate([[0], np.cumsum(keep)])
    rows, offs = {}, None
    if across:
        idx, offs = np.zeros((layers, heads * sum(keep)), np.int32), np.zeros((layers, batch, heads + 1), np.int32)
        for l in range(layers):
            for b in range(batch):
                pick = np.sort(rng.permutation(heads * seqlens[b])[: heads * keep[b]])
                idx[l, heads * ck[b]: heads * ck[b + 1]] = pick % max(1, seqlens[b])
                offs[l, b, 1:] = np.searchsorted(pick, (np.arange(heads) + 1) * seqlens[b])
                for h in range(heads):
                    rows[l, h, b] = idx[l, heads * ck[b] + offs[l, b, h]: heads * ck[b] + offs[l, b, h + 1]]
    else:
        idx = np.zeros((layers, heads, sum(keep)), np.int32)
        for (l, h, b) in np.ndindex(layers, heads, batch):
            rows[l, h, b] = idx[l, h, ck[b]:ck[b + 1]] = np.sort(rng.permutation(seqlens[b])[: keep[b]])
    n = torch.from_numpy(held).cuda()
    st = torch.full(held.shape, 99, dtype=torch.int32, device="cuda")
    kd, vd = k.cuda(), v.cuda()
    if strided:
        kd = kd.transpose(1, 2).contiguous().transpose(1, 2)
    B.paged_fill(cache, B.Shape(layers, heads, 128, 48, seqlens), kd, vd, keep, idx=torch.from_numpy(idx).cuda(),
                 head_offsets=None if offs is None else torch.from_numpy(offs).cuda(), mass_in=attn.cuda(), lengths=n, lengths_out=n,
                 first_layer=first_layer, status=st)
    torch.cuda.synchronize()
    want, want_len = po.fill(host, first_layer, ro.hold4(H.bits(k)), ro.hold4(H.bits(v)), cu, lambda l, h, b: rows[l, h, b], attn.numpy(), None, held)
    got = pools4(cache)
    check_pools(got, want, "fill")
    np.testing.assert_array_equal(got["mass"].view(np.uint32), want["mass"].view(np.uint32))
    np.testing.assert_array_equal(n.cpu().numpy()[first_layer:first_layer + layers], want_len[first_layer:first_layer + layers])
    return st.cpu().numpy()


@pytest.mark.parametrize("page", [8, 16, 256])
@pytest.mark.parametrize("across", [False, True])
def test_fill_with_a_selection(page, across):
    run_fill4([100, 1, 0, 257, 40], [30, 1, 0, 200, 40], page, across=across, seed=page)
    run_fill4([64, 31], [7, 31], page, layers=1, cache_layers=3, first_layer=1, heads=3, across=across, strided=True, seed=page + 1)


def test_fill_behind_what_is_held_and_without_room():
    held = np.array([[[5, 0, -1], [16, 15, 3]], [[0, 1, 2], [31, -4, 8]]])
    run_fill4([4, 33, 6], [4, 20, 6], 16, held=held, seed=3)
    st = run_fill4([40, 40], [40, 33], 16, layers=1, cache_layers=1, held=[[[30, 0], [0, 7]]], room=0, seed=7)
    assert st[0, 0, 0] & 16 and st[0, 0, 1] == 8


@pytest.mark.parametrize("scale", [1e-37, 2.0 ** -119, 2.0 ** -116, 1e30, 2.0 ** 122, 2.0 ** 124, 0.0])
def test_fill_at_the_ends_of_the_range(scale):
    run_fill4([70], [70], 16, scale=scale, seed=11)


def test_fill_of_values_that_are_not_finite_and_of_equal_ones():
    def odd(k, v):
        k[0, 0, 3, 5] = float("inf"); k[0, 0, 4, 40] = float("-inf"); k[0, 1, 5, 127] = float("nan")
        k[0, 0, 6] = 2.5; k[0, 0, 7, :32] = -3.0; k[0, 0, 8, 32:64] = torch.tensor([float("inf"), float("-inf")] * 16)
        v[0, 0, 9] = torch.arange(128).float() - 64
        v[0, 0, 10] = torch.arange(128).float() / 2                       # halves of a step: the lower code
        v[0, 0, 11, ::2] = 3e38; v[0, 0, 11, 1::2] = -3e38
    run_fill4([40], [40], 8, layers=1, cache_layers=1, seed=12, odd=odd)


def test_fill_holds_every_row_as_defined_and_no_further_than_half_a_step():
    """Half a million rows of several distributions: the bytes are the definition's, and no value is further off than half its step and
    the rounding of its difference to the least value, 2^-24 of up to 15 steps."""
    from paper_2507_08143_b200 import binding as B
    g = torch.Generator(device="cuda").manual_seed(3)
    n = 1 << 17
    x = torch.randn(1, 4, n, 128, generator=g, device="cuda")
    x[0, 1] = x[0, 1].exp()
    x[0, 2] = (8 * x[0, 2]).round() / 8                                   # ties between codes
    x[0, 3] *= torch.exp2(torch.randint(-12, 12, (n, 128), generator=g, device="cuda").float())
    x = x.bfloat16()
    page = 1024
    pool = torch.zeros(4 * n // page, page, 80, dtype=torch.uint8, device="cuda")
    table = torch.arange(4 * n // page, dtype=torch.int32, device="cuda").view(1, 4, 1, -1)
    cache = B.PagedCache4(pool, torch.zeros_like(pool), table)
    shape = B.Shape(1, 4, 128, 48, [n])
    lens = torch.zeros(1, 4, 1, dtype=torch.int32, device="cuda")
    B.paged_fill(cache, shape, x, x.flip(2), [n], lengths_out=lens)
    want = ro.hold4(H.bits(x[0]))
    np.testing.assert_array_equal(pool.cpu().numpy().reshape(4, n, 80), want)
    sc, lo = ro.values4(want, True)
    step = np.repeat(bf16_bits_to_f64(np.ascontiguousarray(want[..., 64:]).view(np.uint16)).reshape(4, n, 4, 2)[..., 0], 32, -1)
    assert np.all(np.abs(sc + lo - x[0].double().cpu().numpy()) <= step / 2 + 15 * 2.0 ** -24 * step)
    kb, vb = torch.empty_like(x), torch.empty_like(x)
    B.paged_read(cache, shape, lens, kb, vb)
    assert torch.equal(kb, vb.flip(2))
    np.testing.assert_array_equal(H.bits(kb[0]), ro.f64_to_bf16_bits((sc + lo).astype(np.float32)))


@pytest.mark.parametrize("four", [False, True])
def test_read(four):
    from paper_2507_08143_b200 import binding as B
    lens = np.array([[[40, 0, 7, 100], [3, -1, 64, 9]], [[1, 2, 50, 4], [16, 15, 17, 8]]], np.int32)
    first = np.array([[[0, 0, 3, 90], [1, 0, 70, -2]], [[0, 1, 16, 4], [15, 0, 8, 1]]], np.int32)
    for page in (8, 16, 64):
        host, cache, len_d = (make_cache4 if four else make_cache)(lens, page, 1, page)
        host["table"][1, 0, 2, 1] = -9
        cache.tensors[2][1, 0, 2, 1] = -9
        for use_first, l0, layers, seqlens in ((True, 0, 2, [12, 0, 9, 30]), (False, 1, 1, [20, 5, 64, 3]), (False, 0, 2, [0, 0, 0, 0])):
            total = sum(seqlens)
            out = torch.full((2, layers, total, 2, 128), 7.0, dtype=torch.bfloat16, device="cuda").transpose(2, 3)   # tokens outside heads
            st = torch.full(lens.shape, 99, dtype=torch.int32, device="cuda")
            B.paged_read(cache, B.Shape(layers, 2, 128, 48, seqlens), len_d, out[0], out[1], first=torch.from_numpy(first).cuda() if use_first else None,
                         first_layer=l0, status=st)
            want = np.full((2, layers, 2, total, 128), 7.0)
            flags = np.full(lens.shape, 99); flags[l0:l0 + layers] = 0
            cu = np.concatenate([[0], np.cumsum(seqlens)])
            for (l, h, b) in np.ndindex(layers, 2, 4):
                unit = (l0 + l, h, b)
                f = int(first[unit]) if use_first else 0
                for j in range(seqlens[b]):
                    if f < 0 or f + j >= lens[unit]:
                        continue
                    a = po.slot_of(host, unit, f + j)
                    if a is None:
                        flags[unit] = 8
                        continue
                    for i, name in enumerate(("k", "v")):
                        r = host[name][a]
                        want[i, l, h, cu[b] + j] = bf16_bits_to_f64(ro.f64_to_bf16_bits(ro.values4(r).astype(np.float32)) if four else r)
            np.testing.assert_array_equal(out.double().cpu().numpy(), want)
            np.testing.assert_array_equal(st.cpu().numpy(), flags)


def test_read_of_lengths_beyond_the_pages_and_of_many_sequences():
    from paper_2507_08143_b200 import binding as B
    lens = np.random.default_rng(2).integers(-1, 20, size=(1, 1, 600)).astype(np.int32)
    host, cache, len_d = make_cache(lens, 8, 1, 2)
    len_d[0, 0, 5] = 10 ** 6
    seqlens = np.random.default_rng(3).integers(0, 12, size=600).tolist()
    k, v = (torch.zeros(1, 1, sum(seqlens), 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    st = torch.full(lens.shape, 99, dtype=torch.int32, device="cuda")
    B.paged_read(cache, B.Shape(1, 1, 128, 48, seqlens), len_d, k, v, status=st)
    want, at = np.zeros((sum(seqlens), 128)), 0
    for b, m in enumerate(seqlens):
        for j in range(m):
            if b != 5 and j < lens[0, 0, b]:
                want[at + j] = bf16_bits_to_f64(host["k"][po.slot_of(host, (0, 0, b), j)])
        at += m
    np.testing.assert_array_equal(k[0, 0].double().cpu().numpy(), want)
    assert st[0, 0, 5] == (16 if seqlens[5] else 0) and int(st.sum()) == int(st[0, 0, 5])


# ------------------------------------------------------------------------------------------------ evict
@pytest.mark.parametrize("page, room", [(8, 1), (16, 40)])
def test_evict(page, room):
    from paper_2507_08143_b200 import binding as B
    lens = np.array([[[40, 0, 300, 1000], [3, -1, 64, 129]]], np.int32)
    for strided in (False, True):
        host, cache, len_d = make_cache4(lens, page, room, page, strided)
        budgets = np.array([[[10, 0, 299, 200], [3, 5, 1, 64]]], np.int32)
        nxt = np.array([80, 5, 600, 2000], np.int32)
        out, st = torch.zeros_like(len_d), torch.full_like(len_d, 99)
        B.paged_evict(cache, len_d, torch.from_numpy(budgets).cuda(), out, 1100, recent=4, next_position=torch.from_numpy(nxt).cuda(), status=st)
        units = list(np.ndindex(lens.shape))
        want, want_len = po.evict(host, units, lens, budgets, recent=4, next_position=nxt)
        got = pools4(cache)
        check_pools(got, want, "evict")
        np.testing.assert_array_equal(got["mass"].view(np.uint32), want["mass"].view(np.uint32))
        np.testing.assert_array_equal(out.cpu().numpy(), want_len)
        assert not st.any()


def test_evict_of_a_long_unit_in_a_cluster():
    from paper_2507_08143_b200 import binding as B
    lens = np.array([[[20000, 9000]]], np.int32)
    host, cache, len_d = make_cache4(lens, 64, 1, 9)
    budgets = np.array([[[15000, 100]]], np.int32)
    out = torch.zeros_like(len_d)
    B.paged_evict(cache, len_d, torch.from_numpy(budgets).cuda(), out, 20000)
    want, want_len = po.evict(host, [(0, 0, 0), (0, 0, 1)], lens, budgets)
    check_pools(pools4(cache), want, "evict")
    np.testing.assert_array_equal(out.cpu().numpy(), want_len)
