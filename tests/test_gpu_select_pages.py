"""Key bounds of pages, the choice of pages by them and the attention over the chosen ones, on the GPU against oracle/rows_oracle.py."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from oracle import rows_oracle as ro
from oracle.compactor_oracle import bf16_bits_to_f64
from tests import helpers as H
from tests.test_gpu_paged import attention_bounds, make_cache
from tests.test_gpu_rows4 import attention4_bounds, make_cache4

pytestmark = pytest.mark.gpu


def same_values(got_bits, want_bits):
    np.testing.assert_array_equal(bf16_bits_to_f64(got_bits), bf16_bits_to_f64(want_bits))      # (of either sign a zero is a zero)


def fresh_bounds(host):
    return torch.full((host["k"].shape[0], 2, 128), 5.0, dtype=torch.bfloat16, device="cuda")


@pytest.mark.parametrize("page", [8, 16, 32, 128, 256, 1024])
@pytest.mark.parametrize("four", [False, True])
def test_bounds(page, four):
    from paper_2507_08143_b200 import binding as B
    lens = np.array([[[1, page, 3 * page + 1, 700, 0], [2 * page - 1, -1, page + 7, 9, 5 * page]],
                     [[page // 2, 1500, 2, 3, 4], [5, 6, 7, 8, 2 * page]]], np.int32)
    first = np.array([[[0, page - 1, 2 * page, 650, 0], [page, 0, page, -3, 4 * page + 1]], [[0, 1024, 9, 0, 1], [4, 0, 0, 0, page]]], np.int32)
    for strided in (False, True):
        host, cache, len_d = (make_cache4 if four else make_cache)(lens, page, 1, page, strided)
        for use_first, l0, layers in ((False, 0, 2), (True, 0, 2), (False, 1, 1)):
            bounds = fresh_bounds(host)
            st = torch.full(lens.shape, 99, dtype=torch.int32, device="cuda")
            before = H.bits(bounds)
            B.paged_bounds(cache, len_d, bounds, int(lens.max()), first=torch.from_numpy(first).cuda() if use_first else None, first_layer=l0,
                           layers=layers, status=st)
            units = [u for u in np.ndindex(lens.shape) if l0 <= u[0] < l0 + layers]
            same_values(H.bits(bounds), ro.bounds(host, units, lens, before, first if use_first else None))
            assert np.all(st.cpu().numpy()[l0:l0 + layers] == 0)


def test_bounds_of_values_that_are_no_numbers_and_units_that_do_not_fit():
    from paper_2507_08143_b200 import binding as B
    lens = np.array([[[40, 100, 33, 20]]], np.int32)
    host, cache, len_d = make_cache(lens, 16, 1, 3)
    for page, slot, ch, x in ((0, 3, 5, float("nan")), (1, 0, 6, float("inf")), (1, 9, 6, float("-inf"))):
        p = int(host["table"][0, 0, 0, page])
        cache.tensors[0][p, slot, ch] = x
        host["k"][p, slot, ch] = H.bits(torch.tensor([x]).bfloat16())[0]
    host["table"][0, 0, 2, 1] = -4
    cache.tensors[2][0, 0, 2, 1] = -4
    bounds = fresh_bounds(host)
    before = H.bits(bounds)
    st = torch.zeros_like(len_d)
    B.paged_bounds(cache, len_d, bounds, 50, status=st)
    same_values(H.bits(bounds), ro.bounds(host, list(np.ndindex(lens.shape)), lens, before, max_length=50))
    assert st.cpu().tolist() == [[[0, 16, 8, 0]]]


def run_select(lengths, g, page, pages, first_pages=1, last_pages=1, append=True, four=False, layer=0, seed=0, max_length=None, change=None,
               strided=False):
    from paper_2507_08143_b200 import binding as B
    lengths = np.asarray(lengths, np.int32)
    _, heads, batch = lengths.shape
    host, cache, len_d = (make_cache4 if four else make_cache)(lengths, page, 1, seed)
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((host["k"].shape[0], 2, 128)).astype(np.float32)
    x.sort(1)
    bounds = torch.from_numpy(x).bfloat16().cuda()
    if change is not None:
        change(host, cache, bounds)
    before = H.bits(bounds)
    gen = torch.Generator().manual_seed(seed + 1)
    q, kn = torch.randn(batch, heads * g, 128, generator=gen).bfloat16(), torch.randn(batch, heads, 128, generator=gen).bfloat16()
    q[:, :, 7] = 0
    limit = int(max(1, lengths.max() + 1)) if max_length is None else max_length
    table = torch.full((1, heads, batch, pages), 77, dtype=torch.int32, device="cuda")
    out = torch.full((1, heads, batch), 77, dtype=torch.int32, device="cuda")
    st = torch.full(lengths.shape, 99, dtype=torch.int32, device="cuda")
    ws = torch.full((max(256, B.paged_select_workspace_bytes(cache, limit)),), 255, dtype=torch.uint8, device="cuda")
    qd = q.cuda()
    if strided:
        qd = torch.zeros(heads * g, batch, 136, dtype=torch.bfloat16, device="cuda")[..., :128].transpose(0, 1)
        qd.copy_(q)
    B.paged_select(cache, layer, g, qd, len_d, bounds, table, out, ws, limit, first_pages=first_pages, last_pages=last_pages,
                   k_new=kn.cuda() if append else None, status=st)
    torch.cuda.synchronize()
    want, want_len, after = ro.select(host, layer, g, H.bits(q), lengths, before, pages, first_pages, last_pages, H.bits(kn) if append else None, limit)
    np.testing.assert_array_equal(table[0].cpu().numpy(), want)
    np.testing.assert_array_equal(out[0].cpu().numpy(), want_len)
    same_values(H.bits(bounds), after)
    return host, cache, len_d, table, out, st.cpu().numpy(), q, kn


@pytest.mark.parametrize("append", [True, False])
@pytest.mark.parametrize("pages", [2, 3, 9, 40])
@pytest.mark.parametrize("page", [8, 64])
def test_select(append, pages, page):
    lens = [[[0, 1, page, 5 * page - 1, 12 * page, -1], [39 * page + 3, 40 * page, 41 * page + 1, 3 * page - 1, 2 * page, 9 * page]]]
    run_select(lens, 4, page, pages, append=append, seed=pages + page)
    run_select(lens, 3, page, pages, first_pages=0, last_pages=pages, append=append, seed=pages, strided=True)


@pytest.mark.parametrize("g", [1, 2, 3, 5, 8, 9, 16, 17, 64])
@pytest.mark.parametrize("four", [False, True])
def test_select_head_layouts_and_both_kinds_of_cache(g, four):
    run_select([[[300, 40, 90], [16, 220, -1]], [[700, 3, 64], [128, 127, 129]]], g, 16, 5, four=four, layer=1, seed=g)


def test_select_long_and_many_units():
    run_select([[[9000, 8]]], 2, 8, 300, first_pages=2, last_pages=3, seed=1)              # more pages than threads of a block
    run_select(np.random.default_rng(4).integers(-1, 400, size=(1, 2, 150)), 2, 8, 7, seed=2)


def test_select_equal_scores_go_to_the_lower_pages():
    def change(host, cache, bounds):
        bounds[:] = bounds[:1]
    _, _, _, table, _, _, _, _ = run_select([[[16 * 100]]], 4, 16, 11, last_pages=2, seed=3, change=change)

    def few(host, cache, bounds):                                         # four levels, many pages on each
        bounds[:] = bounds[torch.arange(bounds.shape[0], device="cuda") % 4]
    run_select([[[16 * 100, 16 * 77 + 5]]], 4, 16, 40, seed=4, change=few)


def test_select_bounds_that_are_no_numbers_and_pages_that_are_none():
    def change(host, cache, bounds):
        row = host["table"][0, 0, 0]
        for i, x in ((3, float("nan")), (9, float("inf")), (12, float("-inf"))):
            bounds[int(row[i]), :, 9] = x
        for tbl in (host["table"], cache.tensors[2]):
            tbl[0, 0, 0, 5] = -1
            tbl[0, 0, 0, 6] = 10 ** 9
            tbl[0, 0, 1, 0] = -3
    for pages in (5, 29, 31):                                             # 31 of 32: one of those that are none as well
        *_, st, _, _ = run_select([[[16 * 31 + 2, 40]]], 2, 16, pages, seed=5, change=change)
        assert st[0, 0, 1] == 8 and (st[0, 0, 0] == 8) == (pages == 31)


def test_select_queries_that_are_no_numbers_infinite_or_nothing():
    from paper_2507_08143_b200 import binding as B
    lens = np.array([[[500, 700, 300, 600, 16 * 40]]], np.int32)
    host, cache, len_d = make_cache(lens, 16, 1, 40)
    bounds = torch.randn(host["k"].shape[0], 2, 128, generator=torch.Generator().manual_seed(1)).sort(1).values
    bounds[int(host["table"][0, 0, 4, 7])] *= 1e38                        # sums beyond fp32
    bounds = bounds.bfloat16().cuda()
    q = torch.randn(5, 3, 128, generator=torch.Generator().manual_seed(2)).bfloat16()
    q[0, 1, 3] = float("nan"); q[1, 2, 5] = float("inf"); q[2] = 0; q[3, 0] = -q[3, 0].abs()
    for pages in (3, 20):
        table, short = torch.empty(1, 1, 5, pages, dtype=torch.int32, device="cuda"), torch.empty(1, 1, 5, dtype=torch.int32, device="cuda")
        B.paged_select(cache, 0, 3, q.cuda(), len_d, bounds, table, short, B.alloc_paged_select_workspace(cache, 700), 700)
        with np.errstate(invalid="ignore", over="ignore"):
            want, want_len, _ = ro.select(host, 0, 3, H.bits(q), lens, H.bits(bounds), pages, 1, 1, None, 700)
        np.testing.assert_array_equal(table[0].cpu().numpy(), want)
        np.testing.assert_array_equal(short[0].cpu().numpy(), want_len)


def test_select_units_that_do_not_fit():
    *_, st, _, _ = run_select([[[50, 39, 40, -1]]], 2, 16, 2, max_length=40, seed=6)
    assert st.tolist() == [[[16, 0, 16, 0]]]


@pytest.mark.parametrize("four", [False, True])
def test_attention_over_the_chosen_pages(four):
    """Bounds, choice and attention together: the step attends to what the choice says, the new token lands in its own page and slot."""
    from paper_2507_08143_b200 import binding as B
    lens = np.array([[[500, 0, 77, 1500], [20, 333, -1, 64]]], np.int32)
    g, pages = 4, 6
    host, cache, len_d = (make_cache4 if four else make_cache)(lens, 16, 1, 8)
    bounds = fresh_bounds(host)
    B.paged_bounds(cache, len_d, bounds, 1500)
    before = H.bits(bounds)
    gen = torch.Generator().manual_seed(1)
    q, kn, vn = (torch.randn(4, n, 128, generator=gen).bfloat16() for n in (2 * g, 2, 2))
    table, short = torch.empty(1, 2, 4, pages, dtype=torch.int32, device="cuda"), torch.empty(1, 2, 4, dtype=torch.int32, device="cuda")
    k, v, _, mass, pos = cache.tensors
    few = type(cache)(k, v, table, mass=mass, positions=pos)
    opt = B.decode_options(g, pages * 16, accumulate=True)
    out, lse = torch.empty(4, 2 * g, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(4, 2 * g, device="cuda")
    B.paged_select(cache, 0, g, q.cuda(), len_d, bounds, table, short, B.alloc_paged_select_workspace(cache, 1501), 1501, k_new=kn.cuda())
    B.paged_attention(few, 0, opt, q.cuda(), short, out, B.alloc_paged_attention_workspace(few, opt), k_new=kn.cuda(), v_new=vn.cuda(), lse_out=lse)
    want, want_len, _ = ro.select(host, 0, g, H.bits(q), lens, before, pages, 1, 1, H.bits(kn))
    reduced = dict(host, table=want[None])
    att = ro.attention4 if four else po.attention
    ref, ref_lse, after, info = att(reduced, 0, H.bits(q), want_len[None], np.float64(np.float32(128 ** -0.5)), k_new=H.bits(kn), v_new=H.bits(vn),
                                    accumulate=True)
    o, ls = out.double().cpu().numpy(), lse.double().cpu().numpy()
    for (h, b), (at, p, pv, mag) in info.items():
        rows = slice(h * g, (h + 1) * g)
        dy, rel, tol = attention4_bounds(g, pv, ref[b, rows], mag, 0.0, len(at)) if four else attention_bounds(g, p, pv, ref[b, rows], mag, 128 ** -0.5, 0.0, len(at))
        assert np.all(np.abs(o[b, rows] - ref[b, rows]) <= tol)
        assert np.all(np.abs(ls[b, rows] - ref_lse[b, rows]) <= dy + rel + 2.0 ** -22 * np.abs(ref_lse[b, rows]))
    np.testing.assert_array_equal(k.cpu().numpy() if four else H.bits(k), after["k"])
    for (h, b) in np.ndindex(2, 4):                                       # where the whole cache expects it
        if lens[0, h, b] >= 0:
            a = po.slot_of(host, (0, h, b), int(lens[0, h, b]))
            np.testing.assert_array_equal(after["k"][a], ro.hold4(H.bits(kn)[b, h]) if four else H.bits(kn)[b, h])


def test_select_follows_its_inputs_in_a_graph():
    from paper_2507_08143_b200 import binding as B
    lens = np.array([[[500, 0, 77, 1500], [20, 333, -1, 64]]], np.int32)
    host, cache, len_d = make_cache(lens, 16, 40, 11)
    bounds = fresh_bounds(host)
    B.paged_bounds(cache, len_d, bounds, 1500)
    start = bounds.clone()
    q, kn = torch.randn(4, 8, 128, device="cuda").bfloat16(), torch.randn(4, 2, 128, device="cuda").bfloat16()
    ws = B.alloc_paged_select_workspace(cache, 1540)
    table, short = torch.empty(1, 2, 4, 9, dtype=torch.int32, device="cuda"), torch.empty(1, 2, 4, dtype=torch.int32, device="cuda")

    def call(t, s):
        B.paged_select(cache, 0, 4, q, len_d, bounds, t, s, ws, 1540, last_pages=2, k_new=kn)
    call(table, short)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(table, short)
    for step in (0, 1, 33):
        q.normal_(); kn.normal_()
        len_d.copy_(torch.from_numpy(np.where(lens >= 0, lens + step, lens)))
        bounds.copy_(start)
        graph.replay()
        got = [table.clone(), short.clone(), bounds.clone()]
        bounds.copy_(start)
        t, s = torch.empty_like(table), torch.empty_like(short)
        call(t, s)
        for a, b in zip(got, (t, s, bounds)):
            assert torch.equal(a, b)
