"""Host-side checks, without a GPU, of the entry points around the paged cache: rows in 4 bits, read-back, bounds and choice of pages, norms with
rotation.  Refusals come back before anything is enqueued; the oracle's own pins."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from oracle import rows_oracle as ro
from oracle.compactor_oracle import bf16_bits_to_f64
from paper_2507_08143_b200 import binding as B
from tests.test_paged_abi import _cache

dev = ctypes.c_void_p
rows = lambda r: B.CompactorRows(*r)


def _cache4(**kw):
    return _cache(**{**dict(stride_page=16 * 80, stride_token=80), **kw})


BAD_CACHES4 = [
    (dict(k_pages=0), -1), (dict(v_pages=0), -1), (dict(page_table=0), -1), (dict(k_pages=(1 << 20) + 8), -1), (dict(v_pages=(1 << 20) + 2), -1),
    (dict(mass=(1 << 16) + 2), -1), (dict(positions=(1 << 17) + 1), -1), (dict(d=64), -2), (dict(layers=0), -1), (dict(n_pages=0), -1),
    (dict(max_pages=0), -1), (dict(page_tokens=4), -1), (dict(page_tokens=24), -1), (dict(page_tokens=2048), -1), (dict(stride_token=96), -1),
    (dict(stride_token=64), -1), (dict(stride_page=16 * 80 + 8), -1), (dict(stride_page=15 * 80), -1), (dict(max_pages=1 << 28), -1),
    (dict(stride_page=16 * 128, stride_token=128), -1),                  # rows of bf16
]


def _attention4(cache=None, layer=0, opt=None, q=(1 << 22, 512, 128), kn=(1 << 23, 256, 128), vn=(1 << 24, 256, 128), lengths=1 << 12,
                out=(1 << 25, 512, 128), ws=1 << 26, ws_bytes=1 << 40):
    return B.LIB.compactor_paged4_attention(ctypes.byref(cache or _cache4()), layer, ctypes.byref(opt or B.decode_options(2, 100)), rows(q),
                                            rows(kn), rows(vn), None, dev(lengths), rows(out), None, None, dev(ws), ws_bytes, None)


def _fill4(cache=None, first_layer=0, shape=None, k=(1 << 40, 1 << 20, 1 << 16, 128), v=(1 << 41, 1 << 20, 1 << 16, 128), keep=(5, 0, 7)):
    shape = shape or B.Shape(1, 2, 128, 48, [10, 0, 20])
    return B.LIB.compactor_paged4_fill(ctypes.byref(cache or _cache4()), first_layer, ctypes.byref(shape.c), B.CompactorMat(*k), B.CompactorMat(*v),
                                       dev(1 << 13), None, (ctypes.c_int32 * len(keep))(*keep), None, None, None, None, None, None)


def _evict4(cache=None, lengths=1 << 12, budgets=1 << 13, nxt=1 << 14, recent=4, max_length=100, out=1 << 15, layers=1):
    return B.LIB.compactor_paged4_evict(ctypes.byref(cache or _cache4()), 0, layers, dev(lengths), dev(budgets), dev(nxt), recent, max_length,
                                        dev(out), None, None)


def _read(four, cache=None, first_layer=0, shape=None, lengths=1 << 12, k=(1 << 40, 1 << 20, 1 << 16, 128), v=(1 << 41, 1 << 20, 1 << 16, 128)):
    shape = shape or B.Shape(1, 2, 128, 48, [10, 0, 20])
    f = B.LIB.compactor_paged4_read if four else B.LIB.compactor_paged_read
    return f(ctypes.byref(cache or (_cache4() if four else _cache())), first_layer, ctypes.byref(shape.c), None, dev(lengths), B.CompactorMat(*k),
             B.CompactorMat(*v), None, None)


def _bounds(four, cache=None, first_layer=0, layers=1, lengths=1 << 12, max_length=100, bounds=1 << 13):
    f = B.LIB.compactor_paged4_bounds if four else B.LIB.compactor_paged_bounds
    return f(ctypes.byref(cache or (_cache4() if four else _cache())), first_layer, layers, None, dev(lengths), max_length, dev(bounds), None, None)


def _select(cache=None, layer=0, opt=(2, 100, 4, 1, 1), q=(1 << 22, 512, 128), kn=(1 << 23, 256, 128), lengths=1 << 12, bounds=1 << 13, table=1 << 14,
            out=1 << 15, ws=1 << 26, ws_bytes=1 << 40):
    return B.LIB.compactor_paged_select(ctypes.byref(cache or _cache4()), layer, ctypes.byref(B.CompactorSelectOptions(*opt)), rows(q), rows(kn),
                                        dev(lengths), dev(bounds), dev(table), dev(out), None, dev(ws), ws_bytes, None)


def test_caches_of_the_other_kind_and_bad_ones_are_refused():
    for kw, code in BAD_CACHES4:
        c = _cache4(**kw)
        assert _attention4(c) == code and _evict4(c) == code and _read(True, c) == code and _bounds(True, c) == code, kw
        assert _fill4(c) == code, kw
        if kw != dict(stride_page=16 * 128, stride_token=128):
            assert _select(c) == code, kw
    four, plain = _cache4(), _cache()
    assert _read(False, four) == -1 and _bounds(False, four) == -1
    assert B.LIB.compactor_paged_evict(ctypes.byref(four), 0, 1, dev(1 << 12), dev(1 << 13), dev(1 << 14), 4, 100, dev(1 << 15), None, None) == -1
    size = lambda f, c: f(ctypes.byref(c), ctypes.byref(B.decode_options(2, 100)))
    assert size(B.LIB.compactor_paged_attention_workspace_bytes, four) == 0 and size(B.LIB.compactor_paged4_attention_workspace_bytes, plain) == 0
    assert size(B.LIB.compactor_paged4_attention_workspace_bytes, four) > 0


def test_attention4_refusals():
    assert _attention4(layer=-1) == -1 and _attention4(layer=2) == -1
    for opt, code in ((B.decode_options(0, 100), -1), (B.decode_options(65, 100), -2), (B.decode_options(2, 0), -1), (B.decode_options(2, 100, scale=0.0), -1),
                      (B.decode_options(2, 100, scale=math.nan), -1), (B.decode_options(2, 100, softcap=-1.0), -1), (B.decode_options(2, 100, scale=3e38), -1)):
        assert _attention4(opt=opt) == code
    assert _attention4(_cache4(mass=0), opt=B.decode_options(2, 100, accumulate=True)) == -1
    for bad in ((0, 512, 128), ((1 << 22) + 8, 512, 128), (1 << 22, 516, 128), (1 << 22, -512, 128)):
        assert _attention4(q=bad) == -1 and _attention4(out=bad) == -1 and _attention4(vn=bad) == -1
    assert _attention4(kn=(0, 0, 0)) == -1 and _attention4(out=(1 << 25, 512, 0)) == -1
    assert _attention4(lengths=0) == -1 and _attention4(ws=0) == -1 and _attention4(ws=(1 << 26) + 64) == -1 and _attention4(ws_bytes=256) == -3


def test_fill4_evict4_and_read_refusals():
    assert _fill4(shape=B.Shape(1, 3, 128, 48, [10, 0, 20])) == -1 and _fill4(first_layer=2) == -1 and _fill4(keep=(11, 0, 7)) == -1
    assert _evict4(lengths=None) == -1 and _evict4(recent=-1) == -1 and _evict4(_cache4(mass=0)) == -1 and _evict4(layers=3) == -1
    assert _evict4(_cache4(max_pages=1 << 16), max_length=393217) == -5
    for four in (False, True):
        assert _read(four, shape=B.Shape(1, 3, 128, 48, [10, 0, 20])) == -1 and _read(four, shape=B.Shape(1, 2, 128, 48, [10, 20])) == -1
        assert _read(four, first_layer=2) == -1 and _read(four, first_layer=-1) == -1 and _read(four, lengths=None) == -1
        assert _read(four, shape=B.Shape(1, 2, 64, 48, [10, 0, 20])) == -2
        for bad in ((0, 0, 0, 128), ((1 << 40) + 8, 0, 1 << 16, 128), (1 << 40, 0, 1 << 16, 64), (1 << 40, 0, 0, 128)):      # the last: heads on top of each other
            assert _read(four, k=bad) == -1 and _read(four, v=bad) == -1
        assert _read(four, shape=B.Shape(2, 2, 128, 48, [10, 0, 20]), k=(1 << 40, 0, 1 << 16, 128)) == -1


def test_bounds_and_select_refusals():
    for four in (False, True):
        assert _bounds(four, layers=0) == -1 and _bounds(four, layers=3) == -1 and _bounds(four, first_layer=2) == -1 and _bounds(four, lengths=None) == -1
        assert _bounds(four, max_length=0) == -1 and _bounds(four, bounds=None) == -1 and _bounds(four, bounds=(1 << 13) + 8) == -1
    for opt, code in (((0, 100, 4, 1, 1), -1), ((65, 100, 4, 1, 1), -2), ((2, 0, 4, 1, 1), -1), ((2, 100, 0, 0, 1), -1), ((2, 100, 4, -1, 1), -1),
                      ((2, 100, 4, 1, 0), -1), ((2, 100, 4, 3, 2), -1), ((2, 100, 4, 1 << 30, 1 << 30), -1)):
        assert _select(opt=opt) == code, opt
    assert _select(layer=2) == -1 and _select(q=(0, 0, 0)) == -1 and _select(kn=((1 << 23) + 8, 256, 128)) == -1 and _select(lengths=None) == -1
    assert _select(bounds=None) == -1 and _select(table=None) == -1 and _select(out=None) == -1 and _select(out=1 << 12) == -1
    assert _select(ws=None) == -1 and _select(ws=(1 << 26) + 128) == -1 and _select(ws_bytes=8) == -3
    big = _cache4(max_pages=1 << 16)
    assert _select(big, opt=(2, 1 << 20, 4, 1, 1)) == -5                   # 65536 pages
    size = B.LIB.compactor_paged_select_workspace_bytes
    assert size(ctypes.byref(big), 1 << 20) == 0 and size(ctypes.byref(_cache()), 0) == 0 and size(ctypes.byref(_cache(d=64)), 100) == 0
    assert size(ctypes.byref(_cache()), 100) == 2 * 256 and size(ctypes.byref(_cache4(heads=8, batch=4, max_pages=512)), 8192) == 2 * 8 * 4 * 512 * 4


def test_select_refuses_tables_longer_than_a_cache_may_have():
    """2^31 - 1 pages would run past the end of an int; so would a cache whose table they are."""
    for pages in (2 ** 31 - 1, 2 ** 31 - 600, 2 ** 28):
        assert _select(opt=(2, 100, pages, 1, 1)) == -5, pages


def test_select_refuses_to_write_what_it_reads():
    """lengths_out or table_out inside the cache's own (two layers of 2 x 3 units), not only where they begin."""
    c = _cache4()
    units = c.heads * c.batch
    assert c.layers >= 2
    for n in (1, units, c.layers * units - 1):
        assert _select(out=(1 << 12) + 4 * n) == -1 and _select(out=(1 << 12) - 4 * min(n, units - 1)) == -1, n
    inside = c.page_table + 4 * (c.layers * units * c.max_pages - 1)
    assert _select(table=c.page_table) == -1 and _select(table=inside) == -1 and _select(table=c.page_table - 4) == -1


def _norm(o=(4, 2, 128, 128, 0, 1e-6), tokens=5, q=(1 << 20, 1024, 128), k=(1 << 21, 1024, 128), qw=1 << 12, kw=1 << 12, pos=1 << 13, freq=1 << 14,
          qo=(1 << 22, 512, 128), ko=(1 << 23, 256, 128), kp=(0, 0, 0)):
    return B.LIB.compactor_norm_rope(ctypes.byref(B.CompactorNormRopeOptions(*o)), tokens, rows(q), rows(k), dev(qw), dev(kw), dev(pos), dev(freq),
                                     rows(qo), rows(ko), rows(kp), None)


def test_norm_rope_refusals():
    for o, code in (((-1, 2, 128, 128, 0, 1e-6), -1), ((0, 0, 128, 128, 0, 1e-6), -1), ((4, 2, 64, 64, 0, 1e-6), -2), ((4, 2, 128, 144, 0, 1e-6), -2),
                    ((4, 2, 128, 24, 0, 1e-6), -2), ((4, 2, 128, -16, 0, 1e-6), -2), ((4, 2, 128, 128, 2, 1e-6), -1), ((4, 2, 128, 128, 0, -1.0), -1),
                    ((4, 2, 128, 128, 0, math.nan), -1), ((4, 2, 128, 128, 0, math.inf), -1), ((70000, 2, 128, 128, 0, 0.0), -1)):
        assert _norm(o) == code, o
    assert _norm(tokens=-1) == -1 and _norm(tokens=1 << 31) == -1 and _norm(pos=None) == -1 and _norm(freq=None) == -1 and _norm(pos=(1 << 13) + 1) == -1
    for bad in ((0, 0, 0), ((1 << 20) + 8, 1024, 128), (1 << 20, 1020, 128), (1 << 20, -1024, 128)):
        assert _norm(q=bad) == -1 and _norm(k=bad) == -1 and _norm(qo=bad) == -1 and _norm(ko=bad) == -1
        if bad[0]:
            assert _norm(kp=bad) == -1
    assert _norm(qo=(1 << 22, 512, 0)) == -1 and _norm(qo=(1 << 22, 0, 128)) == -1 and _norm(kp=(1 << 22, 0, 128)) == -1       # rows on top of each other
    assert _norm(qw=(1 << 12) + 8) == -1 and _norm(kw=(1 << 12) + 2) == -1
    assert _norm(o=(4, 0, 128, 128, 0, 1e-6), kp=(1 << 24, 256, 128)) == -1
    assert _norm(tokens=0, q=(0, 0, 0), pos=None) == 0                    # of nothing there are no pointers


def test_binding_refuses_other_tensors():
    u8 = torch.zeros(4, 16, 80, dtype=torch.uint8)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)
    c = B.PagedCache4(u8, u8.clone(), i32(1, 2, 3, 2), mass=torch.zeros(4, 16), positions=i32(4, 16))
    assert (c.layers, c.heads, c.batch, c.max_pages, c.n_pages, c.page_tokens, c.d) == (1, 2, 3, 2, 4, 16, 128)
    for bad in (dict(k_pages=u8.view(torch.int8)), dict(v_pages=u8[:, :8]), dict(k_pages=u8[..., :64], v_pages=u8[..., :64]), dict(page_table=i32(2, 3, 2)),
                dict(mass=torch.zeros(4, 8)), dict(k_pages=torch.zeros(4, 16, 96, dtype=torch.uint8)[..., :80], v_pages=torch.zeros(4, 16, 96, dtype=torch.uint8)[..., :80])):
        with pytest.raises(ValueError):
            B.PagedCache4(**{**dict(k_pages=u8, v_pages=u8, page_table=i32(1, 2, 3, 2)), **bad})
    plain = B.PagedCache(bf(4, 16, 128), bf(4, 16, 128), i32(1, 2, 3, 2))
    shape = B.Shape(1, 2, 128, 48, [4, 0, 3])
    calls = {
        "read": (lambda cache, **kw: B.paged_read(cache, shape, **kw), dict(lengths=i32(6), k_out=bf(1, 2, 7, 128), v_out=bf(1, 2, 7, 128), first=i32(6), status=i32(6)),
                 [("lengths", i32(5)), ("k_out", bf(1, 2, 8, 128)), ("v_out", torch.zeros(1, 2, 7, 128)), ("first", i32(6).long()), ("status", i32(1))]),
        "bounds": (B.paged_bounds, dict(lengths=i32(6), bounds=bf(4, 2, 128), max_length=32, first=i32(6), status=i32(6)),
                   [("lengths", i32(7)), ("bounds", bf(4, 128)), ("bounds", torch.zeros(4, 2, 128)), ("first", torch.zeros(6))]),
        "select": (lambda cache, **kw: B.paged_select(cache, 0, 2, **kw),
                   dict(q=bf(3, 4, 128), lengths=i32(6), bounds=bf(4, 2, 128), table_out=i32(1, 2, 3, 2), lengths_out=i32(1, 2, 3), workspace=bf(256), max_length=32,
                        k_new=bf(3, 2, 128), status=i32(6)),
                   [("q", bf(3, 2, 128)), ("lengths", i32(5)), ("bounds", bf(3, 2, 128)), ("table_out", i32(2, 3, 2)), ("table_out", i32(1, 2, 2, 3)),
                    ("table_out", i32(1, 2, 3, 4)[..., ::2]), ("lengths_out", i32(5)), ("k_new", bf(3, 4, 128)), ("workspace", bf(10, 10).t()[::2])]),
        "fill": (lambda cache, **kw: B.paged_fill(cache, shape, **kw), dict(k_cache=bf(1, 2, 7, 128), v_cache=bf(1, 2, 7, 128), keep_counts=[2, 0, 3], idx=i32(1, 2, 5)),
                 [("k_cache", bf(1, 2, 8, 128)), ("idx", i32(9))]),
        "attention": (lambda cache, **kw: B.paged_attention(cache, 0, B.decode_options(2, 20), **kw), dict(q=bf(3, 4, 128), lengths=i32(6), out=bf(3, 4, 128), workspace=bf(100)),
                      [("q", bf(3, 5, 128)), ("out", bf(12, 128))]),
        "evict": (B.paged_evict, dict(lengths=i32(6), budgets=i32(6), lengths_out=i32(6), max_length=32), [("budgets", i32(6).long())]),
    }
    for name, (call, ok, bads) in calls.items():
        for cache in (c, plain):
            with pytest.raises(ValueError, match="current CUDA device"):
                call(cache, **ok)
            for arg, bad in bads:
                with pytest.raises(ValueError, match=arg):
                    call(cache, **{**ok, arg: bad})
        for other in (None, shape, c.c, u8):
            with pytest.raises(TypeError):
                call(other, **ok)
    for arg in ("q", "lengths", "bounds", "table_out", "lengths_out", "workspace"):
        with pytest.raises(TypeError):
            calls["select"][0](c, **{**calls["select"][1], arg: None})
    ok = dict(q=bf(5, 4, 128), k=bf(5, 2, 128), positions=i32(5), inv_freq=torch.zeros(64), q_out=bf(5, 4, 128), k_out=bf(5, 2, 128), k_plain_out=bf(5, 2, 128),
              q_weight=bf(128), k_weight=bf(128))
    with pytest.raises(ValueError, match="current CUDA device"):
        B.norm_rope(**ok)
    for arg, bad in (("q", bf(5, 4, 64)), ("k", bf(4, 2, 128)), ("q_out", bf(5, 3, 128)), ("k_out", torch.zeros(5, 2, 128)), ("k_plain_out", bf(5, 128, 2).transpose(1, 2)),
                     ("positions", i32(4)), ("positions", i32(5).long()), ("inv_freq", torch.zeros(65)), ("inv_freq", torch.zeros(64).double()), ("q_weight", bf(64)),
                     ("k_weight", torch.zeros(128)), ("q_out", None), ("k_out", None), ("inv_freq", None), ("positions", None)):
        with pytest.raises(ValueError, match=arg if arg != "q_out" or bad is not None else "q"):
            B.norm_rope(**{**ok, arg: bad})
    with pytest.raises(ValueError, match="k_plain_out"):
        B.norm_rope(**{**ok, "k": None, "k_out": None})
    with pytest.raises(TypeError):
        B.norm_rope(**{**ok, "q": None, "q_out": None, "k": None, "k_out": None, "k_plain_out": None})
    with pytest.raises(TypeError):
        B.norm_rope(**{**ok, "eps": "small"})


def test_oracle_rows_in_4_bits():
    bits = lambda x: ro.f64_to_bf16_bits(np.asarray(x, np.float64))
    x = np.zeros(128)
    x[:32] = np.arange(32) / 31 * 15 - 3                                  # step 1 exactly: every code is the nearest whole number
    x[32:64] = 2.5
    x[64:96] = np.tile([-1.0, 14.0], 16)
    x[96:] = np.tile([0.0, 7.5, 15.0, 0.5], 8)                            # halves of a step: the lower code
    b = bf16_bits_to_f64(bits(x))
    rows_ = ro.hold4(bits(x))
    v = ro.values4(rows_)
    assert rows_.shape == (80,) and np.all(v[32:64] == 2.5) and np.array_equal(v[64:96], b[64:96])
    np.testing.assert_array_equal(v[:32], np.ceil(b[:32] + 3 - 0.5) - 3)
    np.testing.assert_array_equal(v[96:], np.tile([0.0, 7.0, 15.0, 0.0], 8))
    p = np.ascontiguousarray(rows_[64:]).view(np.uint16)
    np.testing.assert_array_equal(bf16_bits_to_f64(p), [1, -3, 0, 2.5, 1, -1, 1, 0])
    rng = np.random.default_rng(0)
    y = bits(rng.standard_normal((500, 128)) * np.exp(rng.standard_normal((500, 1)) * 3))
    held = ro.hold4(y)
    step = np.repeat(bf16_bits_to_f64(np.ascontiguousarray(held[:, 64:]).view(np.uint16)).reshape(500, 4, 2)[..., 0], 32, 1)
    assert np.all(np.abs(ro.values4(held) - bf16_bits_to_f64(y)) <= step / 2)
    assert np.array_equal(ro.hold4(bits(ro.values4(held)))[:, 64:].shape, held[:, 64:].shape)
    for bad in (np.inf, -np.inf, np.nan):
        z = x.copy(); z[40] = bad
        w = ro.values4(ro.hold4(bits(z)))
        assert np.isnan(w[32:64]).all() and np.isfinite(w[:32]).all() and np.isfinite(w[64:]).all()
    assert np.isnan(ro.values4(ro.hold4(bits(np.tile([3e38, -3e38], 64))))).all()
    for v, want in ((1.0, 0x3F80), (1 + 2.0 ** -8, 0x3F80), (1 + 3 * 2.0 ** -8, 0x3F82), (1 + 2.0 ** -8 + 2.0 ** -40, 0x3F81), (-2.0 ** -126, 0x8080)):
        assert int(ro.f64_to_bf16_bits(np.array(v))) == want


def test_oracle_bounds_and_select_pins():
    rng = np.random.default_rng(1)
    c = dict(k=ro.f64_to_bf16_bits(rng.standard_normal((6, 8, 128))), v=np.zeros((6, 8, 128), np.uint16), mass=np.zeros((6, 8), np.float32),
             positions=np.zeros((6, 8), np.int32), table=np.array([[[[3, 0, 5, 1, 2]]]], np.int32))
    n = np.array([[[35]]], np.int32)
    b = ro.bounds(c, [(0, 0, 0)], n, np.zeros((6, 2, 128), np.uint16))
    k = bf16_bits_to_f64(c["k"])
    np.testing.assert_array_equal(bf16_bits_to_f64(b[3]), [k[3].min(0), k[3].max(0)])
    np.testing.assert_array_equal(bf16_bits_to_f64(b[2]), [k[2, :3].min(0), k[2, :3].max(0)])
    assert not b[4].any()
    q = ro.f64_to_bf16_bits(rng.standard_normal((1, 2, 128)))
    qq = bf16_bits_to_f64(q[0])
    top = {p: (qq @ k[p, : 3 if p == 2 else 8].T).max() for p in (3, 0, 5, 1, 2)}
    score = {p: np.maximum(qq * bf16_bits_to_f64(b[p, 0]), qq * bf16_bits_to_f64(b[p, 1])).sum(1).max() for p in top}
    assert all(score[p] >= top[p] for p in top)                           # no key of the page scores more
    table, out, _ = ro.select(c, 0, 2, q, n, b, 3, 1, 1)
    middle = max((0, 5, 1), key=lambda p: score[p])
    assert table[0, 0].tolist() == [3, middle, 2] and out[0, 0] == 2 * 8 + 3
    table, out, after = ro.select(c, 0, 2, q, np.array([[[24]]], np.int32), b, 9, 0, 1, k_new=np.full((1, 1, 128), 0x4120, np.uint16))
    assert table[0, 0].tolist() == [3, 0, 5, 1] + [-1] * 5 and out[0, 0] == 24 and np.all(after[1] == 0x4120)     # 10.0: first of its page


def test_oracle_norm_rope_pins():
    rng = np.random.default_rng(2)
    x = rng.standard_normal((3, 2, 128))
    freq = 100.0 ** -(np.arange(64) / 64)
    for inter in (False, True):
        y, plain, _ = ro.norm_rope(x, None, 0.0, np.array([0, 5, -7]), freq, inter)
        np.testing.assert_allclose(y[0], x[0], rtol=1e-15)                # no rotation at position 0
        np.testing.assert_allclose((y ** 2).sum(-1), (x ** 2).sum(-1), rtol=1e-12)
        np.testing.assert_array_equal(plain, x)
        back, _, _ = ro.norm_rope(y, None, 0.0, np.array([0, -5, 7]), freq, inter)
        np.testing.assert_allclose(back, x, atol=1e-12)
        # a product of a query and a key depends on the difference of their positions alone
        a, _, _ = ro.norm_rope(x[:1], None, 0.0, np.array([40]), freq, inter)
        b, _, _ = ro.norm_rope(x[1:2], None, 0.0, np.array([37]), freq, inter)
        a2, _, _ = ro.norm_rope(x[:1], None, 0.0, np.array([3]), freq, inter)
        np.testing.assert_allclose((a * b).sum(-1), (a2 * x[1:2]).sum(-1), atol=1e-11)
    y, _, _ = ro.norm_rope(x, np.ones(128), 0.0, np.zeros(3), freq, False)
    np.testing.assert_allclose((y ** 2).mean(-1), 1, rtol=1e-12)
    y, _, _ = ro.norm_rope(np.eye(128)[None, :1] * 2, None, 0.0, np.array([1]), np.array([math.pi / 2] + [0.0] * 31), False)
    np.testing.assert_allclose(y[0, 0, [0, 32]], [0, 2], atol=1e-15)      # a quarter turn takes channel 0 to its partner
