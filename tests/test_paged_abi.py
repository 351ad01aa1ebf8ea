"""Host-side checks of the paged-cache entry points that need no GPU: every refusal comes back before anything is enqueued,
workspace sizes, and the oracle's own pins."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from paper_2507_08143_b200 import binding as B

dev = ctypes.c_void_p


def _cache(**kw):
    d = dict(k_pages=1 << 20, v_pages=1 << 30, stride_page=16 * 128, stride_token=128, mass=1 << 16, positions=1 << 17,
             page_table=1 << 18, n_pages=64, page_tokens=16, max_pages=8, layers=2, heads=2, batch=3, d=128)
    d.update(kw)
    return B.CompactorPagedCache(**d)


BAD_CACHES = [
    (dict(k_pages=0), -1), (dict(v_pages=0), -1), (dict(page_table=0), -1), (dict(k_pages=(1 << 20) + 8), -1),
    (dict(v_pages=(1 << 20) + 2), -1), (dict(mass=(1 << 16) + 2), -1), (dict(positions=(1 << 17) + 1), -1),
    (dict(page_table=(1 << 18) + 2), -1), (dict(d=64), -2), (dict(layers=0), -1), (dict(heads=0), -1), (dict(batch=0), -1),
    (dict(n_pages=0), -1), (dict(max_pages=0), -1), (dict(page_tokens=4), -1), (dict(page_tokens=24), -1),
    (dict(page_tokens=2048), -1), (dict(stride_token=120), -1), (dict(stride_token=132), -1), (dict(stride_page=16 * 128 + 4), -1),
    (dict(stride_page=15 * 128), -1), (dict(max_pages=1 << 28), -1), (dict(layers=300, heads=300), -1),
]


def _attention(cache=None, layer=0, opt=None, q=(1 << 22, 512, 128), kn=(1 << 23, 256, 128), vn=(1 << 24, 256, 128), lengths=1 << 12,
               out=(1 << 25, 512, 128), ws=1 << 26, ws_bytes=1 << 40):
    rows = lambda r: B.CompactorRows(*r)
    return B.LIB.compactor_paged_attention(ctypes.byref(cache or _cache()), layer, ctypes.byref(opt or B.decode_options(2, 100)), rows(q),
                                           rows(kn), rows(vn), None, dev(lengths), rows(out), None, None, dev(ws), ws_bytes, None)


def test_attention_refusals():
    for kw, code in BAD_CACHES:
        assert _attention(_cache(**kw)) == code, kw
    assert _attention(layer=-1) == -1 and _attention(layer=2) == -1
    for opt, code in ((B.decode_options(0, 100), -1), (B.decode_options(65, 100), -2), (B.decode_options(2, 0), -1),
                      (B.decode_options(2, 100, scale=0.0), -1), (B.decode_options(2, 100, scale=math.nan), -1),
                      (B.decode_options(2, 100, scale=math.inf), -1), (B.decode_options(2, 100, softcap=-1.0), -1),
                      (B.decode_options(2, 100, softcap=math.nan), -1)):
        assert _attention(opt=opt) == code
    assert _attention(_cache(mass=0), opt=B.decode_options(2, 100, accumulate=True)) == -1
    for bad in ((0, 512, 128), ((1 << 22) + 8, 512, 128), (1 << 22, 516, 128), (1 << 22, 512, 132), (1 << 22, -512, 128)):
        assert _attention(q=bad) == -1 and _attention(out=bad) == -1 and _attention(vn=bad) == -1
    assert _attention(kn=(0, 0, 0)) == -1                                # k_new without v_new, and the other way round
    assert _attention(vn=(0, 0, 0)) == -1
    assert _attention(out=(1 << 25, 512, 0)) == -1 and _attention(out=(1 << 25, 0, 128)) == -1       # rows on top of each other
    assert _attention(lengths=0) == -1 and _attention(ws=0) == -1 and _attention(ws=(1 << 26) + 64) == -1
    assert _attention(ws_bytes=256) == -3
    huge = _cache(heads=8, batch=8000, max_pages=1 << 20, page_tokens=1024, stride_page=1024 * 128)
    assert _attention(huge, opt=B.decode_options(2, 1 << 30), out=(1 << 25, 2048, 128)) == -5


def test_attention_workspace_bytes():
    c = _cache(heads=8, batch=4, max_pages=512)
    size = lambda cache, opt: B.LIB.compactor_paged_attention_workspace_bytes(ctypes.byref(cache), ctypes.byref(opt))
    plain, acc = size(c, B.decode_options(4, 8192)), size(c, B.decode_options(4, 8192, accumulate=True))
    assert 0 < plain < acc and plain % 256 == 0
    assert acc - plain == 8 * 4 * 8192 * 4 * 4                            # one score per token and query head
    assert size(c, B.decode_options(4, 1 << 20, accumulate=True)) == acc   # no more than the table's pages hold
    assert size(c, B.decode_options(0, 8192)) == 0 and size(_cache(d=64), B.decode_options(4, 64)) == 0


def _fill(cache=None, first_layer=0, shape=None, k=(1 << 40, 1 << 20, 1 << 16, 128), v=(1 << 41, 1 << 20, 1 << 16, 128), idx=1 << 13,
          offs=None, keep=(5, 0, 7)):
    shape = shape or B.Shape(1, 2, 128, 48, [10, 0, 20])
    keep = None if keep is None else (ctypes.c_int32 * len(keep))(*keep)
    return B.LIB.compactor_paged_fill(ctypes.byref(cache or _cache()), first_layer, ctypes.byref(shape.c), B.CompactorMat(*k),
                                      B.CompactorMat(*v), dev(idx), dev(offs), keep, None, None, None, None, None, None)


def test_fill_refusals():
    for kw, code in BAD_CACHES:
        if set(kw) != {"heads"} and set(kw) != {"batch"}:
            assert _fill(_cache(**kw)) == code, kw
    assert _fill(shape=B.Shape(1, 3, 128, 48, [10, 0, 20])) == -1         # other heads, batch, layers than the cache's
    assert _fill(shape=B.Shape(1, 2, 128, 48, [10, 20]), keep=(5, 7)) == -1
    assert _fill(shape=B.Shape(3, 2, 128, 48, [10, 0, 20])) == -1 and _fill(first_layer=2) == -1 and _fill(first_layer=-1) == -1
    assert _fill(shape=B.Shape(1, 2, 64, 48, [10, 0, 20])) == -2
    assert _fill(keep=None) == -1 and _fill(keep=(11, 0, 7)) == -1 and _fill(keep=(-1, 0, 7)) == -1
    assert _fill(idx=None, offs=1 << 14) == -1                            # offsets of a selection without its indices
    for bad in ((0, 0, 0, 128), ((1 << 40) + 8, 0, 0, 128), (1 << 40, 0, 0, 64), (1 << 40, 4, 0, 128)):
        assert _fill(k=bad) == -1 and _fill(v=bad) == -1


def _evict(cache=None, first_layer=0, layers=1, lengths=1 << 12, budgets=1 << 13, nxt=1 << 14, recent=4, max_length=100, out=1 << 15):
    return B.LIB.compactor_paged_evict(ctypes.byref(cache or _cache()), first_layer, layers, dev(lengths), dev(budgets), dev(nxt), recent,
                                       max_length, dev(out), None, None)


def test_evict_refusals():
    for kw, code in BAD_CACHES:
        assert _evict(_cache(**kw)) == code, kw
    assert _evict(layers=0) == -1 and _evict(layers=3) == -1 and _evict(first_layer=2) == -1 and _evict(first_layer=-1) == -1
    assert _evict(lengths=None) == -1 and _evict(budgets=None) == -1 and _evict(out=None) == -1
    assert _evict(nxt=None) == -1 and _evict(recent=-1) == -1 and _evict(max_length=0) == -1
    assert _evict(_cache(mass=0)) == -1 and _evict(_cache(positions=0)) == -1
    assert _evict(_cache(max_pages=1 << 16), max_length=393217) == -5


def test_binding_refuses_tensors_of_other_shapes():
    k = torch.zeros(4, 16, 128, dtype=torch.bfloat16)
    table = torch.zeros(1, 2, 3, 2, dtype=torch.int32)
    c = B.PagedCache(k, k.clone(), table, mass=torch.zeros(4, 16), positions=torch.zeros(4, 16, dtype=torch.int32))
    assert (c.layers, c.heads, c.batch, c.max_pages, c.n_pages, c.page_tokens, c.d) == (1, 2, 3, 2, 4, 16, 128)
    for bad in (dict(k_pages=k.float()), dict(v_pages=k[:, :8]), dict(page_table=table[0]), dict(page_table=table.long()),
                dict(mass=torch.zeros(4, 8)), dict(positions=torch.zeros(4, 16)), dict(v_pages=torch.zeros(4, 128, 16, dtype=torch.bfloat16).transpose(1, 2))):
        with pytest.raises(ValueError):
            B.PagedCache(**{**dict(k_pages=k, v_pages=k, page_table=table), **bad})


def test_calls_refuse_tensors_of_other_shapes_types_and_devices():
    # every wrong tensor is named; with all of them right, a cache outside the current CUDA device is what is left to refuse
    k = torch.zeros(4, 16, 128, dtype=torch.bfloat16)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)
    c = B.PagedCache(k, k.clone(), i32(1, 2, 3, 2), mass=torch.zeros(4, 16), positions=i32(4, 16))
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)
    ok = dict(q=bf(3, 4, 128), lengths=i32(1, 2, 3), out=bf(3, 4, 128), workspace=bf(100), k_new=bf(3, 2, 128), v_new=bf(3, 2, 128),
              new_positions=i32(3), lse_out=torch.zeros(3, 4), status=i32(1, 2, 3))
    call = lambda **kw: B.paged_attention(c, 0, B.decode_options(2, 20), **{**ok, **kw})
    with pytest.raises(ValueError, match="current CUDA device"):
        call()
    for name, bad in (("q", bf(3, 5, 128)), ("q", bf(2, 4, 128)), ("q", bf(3, 4, 64)), ("q", torch.zeros(3, 4, 128)), ("q", bf(3, 128, 4).transpose(1, 2)),
                      ("out", bf(3, 2, 128)), ("out", bf(12, 128)), ("k_new", bf(3, 4, 128)), ("v_new", bf(3, 2, 128).half()),
                      ("lengths", i32(5)), ("lengths", i32(1, 2, 3).long()), ("lengths", i32(1, 2, 6)[..., ::2]), ("new_positions", i32(4)),
                      ("lse_out", torch.zeros(3, 3)), ("lse_out", bf(3, 4)), ("status", i32(2)), ("workspace", bf(10, 10).t()[::2])):
        with pytest.raises(ValueError, match=name):
            call(**{name: bad})
    for name in ("k_new", "v_new"):
        with pytest.raises(ValueError, match="come together"):
            call(**{name: None})
    for name in ("q", "lengths", "out", "workspace"):
        with pytest.raises(TypeError):
            call(**{name: None})
        with pytest.raises(TypeError):
            call(**{name: 7})
    shape = B.Shape(1, 2, 128, 48, [4, 0, 3])
    ok_f = dict(k_cache=bf(1, 2, 7, 128), v_cache=bf(1, 2, 7, 128), keep_counts=[2, 0, 3], idx=i32(1, 2, 5), head_offsets=i32(1, 3, 3),
                mass_in=torch.zeros(1, 2, 7), first_position=i32(3), lengths=i32(6), lengths_out=i32(6), status=i32(6))
    fill = lambda **kw: B.paged_fill(c, shape, **{**ok_f, **kw})
    with pytest.raises(ValueError, match="current CUDA device"):
        fill()
    for name, bad in (("k_cache", bf(1, 2, 8, 128)), ("v_cache", torch.zeros(1, 2, 7, 128)), ("v_cache", bf(1, 2, 128, 7).transpose(2, 3)),
                      ("keep_counts", [2, 0]), ("idx", i32(9)), ("idx", i32(10).long()), ("head_offsets", i32(8)), ("mass_in", torch.zeros(13)),
                      ("first_position", i32(2)), ("lengths", i32(5)), ("lengths_out", torch.zeros(6)), ("status", i32(7))):
        with pytest.raises(ValueError, match=name):
            fill(**{name: bad})
    with pytest.raises(TypeError):
        fill(keep_counts=None)
    with pytest.raises(TypeError):
        fill(keep_counts=[2, 0, "3"])
    ok_e = dict(lengths=i32(6), budgets=i32(6), lengths_out=i32(6), max_length=32, recent=1, next_position=i32(3), status=i32(6))
    evict = lambda **kw: B.paged_evict(c, **{**ok_e, **kw})
    with pytest.raises(ValueError, match="current CUDA device"):
        evict()
    for name, bad in (("lengths", i32(5)), ("budgets", i32(6).long()), ("lengths_out", i32(7)), ("next_position", i32(6)), ("status", i32(1))):
        with pytest.raises(ValueError, match=name):
            evict(**{name: bad})
    with pytest.raises(OverflowError):
        evict(max_length=1 << 40)


def _small(seed=0, layers=1, heads=1, batch=1, page=8, max_pages=3):
    rng = np.random.default_rng(seed)
    n_pages = layers * heads * batch * max_pages
    bits = lambda *s: (rng.standard_normal(s).astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)
    return dict(k=bits(n_pages, page, 4), v=bits(n_pages, page, 4), mass=rng.random((n_pages, page), dtype=np.float32),
                positions=np.zeros((n_pages, page), np.int32),
                table=rng.permutation(n_pages).astype(np.int32).reshape(layers, heads, batch, max_pages)), rng, bits


def test_oracle_attention_pins():
    c, rng, bits = _small()
    lengths = np.array([[[11]]], np.int32)
    zero_q = np.zeros((1, 2, 4), np.uint16)
    out, lse, after, _ = po.attention(c, 0, zero_q, lengths, 0.5, accumulate=True)      # equal scores: the mean of the rows
    rows = np.array([po.bf16_bits_to_f64(c["v"][po.slot_of(c, (0, 0, 0), t)]) for t in range(11)])
    np.testing.assert_allclose(out[0], np.tile(rows.mean(0), (2, 1)), rtol=1e-12)
    np.testing.assert_allclose(lse, math.log(11), rtol=1e-12)
    gained = after["mass"] - c["mass"]
    np.testing.assert_allclose(sorted(gained.ravel())[-11:], 2 / 11, rtol=1e-6)
    assert np.count_nonzero(gained) == 11
    q = bits(1, 2, 4)
    out1, lse1, _, _ = po.attention(c, 0, q, lengths, 0.5)
    out2, lse2, _, _ = po.attention(c, 0, q, lengths, 0.5, softcap=1e6)                  # a cap far away changes nothing
    np.testing.assert_allclose(out1, out2, atol=1e-9)
    # the token appended equals a cache that had it
    longer = po.attention(c, 0, q, lengths + 1, 0.5)
    at = po.slot_of(c, (0, 0, 0), 11)
    appended = po.attention(c, 0, q, lengths, 0.5, k_new=c["k"][at][None, None], v_new=c["v"][at][None, None])
    np.testing.assert_allclose(longer[0], appended[0], rtol=1e-12)
    none = po.attention(c, 0, q, np.array([[[0]]], np.int32), 0.5)
    assert np.all(none[0] == 0) and np.all(none[1] == -np.inf)


def test_oracle_evict_pins():
    c, _, _ = _small(seed=3)
    unit = (0, 0, 0)
    at = [po.slot_of(c, unit, t) for t in range(20)]
    for t in range(20):
        c["mass"][at[t]] = [5, 1, 4, 1, 3, 9, 2, 6, 5, 3, 5, 8, 9, 7, 9, 3, 2, 3, 8, 4][t]
        c["positions"][at[t]] = t
    n = np.array([[[20]]], np.int32)
    after, out = po.evict(c, [unit], n, np.array([[[6]]], np.int32))
    # kept: the 9s (5, 12, 14), the 8s (11, 18) and the 7 (13); holes 0-4 take 11, 12, 13, 14, 18 in order
    assert out[unit] == 6
    assert [int(after["positions"][at[t]]) for t in range(6)] == [11, 12, 13, 14, 18, 5]
    after, _ = po.evict(c, [unit], n, np.array([[[6]]], np.int32), recent=3, next_position=[20])
    assert [int(after["positions"][at[t]]) for t in range(6)] == [12, 14, 17, 18, 19, 5]
    after, out = po.evict(c, [unit], n, np.array([[[20]]], np.int32))
    assert out[unit] == 20 and all(np.array_equal(after[k], c[k]) for k in c)


def test_fill_of_nothing_across_heads():
    """Where no sequence keeps a row, a selection across heads has no indices: an empty tensor, whose address is null."""
    assert _fill(idx=None, offs=1 << 14, keep=(0, 0, 0)) == 0
    assert _fill(idx=None, offs=1 << 14, keep=(0, 0, 1)) == -1


def test_attention_refuses_scales_that_leave_fp32():
    """The kernel works with scale log2(e), scale / softcap and softcap log2(e): one of them infinite gives inf * 0, one of them
    below the normal numbers loses the scores' bits."""
    fine = _attention(opt=B.decode_options(2, 100, scale=1e30, softcap=1e30), ws_bytes=256)
    assert fine == -3 and _attention(opt=B.decode_options(2, 100, scale=1e-30, softcap=1e-30), ws_bytes=256) == -3
    for scale, softcap in ((3e38, 0.0), (1e-39, 0.0), (1.0, 1e-39), (1.0, 3e38), (1e-20, 1e20), (1e20, 1e-20)):
        assert _attention(opt=B.decode_options(2, 100, scale=scale, softcap=softcap), ws_bytes=256) == -1, (scale, softcap)
        assert B.LIB.compactor_paged_attention_workspace_bytes(ctypes.byref(_cache()), ctypes.byref(B.decode_options(2, 100, scale=scale, softcap=softcap))) == 0
