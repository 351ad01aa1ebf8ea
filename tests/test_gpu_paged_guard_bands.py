"""Guard bands around everything that the paged calls may write: pools, workspace (to the byte), results, status and lengths are
carved out of larger patterned buffers, and what lies outside must keep its pattern."""
import numpy as np
import pytest
import torch

from tests.test_gpu_guard_bands import Guarded
from tests.test_gpu_paged import make_cache, _prefill

pytestmark = pytest.mark.gpu


def _guarded(t):
    g = Guarded(tuple(t.shape), t.dtype)
    g.t.copy_(t)
    return g


def _cache(lengths, page, room, seed):
    """make_cache, its pools and lengths between guard bands."""
    from paper_2507_08143_b200 import binding as B
    _, cache, len_d = make_cache(lengths, page, room, seed, spare=0)
    k, v, table, mass, pos = cache.tensors
    g = dict(k_pages=_guarded(k), v_pages=_guarded(v), mass=_guarded(mass), positions=_guarded(pos), lengths=_guarded(len_d),
             status=_guarded(torch.zeros_like(len_d)))
    return B.PagedCache(g["k_pages"].t, g["v_pages"].t, table, mass=g["mass"].t, positions=g["positions"].t), g


def _check(g, what):
    torch.cuda.synchronize()
    for name, buf in g.items():
        buf.check(f"{what}: {name}")


RAGGED = np.random.default_rng(1).integers(-1, 260, size=(1, 3, 40)).astype(np.int32)


@pytest.mark.parametrize("lengths,g,page", [([[[511]]], 1, 16), ([[[0, 15, 16, 17], [700, -1, 31, 33]]], 5, 8), ([[[9000], [40]]], 16, 64),
                                            ([[[1000, 7]]], 33, 16), (RAGGED, 2, 32)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_attention_writes_nothing_outside_its_buffers(lengths, g, page, accumulate):
    from paper_2507_08143_b200 import binding as B
    lengths = np.asarray(lengths, np.int32)
    _, heads, batch = lengths.shape
    cache, bufs = _cache(lengths, page, 1, g)
    rows = lambda h: torch.randn(batch, h, 128, device="cuda").bfloat16()
    for append in (False, True):
        opt = B.decode_options(g, int(lengths.max()) + append, accumulate=accumulate)
        bufs.update(out=_guarded(rows(heads * g)), lse=_guarded(torch.zeros(batch, heads * g, device="cuda")),
                    workspace=Guarded((B.paged_attention_workspace_bytes(cache, opt),), torch.uint8, 255))
        new = dict(k_new=rows(heads), v_new=rows(heads)) if append else {}
        B.paged_attention(cache, 0, opt, rows(heads * g), bufs["lengths"].t, bufs["out"].t, bufs["workspace"].t, lse_out=bufs["lse"].t,
                          status=bufs["status"].t, **new)
        _check(bufs, f"append {append}")
        assert torch.isfinite(bufs["out"].t.float()).all() and not bufs["status"].t.any()


@pytest.mark.parametrize("page", [8, 64])
def test_fill_and_evict_write_nothing_outside_their_buffers(page):
    from paper_2507_08143_b200 import binding as B
    seqlens = [100, 0, 257, 33]
    lengths = np.array([[[0, 5, 16, -1], [63, 64, 1, 0]]], np.int32)
    cache, bufs = _cache(lengths, page, max(seqlens), page)
    k, v, w = (t.cuda() for t in _prefill(1, 2, seqlens, page))
    B.paged_fill(cache, B.Shape(1, 2, 128, 48, seqlens), k, v, seqlens, mass_in=w, lengths=bufs["lengths"].t, lengths_out=bufs["lengths"].t,
                 status=bufs["status"].t)
    _check(bufs, "fill")
    filled = bufs["lengths"].t.cpu().numpy()
    assert np.array_equal(filled, np.where(lengths < 0, lengths, lengths + np.array(seqlens))) and not bufs["status"].t.any()
    budgets = torch.tensor([[[60, 5, 100, 3], [0, 63, 257, 1]]], dtype=torch.int32, device="cuda")
    B.paged_evict(cache, bufs["lengths"].t, budgets, bufs["lengths"].t, int(filled.max()), recent=2,
                  next_position=torch.full((4,), 200, dtype=torch.int32, device="cuda"), status=bufs["status"].t)
    _check(bufs, "evict")
    assert np.array_equal(bufs["lengths"].t.cpu().numpy(), np.where(filled < 0, filled, np.minimum(filled, budgets.cpu().numpy())))


@pytest.mark.parametrize("units,n", [(3, 20000), (40, 9000)])
def test_evict_of_long_units_writes_nothing_outside_its_buffers(units, n):
    from paper_2507_08143_b200 import binding as B
    lengths = np.full((1, 1, units), n, np.int32)
    lengths[0, 0, 1::2] -= 7001
    cache, bufs = _cache(lengths, 64, 0, units)
    budgets = bufs["lengths"].t - 1500
    out = _guarded(budgets)
    B.paged_evict(cache, bufs["lengths"].t, budgets, out.t, n, status=bufs["status"].t)
    _check({**bufs, "lengths_out": out}, "evict")
    assert torch.equal(out.t, budgets) and not bufs["status"].t.any()
