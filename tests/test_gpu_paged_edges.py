"""Calls of the paged cache at the edges of what the header allows."""
import numpy as np
import pytest
import torch

from tests import helpers as H
from tests.test_gpu_paged import make_cache, pools_of, run_attention, run_evict, same_bits

pytestmark = pytest.mark.gpu


def test_fill_of_nothing_across_heads():
    from paper_2507_08143_b200 import binding as B
    _, cache, len_d = make_cache([[[4, -1], [0, 9]]], 8, 2, 8)
    before = pools_of(cache)
    empty = torch.empty(1, 2, 0, 128, dtype=torch.bfloat16, device="cuda")
    out, st = torch.full_like(len_d, 9), torch.full_like(len_d, 9)
    B.paged_fill(cache, B.Shape(1, 2, 128, 48, [0, 0]), empty, empty, [0, 0], idx=torch.empty(1, 0, dtype=torch.int32, device="cuda"),
                 head_offsets=torch.zeros(1, 2, 3, dtype=torch.int32, device="cuda"), lengths=len_d, lengths_out=out, status=st)
    assert torch.equal(out, len_d) and not st.any()
    same_bits(pools_of(cache), before, "nothing")


def test_evict_window_that_begins_below_the_least_position():
    """next_position - recent below -2^31: every token is recent, so the lowest slots stay and nothing moves."""
    from paper_2507_08143_b200 import binding as B
    _, cache, len_d = make_cache([[[50]]], 16, 0, 3)
    before = pools_of(cache)
    out, budgets = torch.zeros_like(len_d), torch.full_like(len_d, 20)
    nxt = torch.tensor([-2 ** 31 + 5], dtype=torch.int32, device="cuda")
    B.paged_evict(cache, len_d, budgets, out, 50, recent=10, next_position=nxt)
    assert int(out) == 20
    same_bits(pools_of(cache), before, "nothing moves")


@pytest.mark.parametrize("units,n", [(16, 40000), (12, 40001), (8, 70000), (9, 70001), (5, 33000)])
def test_evict_of_as_many_long_units_as_the_clusters_differ_for(units, n):
    """Few long units take clusters as large as the GPU has room for beside each other: sizes of 6 to 16 CTAs, whose slices end at
    other places.  Equal weights on both sides of the line, so that ranks are counted across the slices."""
    lengths = np.full((1, 1, units), n, np.int32)
    lengths[0, 0, 1::3] -= np.arange(len(lengths[0, 0, 1::3])) * 1777 + 5        # some of them use fewer CTAs than their cluster has
    budgets = lengths - np.int32(1) - (np.arange(units, dtype=np.int32) * 3001) % (n // 2)
    run_evict(lengths, budgets, page=64, recent=300, weights=lambda u, t: float((t * 7919) % 13), seed=units)


@pytest.mark.parametrize("alias", [False, True])
def test_evict_of_many_units_under_a_bound_for_long_ones(alias):
    """48 ragged units and one that needs a cluster of eight: beyond 66048 tokens all units take the long units' route."""
    rng = np.random.default_rng(14)
    lengths = rng.integers(1, 300, size=(2, 4, 6)).astype(np.int32)
    lengths[0, 1] = [70001, 8257, 20000, 12288, 12289, 0]
    lengths[1, 3, :3] = [-1, 49153, 31]
    budgets = np.maximum(0, lengths - rng.integers(-2, 200, size=lengths.shape)).astype(np.int32)
    budgets[0, 1, :3] = [35000, 1, 19999]
    st = run_evict(lengths, budgets, page=32, recent=16, alias=alias, seed=16)
    assert not st.any()


def test_attention_of_few_and_many_query_heads_over_the_same_pages():
    """64 query heads per KV head, four groups of 16 that share the pages and one new token's row."""
    run_attention([[[300, 16], [15, 1000]]], 64, 8, accumulate=True, seed=64)
    run_attention([[[5000]]], 49, 64, accumulate=True, softcap=20.0, seed=65)
