"""Choice of pages by scores next to the least numbers of fp32, where products lose bits or vanish: the choice is still that of sums in 64 bits,
rounded once."""
import numpy as np
import pytest
import torch

from oracle import rows_oracle as ro
from tests import helpers as H
from tests.test_gpu_paged import make_cache

pytestmark = pytest.mark.gpu


def scaled(x, exponent):
    return torch.from_numpy(np.ldexp(x.double().numpy(), exponent).astype(np.float32)).bfloat16()


@pytest.mark.parametrize("q_exponent, exponent", [(-133, 0), (-130, -16), (-130, -22), (-130, -24), (-127, -27), (-76, -76), (-20, -130)])
@pytest.mark.parametrize("g", [1, 4, 11])
def test_scores_next_to_the_least_numbers(q_exponent, exponent, g):
    from paper_2507_08143_b200 import binding as B
    lens = np.array([[[16 * 300, 16 * 97 + 3, 16 * 900]]], np.int32)
    host, cache, len_d = make_cache(lens, 16, 1, 5)
    gen = torch.Generator().manual_seed(3)
    q = scaled(torch.randn(3, g, 128, generator=gen).bfloat16(), q_exponent)
    bounds = scaled(torch.randn(host["k"].shape[0], 2, 128, generator=gen).sort(1).values.bfloat16(), exponent)
    ws = B.alloc_paged_select_workspace(cache, 16 * 900)
    for pages in (3, 20, 64):
        table, short = torch.empty(1, 1, 3, pages, dtype=torch.int32, device="cuda"), torch.empty(1, 1, 3, dtype=torch.int32, device="cuda")
        B.paged_select(cache, 0, g, q.cuda(), len_d, bounds.cuda(), table, short, ws, 16 * 900)
        want, want_len, _ = ro.select(host, 0, g, H.bits(q), lens, H.bits(bounds), pages, 1, 1, None, 16 * 900)
        np.testing.assert_array_equal(table[0].cpu().numpy(), want)
        np.testing.assert_array_equal(short[0].cpu().numpy(), want_len)


@pytest.mark.parametrize("nothing", ["queries", "bounds", "both"])
def test_scores_of_nothing_are_equal(nothing):
    """Zeros of either sign: the first pages, and the last."""
    from paper_2507_08143_b200 import binding as B
    lens = np.array([[[16 * 900]]], np.int32)
    host, cache, len_d = make_cache(lens, 16, 1, 6)
    gen = torch.Generator().manual_seed(4)
    q, bounds = torch.randn(1, 5, 128, generator=gen).bfloat16(), torch.randn(host["k"].shape[0], 2, 128, generator=gen).sort(1).values.bfloat16()
    q, bounds = q * (nothing == "bounds"), bounds * (nothing == "queries")
    table, short = torch.empty(1, 1, 1, 40, dtype=torch.int32, device="cuda"), torch.empty(1, 1, 1, dtype=torch.int32, device="cuda")
    B.paged_select(cache, 0, 5, q.cuda(), len_d, bounds.cuda(), table, short, B.alloc_paged_select_workspace(cache, 16 * 900), 16 * 900, last_pages=3)
    np.testing.assert_array_equal(table.view(-1).cpu().numpy(), host["table"][0, 0, 0][np.r_[0:37, 897:900]])
