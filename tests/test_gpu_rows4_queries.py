"""Attention over rows in 4 bits with queries of a wide range: heads that are too large."""
import numpy as np
import pytest
import torch

from oracle import rows_oracle as ro
from oracle.compactor_oracle import bf16_bits_to_f64

pytestmark = pytest.mark.gpu


def attend(k, v, q, scale):
    """One unit of all rows of k, v (values of bf16 [n, 128], float64); q [g, 128].  Returns out, lse and the values that k and v are held as."""
    from paper_2507_08143_b200 import binding as B
    n, g = k.shape[0], q.shape[0]
    bits = [ro.f64_to_bf16_bits(x) for x in (k, v)]
    rows = [torch.from_numpy(ro.hold4(b)).cuda() for b in bits]
    pools = [torch.full((-(-n // 16), 16, 80), 255, dtype=torch.uint8, device="cuda") for _ in rows]
    for p, r in zip(pools, rows):
        p.view(-1, 80)[:n] = r
    table = torch.arange(pools[0].shape[0], dtype=torch.int32, device="cuda").view(1, 1, 1, -1)
    cache = B.PagedCache4(*pools, table)
    opt = B.decode_options(g, n, scale=scale)
    qd = torch.from_numpy(q).bfloat16().cuda().view(1, g, 128)
    assert np.array_equal(qd[0].double().cpu().numpy(), q)
    out, lse = torch.empty_like(qd), torch.empty(1, g, device="cuda")
    B.paged_attention(cache, 0, opt, qd, torch.full((1, 1, 1), n, dtype=torch.int32, device="cuda"), out, B.alloc_paged_attention_workspace(cache, opt), lse_out=lse)
    return out[0].double().cpu().numpy(), lse[0].double().cpu().numpy(), [ro.values4(ro.hold4(b), True) for b in bits]


def bf16(x):
    return bf16_bits_to_f64(ro.f64_to_bf16_bits(np.asarray(x, np.float64)))


@pytest.mark.parametrize("g", [4, 12])
def test_heads_of_2_to_the_118_and_more_give_not_a_number(g):
    """And only they: the head below is exact, also where it reaches the limit.  Whatever the sign of their scores."""
    rng = np.random.default_rng(4)
    n = 50
    k, v = bf16((rng.random((n, 128)) + 0.5) * 2.0 ** -114), bf16(rng.standard_normal((n, 128)))
    k[:, 1:32] = k[:, :1]                                    # (a group of two values, so that channel 0 has codes above 0 in all rows)
    k[:, 31] = 0.0
    q = np.zeros((g, 128))
    q[:, 64:] = bf16(rng.standard_normal((g, 64)))
    q[0, 0] = -2.0 ** 118
    q[1, 0] = 2.0 ** 118
    q[2, 0] = (2 - 2.0 ** -7) * 2.0 ** 117
    q[3, 0] = -(2 - 2.0 ** -7) * 2.0 ** 127
    out, lse, ((ks, kl), (vs, vl)) = attend(k, v, q, 1.0)
    assert np.all(ks[:, 0] > 0)
    for j in (0, 1, 3):
        assert np.isnan(out[j]).all() and np.isnan(lse[j]), j
    fine = [j for j in range(g) if j not in (0, 1, 3)]
    y = q[fine] @ (ks + kl).T
    mag = (np.abs(q[fine]) @ (np.abs(ks) + np.abs(kl)).T).max()
    dy = 161 * 2.0 ** -23 * mag
    want = np.log(np.exp(y).sum(1))
    rel = 2 * dy + 2 * 2.0 ** -22 + (n / 8 + 64) * 2.0 ** -24
    assert np.all(np.abs(lse[fine] - want) <= dy + rel + 2.0 ** -22 * np.abs(want))
    p = np.exp(y - want[:, None])
    tol = (np.expm1(rel) + 2.0 ** -16 + (n / 16 + 17) * 17 * 2.0 ** -23) * 1.01 * (p @ (np.abs(vs) + np.abs(vl))) + 2.0 ** -8 * np.abs(p @ (vs + vl))
    assert np.all(np.abs(out[fine] - p @ (vs + vl)) <= tol)
