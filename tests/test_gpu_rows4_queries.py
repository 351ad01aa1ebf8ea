"""Attention over rows in 4 bits with queries of a wide range: how many bits of a channel far below its head's greatest count, and heads that are too large."""
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


@pytest.mark.parametrize("g", [3, 11])
@pytest.mark.parametrize("channel, exponent, exact", [(40, -31, True), (41, -27, True), (40, -35, False), (41, -31, False), (41, -28, False)])
def test_channels_far_below_the_greatest(g, channel, exponent, exact):
    """One channel of the queries lies 2^exponent below the greatest, 1, with keys that make up for it.  Queries enter as fp16 of 2^14 q, those of odd
    channels as 2^10 q, whose last place is never below 2^-24: a bf16 of eight bits fits from 2^-31 (odd: 2^-27) on, and is off by at most 2^-25 2^-14 =
    2^-39 (2^-35) below.  Everything else as in the other tests: 161 2^-23 of the largest sum for a score."""
    rng = np.random.default_rng(3)
    n = 60
    k, v = bf16(rng.standard_normal((n, 128))), bf16(rng.standard_normal((n, 128)))
    k[:, 32:64] = 0.0
    k[:, channel] = bf16(rng.standard_normal(n) * 2.0 ** -exponent)
    q = bf16(rng.uniform(-0.25, 0.25, (g, 128)))
    q[:, 32:64] = 0.0
    q[:, 0] = 1.0
    q[:, channel] = (2 - 2.0 ** -7 * (1 + 2 * np.arange(g))) * 2.0 ** exponent            # odd in the last of eight bits
    out, lse, ((ks, kl), (vs, vl)) = attend(k, v, q, 1.0)
    y = q @ (ks + kl).T
    mag = (np.abs(q) @ (np.abs(ks) + np.abs(kl)).T).max()
    dy = 161 * 2.0 ** -23 * mag
    if not exact:
        dy += (2.0 ** -39 * np.abs(ks[:, 0::2]).sum(1) + 2.0 ** -35 * np.abs(ks[:, 1::2]).sum(1)).max()
    top = y.max(1, keepdims=True)
    want = (top + np.log(np.exp(y - top).sum(1, keepdims=True)))[:, 0]
    rel = 2 * dy + 2 * 2.0 ** -22 + (n / 8 + 64) * 2.0 ** -24
    assert np.all(np.abs(lse - want) <= dy + rel + 2.0 ** -22 * np.abs(want))
    p = np.exp(y - want[:, None])
    tol = (np.expm1(rel) + 2.0 ** -16 + (n / 16 + 17) * 17 * 2.0 ** -23) * 1.01 * (p @ (np.abs(vs) + np.abs(vl))) + 2.0 ** -8 * np.abs(p @ (vs + vl))
    assert np.all(np.abs(out - p @ (vs + vl)) <= tol)


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


@pytest.mark.parametrize("softcap", [0.0, 2.0 ** -100])
@pytest.mark.parametrize("g", [2, 9])
def test_scores_of_small_queries_and_small_scales_are_small(g, softcap):
    """Queries at 2^-112 times keys at 2^123 times a scale of 2^-126: all scores are below 2^-100, and the output is the mean, whose two halves are opposite.
    What is left of a score may be off by 2^121 (the largest sum of a query 2^126 of its size) times the least fp32."""
    from paper_2507_08143_b200 import binding as B
    n = 64
    sign = np.where(np.arange(n) % 2 == 0, 1.0, -1.0)[:, None]
    rows = [torch.from_numpy(ro.hold4(ro.f64_to_bf16_bits(sign * x * np.ones(128)))).cuda() for x in (2.0 ** 123, 1.0)]
    pools = [r.view(4, 16, 80).contiguous() for r in rows]
    cache = B.PagedCache4(*pools, torch.arange(4, dtype=torch.int32, device="cuda").view(1, 1, 1, 4))
    q = torch.full((1, g, 128), 2.0 ** -112, device="cuda").bfloat16()
    opt = B.decode_options(g, n, scale=2.0 ** -126, softcap=softcap)
    out, lse = torch.empty_like(q), torch.empty(1, g, device="cuda")
    B.paged_attention(cache, 0, opt, q, torch.full((1, 1, 1), n, dtype=torch.int32, device="cuda"), out, B.alloc_paged_attention_workspace(cache, opt), lse_out=lse)
    assert torch.all(out.double().abs() <= 2 * 2.0 ** (121 - 149) + (n / 8 + 64) * 2.0 ** -24)
    assert torch.all((lse.double() - np.log(n)).abs() <= 2.0 ** -22 * np.log(n) + (n / 8 + 64) * 2.0 ** -24)
