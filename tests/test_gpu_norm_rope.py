"""Norms of queries and keys with the rotation on the GPU against the fp64 statement in oracle/rows_oracle.py."""
import numpy as np
import pytest
import torch

from oracle import rows_oracle as ro

pytestmark = pytest.mark.gpu


def check(got, x, w, eps, pos, freq, interleaved, rotated=True):
    """Per channel: the row's sum of squares 12 roundings of 2^-24, halved by the root, the root and its reciprocal 2^-22, two products; a sine
    or cosine 2^-22 (2 ulp and the rounding of its fraction of a turn, 2 pi 2^-25), a product and a sum; the result rounded to bf16, 2^-8."""
    y, plain, size = ro.norm_rope(x.double().cpu().numpy(), None if w is None else w.double().cpu().numpy(), eps, pos.cpu().numpy(),
                                  freq.cpu().numpy(), interleaved)
    want, scale = (y, size) if rotated else (plain, np.abs(plain))
    rel = 6 * 2.0 ** -24 + 2.0 ** -22 + 3 * 2.0 ** -24 + 2 * 2.0 ** -22 + 2 * 2.0 ** -24
    err = np.abs(got.double().cpu().numpy() - want)
    tol = 1.01 * rel * scale + 2.0 ** -8 * np.abs(want) + 1e-38
    assert np.all(err <= tol), f"{np.nanmax(err / tol):.2f} of the bound"


def run(tokens, qh, kh, rotary=128, interleaved=False, weights="qk", plain=True, strided=False, far=False, seed=0, scale=1.0):
    from paper_2507_08143_b200 import binding as B
    g = torch.Generator(device="cuda").manual_seed(seed)
    pad = 16 if strided else 0
    qkv = (scale * torch.randn(tokens, qh + kh + 2, 128 + pad, generator=g, device="cuda")).bfloat16()
    q, k = qkv[:, :qh, :128], qkv[:, qh:qh + kh, :128]
    pos = torch.randint(-2 ** 31 if far else 0, 2 ** 31 - 1 if far else 131072, (tokens,), generator=g, device="cuda").to(torch.int32)
    freq = (500000.0 ** (-torch.arange(0, rotary, 2, device="cuda", dtype=torch.float64) / max(rotary, 1))).float()
    w = lambda on: (1 + 0.3 * torch.randn(128, generator=g, device="cuda")).bfloat16() if on else None
    qw, kw = w("q" in weights), w("k" in weights)

    def rows(n):
        if not strided:
            return None, torch.full((tokens, n, 128), 7.0, dtype=torch.bfloat16, device="cuda")
        whole = torch.full((n, tokens, 144), 7.0, dtype=torch.bfloat16, device="cuda")       # heads outside tokens, rows with a gap
        return whole, whole[..., 8:136].transpose(0, 1)
    (qb, qo), (kb, ko), (pb, kp) = rows(qh), rows(kh), rows(kh)
    B.norm_rope(q if qh else None, k if kh else None, pos if rotary else None, freq if rotary else None, qo if qh else None, ko if kh else None,
                k_plain_out=kp if plain and kh else None, q_weight=qw, k_weight=kw, eps=1e-5, interleaved=interleaved)
    if qh:
        check(qo, q, qw, 1e-5, pos, freq, interleaved)
    if kh:
        check(ko, k, kw, 1e-5, pos, freq, interleaved)
        if plain:
            check(kp, k, kw, 1e-5, pos, freq, interleaved, rotated=False)
        else:
            assert torch.all(kp == 7.0)
    for whole in (qb, kb, pb):
        if whole is not None:
            assert torch.all(whole[..., :8] == 7.0) and torch.all(whole[..., 136:] == 7.0)


@pytest.mark.parametrize("tokens", [1, 2, 7, 64, 333, 2500])
@pytest.mark.parametrize("qh, kh", [(1, 1), (4, 2), (32, 8), (28, 4), (0, 3), (5, 0)])
def test_tokens_and_heads(tokens, qh, kh):
    run(tokens, qh, kh, strided=tokens % 2 == 1, seed=tokens + qh)


@pytest.mark.parametrize("rotary", [0, 16, 32, 48, 64, 96, 112, 128])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("weights", ["qk", "q", ""])
def test_rotations_and_norms(rotary, interleaved, weights):
    run(19, 6, 2, rotary=rotary, interleaved=interleaved, weights=weights, strided=True, seed=rotary)


def test_many_heads_and_far_positions():
    run(3, 300, 70, seed=1)
    run(700, 2, 1, seed=2, plain=False)
    from paper_2507_08143_b200 import binding as B
    # angles of up to 2^31: a turn's fraction is good to 2^31 / (2 pi) * 2^-52 turns in 64 bits on either side
    run(200, 3, 2, far=True, seed=3)
    x = torch.randn(1, 1, 128, device="cuda").bfloat16()
    out = torch.empty_like(x)
    for n in (131071, 1048576):                                           # frequency 1: the angle is the position
        pos = torch.full((1,), n, dtype=torch.int32, device="cuda")
        B.norm_rope(x, None, pos, torch.ones(64, device="cuda"), out, None)
        check(out, x, None, 0.0, pos, torch.ones(64), False)


@pytest.mark.parametrize("scale", [1e-18, 1e-4, 1e18])
def test_sizes_of_values(scale):
    """At 1e-18 the mean square is far below eps, at 1e18 its sum is near the end of fp32's range."""
    run(9, 3, 2, scale=scale, seed=4)


def test_in_place_and_rows_that_are_no_numbers():
    from paper_2507_08143_b200 import binding as B
    q, k = torch.randn(50, 6, 128, device="cuda").bfloat16(), torch.randn(50, 2, 128, device="cuda").bfloat16()
    q[3, 1, 5] = float("nan"); k[4, 0, 2] = float("inf")
    pos, freq = torch.arange(50, dtype=torch.int32, device="cuda"), torch.rand(32, device="cuda")
    w = torch.rand(128, device="cuda").bfloat16()
    for weight in (w, None):
        q1, k1 = torch.empty_like(q), torch.empty_like(k)
        B.norm_rope(q, k, pos, freq, q1, k1, q_weight=weight, k_weight=weight)
        q2, k2 = q.clone(), k.clone()
        B.norm_rope(q2, k2, pos, freq, q2, k2, q_weight=weight, k_weight=weight)
        for a, b, bad in ((q1, q2, (3, 1)), (k1, k2, (4, 0))):
            assert torch.equal(a.view(torch.int16), b.view(torch.int16))
            rows = torch.isfinite(a).all(-1)
            assert not rows[bad] and rows.sum() == rows.numel() - 1
    B.norm_rope(q[:0], k[:0], pos[:0], freq, q1[:0], k1[:0])               # no tokens


def test_graph_and_streams():
    from paper_2507_08143_b200 import binding as B
    q, k = torch.randn(5, 8, 128, device="cuda").bfloat16(), torch.randn(5, 2, 128, device="cuda").bfloat16()
    pos, freq = torch.arange(5, dtype=torch.int32, device="cuda"), torch.rand(64, device="cuda")
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.norm_rope(q, k, pos, freq, qo, ko)
        pos += 1
    for step in range(3):
        q.normal_()
        graph.replay()
        at = torch.arange(5, dtype=torch.int32, device="cuda") + step
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        q1, k1 = torch.empty_like(q), torch.empty_like(k)
        with torch.cuda.stream(side):
            B.norm_rope(q, k, at, freq, q1, k1)
        torch.cuda.synchronize()
        assert torch.equal(qo, q1) and torch.equal(ko, k1)
