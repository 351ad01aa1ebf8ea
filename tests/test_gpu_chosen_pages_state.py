"""What attention over chosen pages leaves behind, step by step: rows, positions and weights in the whole cache's pages, bounds kept up by the choice
against bounds made anew, and the eviction that goes by all of them."""
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


@pytest.mark.parametrize("page", [8, 16])
@pytest.mark.parametrize("four", [False, True])
def test_steps_over_chosen_pages_and_an_eviction(four, page):
    from paper_2507_08143_b200 import binding as B
    lens = np.array([[[500, 0, 77, 700], [20, 333, -1, 64]]], np.int32)
    g, pages, steps, heads, batch = 3, 6, page + 3, 2, 4
    host, cache, len_d = (make_cache4 if four else make_cache)(lens, page, steps, 17)
    k, v, _, mass, pos = cache.tensors
    bits = (lambda t: t.cpu().numpy()) if four else H.bits
    room = int(lens.max()) + steps
    bounds = torch.full((cache.n_pages, 2, 128), 5.0, dtype=torch.bfloat16, device="cuda")
    B.paged_bounds(cache, len_d, bounds, room)
    hb = H.bits(bounds)
    table, short = torch.empty(1, heads, batch, pages, dtype=torch.int32, device="cuda"), torch.empty(1, heads, batch, dtype=torch.int32, device="cuda")
    few = type(cache)(k, v, table, mass=mass, positions=pos)
    opt = B.decode_options(g, pages * page, accumulate=True)
    ws, ws_select = B.alloc_paged_attention_workspace(few, opt), B.alloc_paged_select_workspace(cache, room)
    out, lse = torch.empty(batch, heads * g, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(batch, heads * g, device="cuda")
    gen = torch.Generator().manual_seed(2)
    n, next_position = lens.copy(), np.maximum(2 * lens.max((0, 1)), 0).astype(np.int32)
    mass_tol, largest_step = np.zeros(host["mass"].shape), 0.0
    host = dict(host, mass=host["mass"].astype(np.float64))
    for _ in range(steps):
        q, kn, vn = (torch.randn(batch, m, 128, generator=gen).bfloat16() for m in (heads * g, heads, heads))
        qd, kd, vd = q.cuda(), kn.cuda(), vn.cuda()
        B.paged_select(cache, 0, g, qd, len_d, bounds, table, short, ws_select, room, k_new=kd)
        B.paged_attention(few, 0, opt, qd, short, out, ws, k_new=kd, v_new=vd, new_positions=torch.from_numpy(next_position).cuda(), lse_out=lse)
        want, want_len, hb = ro.select(host, 0, g, H.bits(q), n, hb, pages, 1, 1, H.bits(kn), room)
        np.testing.assert_array_equal(table[0].cpu().numpy(), want)
        np.testing.assert_array_equal(bf16_bits_to_f64(H.bits(bounds)), bf16_bits_to_f64(hb))
        ref, _, after, info = (ro.attention4 if four else po.attention)(dict(host, table=want[None]), 0, H.bits(q), want_len[None], np.float64(np.float32(128 ** -0.5)),
                                                                        k_new=H.bits(kn), v_new=H.bits(vn), new_positions=next_position, accumulate=True)
        for (h, b), (at, p, pv, mag) in info.items():
            r = slice(h * g, (h + 1) * g)
            _, rel, tol = attention4_bounds(g, pv, ref[b, r], mag, 0.0, len(at)) if four else attention_bounds(g, p, pv, ref[b, r], mag, 128 ** -0.5, 0.0, len(at))
            assert np.all(np.abs(out[b, r].double().cpu().numpy() - ref[b, r]) <= tol)
            for j, a in enumerate(at):                       # (as in the attention's own tests, one step upon the other; the new token's begins here)
                mass_tol[a] = (0.0 if j == len(at) - 1 else mass_tol[a]) + (1.01 * rel + (g + 2) * 2.0 ** -24) * p[:, j].sum() + 2.0 ** -24 * abs(after["mass"][a])
            if four:
                row = ro.hold4(H.bits(kn)[b, h])
                largest_step = max(largest_step, bf16_bits_to_f64(np.ascontiguousarray(row[64:]).view(np.uint16))[0::2].max())
        host = dict(after, table=host["table"])
        for name, t in (("k", k), ("v", v)):
            np.testing.assert_array_equal(bits(t), host[name], err_msg=name)
        np.testing.assert_array_equal(pos.cpu().numpy(), host["positions"])
        got, live = mass.double().cpu().numpy(), ~np.isnan(host["mass"])
        assert np.array_equal(live, ~np.isnan(got)) and np.all(np.abs(got - host["mass"])[live] <= mass_tol[live])
        n = np.where(n >= 0, n + 1, n)
        len_d.copy_(torch.from_numpy(n))
        next_position += 1
    # ---- bounds made anew: of bf16 those that the steps kept up; in 4 bits of the rows as they are held, up to half a step off the keys (and 15 2^-24 of
    # one, the difference's rounding), and rounded to bf16 by 2^-9
    units = list(np.ndindex(lens.shape))
    anew = ro.bounds(host, units, n, hb)
    x, y = bf16_bits_to_f64(hb), bf16_bits_to_f64(anew)
    if four:
        assert np.all(np.abs(x - y) <= largest_step * (0.5 + 15 * 2.0 ** -24) + 2.0 ** -8 * np.abs(y))
    else:
        np.testing.assert_array_equal(x, y)
    # ---- eviction by the weights and positions that the steps left, and the bounds of what stays
    budgets = np.where(n > 60, n // 2, n).astype(np.int32)
    host = dict(k=bits(k), v=bits(v), mass=mass.cpu().numpy(), positions=pos.cpu().numpy(), table=host["table"])
    B.paged_evict(cache, len_d, torch.from_numpy(budgets).cuda(), len_d, room, recent=12, next_position=torch.from_numpy(next_position).cuda())
    host, n = po.evict(host, units, n, budgets, recent=12, next_position=next_position)
    for name, t in (("k", k), ("v", v)):
        np.testing.assert_array_equal(bits(t), host[name], err_msg=name)
    np.testing.assert_array_equal(pos.cpu().numpy(), host["positions"])
    np.testing.assert_array_equal(mass.cpu().numpy().view(np.uint32), host["mass"].view(np.uint32))
    np.testing.assert_array_equal(len_d.cpu().numpy(), n)
    B.paged_bounds(cache, len_d, bounds, room)
    np.testing.assert_array_equal(bf16_bits_to_f64(H.bits(bounds)), bf16_bits_to_f64(ro.bounds(host, units, n, hb)))
