"""Plain fp64 statements of the operators around the paged cache: rows in 4 bits and the attention over them, key bounds of pages
and the choice of pages by them, norms with rotation.  Written from their definitions; caches as in paged_oracle, with rows of 80
uint8 in the place of 128 bf16 where they are held in 4 bits."""
from __future__ import annotations

import math

import numpy as np

from . import paged_oracle as po
from .compactor_oracle import bf16_bits_to_f64


def f64_to_bf16_bits(x: np.ndarray) -> np.ndarray:
    """Nearest bf16 (ties to even) of float64 values, as bits."""
    x = np.asarray(x, np.float64)
    with np.errstate(over="ignore"):
        y = x.astype(np.float32)
    # rounding to odd at 24 bits first, so that the second rounding sees which side of a tie it is on
    u = y.view(np.uint32).copy()
    off = np.isfinite(y) & (y.astype(np.float64) != x)
    toward = np.where(np.abs(y.astype(np.float64)) > np.abs(x), u - 1, u)       # cut off
    u = np.where(off, toward | 1, u)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)
    return np.where(np.isnan(x), np.uint16(0x7FFF), r)


def hold4(bits: np.ndarray) -> np.ndarray:
    """Rows of 128 bf16 as 80 bytes: codes, then step and least value of each group of 32.  Differences to the least value are taken in fp32."""
    x = bf16_bits_to_f64(bits).reshape(bits.shape[:-1] + (4, 32))
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        lo, hi = x.min(-1, keepdims=True) + 0.0, x.max(-1, keepdims=True)          # (-0 is 0)
        minus = lambda a, b: (a.astype(np.float32) - b.astype(np.float32)).astype(np.float64)
        m, e = np.frexp(minus(hi, lo) / 15)
        step = np.ldexp(np.ceil(m * 16) / 16, e)
        step = np.where(step < 2.0 ** -120, 0.0, step)
        bad = ~(np.isfinite(x).all(-1, keepdims=True) & (step <= 2.0 ** 120))
        code = np.where(step > 0, np.ceil(minus(x, lo) / np.where(step > 0, step, 1.0) - 0.5), 0.0)
    code = np.where(bad, 0, code).astype(np.uint8).reshape(bits.shape[:-1] + (64, 2))
    params = np.concatenate([f64_to_bf16_bits(np.where(bad, np.nan, step)), f64_to_bf16_bits(np.where(bad, np.nan, lo))], -1)
    params = np.ascontiguousarray(params.reshape(bits.shape[:-1] + (8,))).view(np.uint8)
    return np.concatenate([code[..., 0] | (code[..., 1] << 4), params], -1)


def values4(rows: np.ndarray, parts: bool = False):
    """What rows of 80 bytes stand for; with `parts` (s c, lo) per channel."""
    codes, params = rows[..., :64], np.ascontiguousarray(rows[..., 64:]).view(np.uint16)
    c = np.stack([codes & 15, codes >> 4], -1).reshape(rows.shape[:-1] + (4, 32)).astype(np.float64)
    p = bf16_bits_to_f64(params).reshape(rows.shape[:-1] + (4, 2))
    sc = (p[..., :1] * c).reshape(rows.shape[:-1] + (128,))
    lo = np.repeat(p[..., 1], 32, axis=-1)
    return (sc, lo) if parts else sc + lo


def attention4(c: dict, layer, q, lengths, scale, softcap=0.0, k_new=None, v_new=None, new_positions=None, accumulate=False,
               max_length=None):
    """As paged_oracle.attention, over rows in 4 bits.  info[h, b] = (slots, p, sum p (|s c| + |lo|), largest scale sum |q| (|s c| + |lo|))."""
    c = po.copy_cache(c)
    c["mass"] = c["mass"].astype(np.float64)
    _, heads, batch = c["table"].shape[:3]
    g = q.shape[1] // heads
    out, lse, info = np.zeros(q.shape), np.full(q.shape[:2], -np.inf), {}
    limit = po.capacity(c) if max_length is None else min(max_length, po.capacity(c))
    for h in range(heads):
        for b in range(batch):
            unit = (layer, h, b)
            n = int(lengths[unit])
            if n < 0 or n + (k_new is not None) > limit:
                continue
            at = [a for a in (po.slot_of(c, unit, t) for t in range(n)) if a is not None]
            kr, vr = [c["k"][a] for a in at], [c["v"][a] for a in at]
            if k_new is not None:
                a = po.slot_of(c, unit, n)
                at.append(a)
                kr.append(hold4(k_new[b, h])); vr.append(hold4(v_new[b, h]))
                if a is not None:
                    c["k"][a], c["v"][a], c["mass"][a] = kr[-1], vr[-1], 0.0
                    c["positions"][a] = n if new_positions is None else new_positions[b]
            if not at:
                continue
            (ks, kl), (vs, vl) = values4(np.array(kr), True), values4(np.array(vr), True)
            qq = bf16_bits_to_f64(q[b, h * g:(h + 1) * g])
            y = scale * (qq @ (ks + kl).T)
            mag = scale * (np.abs(qq) @ (np.abs(ks) + np.abs(kl)).T)
            if softcap > 0:
                y = softcap * np.tanh(y / softcap)
            top = y.max(1, keepdims=True)
            e = np.exp(y - top)
            z = e.sum(1, keepdims=True)
            p = e / z
            out[b, h * g:(h + 1) * g] = p @ (vs + vl)
            lse[b, h * g:(h + 1) * g] = (top + np.log(z))[:, 0]
            info[(h, b)] = (at, p, p @ (np.abs(vs) + np.abs(vl)), mag.max())
            if accumulate:
                for j, a in enumerate(at):
                    if a is not None:
                        c["mass"][a] += p[:, j].sum()
    return out, lse, c, info


def bounds(c: dict, units, lengths, before: np.ndarray, first=None, max_length=None) -> np.ndarray:
    """Bounds [n_pages][2][128] (bits) after the pages of the given units are brought up to date."""
    after, page = before.copy(), c["k"].shape[1]
    limit = po.capacity(c) if max_length is None else min(max_length, po.capacity(c))
    for unit in units:
        n, f = int(lengths[unit]), 0 if first is None else max(0, int(first[unit]))
        if n > limit:
            continue
        for t in range(f // page * page, max(n, 0), page):
            a = po.slot_of(c, unit, t)
            if a is None:
                continue
            rows = c["k"][a[0], : min(page, n - t)]
            x = values4(rows) if rows.shape[-1] == 80 else bf16_bits_to_f64(rows)
            after[a[0], 0], after[a[0], 1] = f64_to_bf16_bits(x.min(0)), f64_to_bf16_bits(x.max(0))
    return after


def select(c: dict, layer, g, q, lengths, bnds: np.ndarray, pages, first_pages, last_pages, k_new=None, max_length=None):
    """Returns (table [heads][batch][pages], lengths [heads][batch], bounds after)."""
    _, heads, batch = c["table"].shape[:3]
    page, n_pages = c["k"].shape[1], c["k"].shape[0]
    table, out, after = np.full((heads, batch, pages), -1, np.int32), np.zeros((heads, batch), np.int32), bnds.copy()
    limit = po.capacity(c) if max_length is None else min(max_length, po.capacity(c))
    for h in range(heads):
        for b in range(batch):
            unit = (layer, h, b)
            n = int(lengths[unit])
            t = n + (k_new is not None)
            if n < 0 or t > limit:
                out[h, b] = n if n < 0 else -1
                continue
            if k_new is not None:
                a = po.slot_of(c, unit, n)
                if a is not None:
                    x = bf16_bits_to_f64(k_new[b, h])
                    old = bf16_bits_to_f64(after[a[0]])
                    after[a[0], 0] = f64_to_bf16_bits(np.minimum(old[0], x) if a[1] > 0 else x)
                    after[a[0], 1] = f64_to_bf16_bits(np.maximum(old[1], x) if a[1] > 0 else x)
            count = -(-t // page)
            qq = bf16_bits_to_f64(q[b, h * g:(h + 1) * g])

            def rank(i):
                p = int(c["table"][unit][i])
                if i < first_pages or i >= count - last_pages:
                    return (0, 0.0, i)
                if not 0 <= p < n_pages:
                    return (3, 0.0, i)
                lo, hi = bf16_bits_to_f64(bnds[p])
                terms = qq * np.where(qq > 0, hi, lo)
                if not np.isfinite(terms).all():
                    s = np.nan if np.isnan(terms.sum(1)).any() else terms.sum(1).max()
                else:
                    s = max(math.fsum(r) for r in terms)
                s = float(np.float32(s))
                return (1, 0.0, i) if math.isnan(s) else (2, -s, i)

            taken = sorted(sorted(range(count), key=rank)[:pages])
            table[h, b, : len(taken)] = c["table"][unit][taken]
            out[h, b] = n - (count - len(taken)) * page
    return table, out, after


def norm_rope(x: np.ndarray, weight, eps, positions, inv_freq: np.ndarray, interleaved):
    """x [tokens][heads][128] float64.  Returns (rotated, before the rotation, |a| + |b| of each channel's pair)."""
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * weight
    r = 2 * len(inv_freq)
    i = np.arange(r // 2)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + r // 2)
    angle = (positions.astype(np.float64)[:, None] * inv_freq.astype(np.float64))[:, None, :]
    y, size = x.copy(), np.abs(x)
    y[..., a] = x[..., a] * np.cos(angle) - x[..., b] * np.sin(angle)
    y[..., b] = x[..., b] * np.cos(angle) + x[..., a] * np.sin(angle)
    size[..., a] = size[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    return y, x, size
