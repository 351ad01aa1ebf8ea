"""Plain fp64 statements of the paged-cache operators, unit by unit and slot by slot, written from their definitions.

A cache here is a dict of numpy arrays: k, v [n_pages][page][d] (uint16 bit patterns), mass [n_pages][page] float32, positions
[n_pages][page] int32, table [layers][heads][batch][max_pages] int32.  The functions return new arrays and leave their
arguments alone."""
from __future__ import annotations

import numpy as np

from .compactor_oracle import bf16_bits_to_f64


def copy_cache(c: dict) -> dict:
    return {k: v.copy() for k, v in c.items()}


def slot_of(c: dict, unit, t: int):
    """(page, slot) of token t of a unit (layer, head, sequence); None where the table holds no page of the pool."""
    page_tokens = c["k"].shape[1]
    p = int(c["table"][unit][t // page_tokens])
    return (p, t % page_tokens) if 0 <= p < c["k"].shape[0] else None


def capacity(c: dict) -> int:
    return c["table"].shape[-1] * c["k"].shape[1]


def fill(c: dict, first_layer, k, v, cu, rows, mass_in=None, first_position=None, lengths=None):
    """rows(l, h, b) -> indices of the kept rows of that unit.  k, v: [layers][heads][tokens][d] bits.  Returns (cache, lengths)."""
    c = copy_cache(c)
    _, heads, batch = c["table"].shape[:3]
    out = np.zeros(c["table"].shape[:3], dtype=np.int32) if lengths is None else lengths.copy()
    start = out.copy()
    for l in range(k.shape[0]):
        for h in range(heads):
            for b in range(batch):
                unit = (first_layer + l, h, b)
                idx = np.asarray(rows(l, h, b), dtype=np.int64)
                n0 = int(start[unit])
                if n0 < 0 or n0 + len(idx) > capacity(c):
                    continue
                for j, i in enumerate(idx):
                    at = slot_of(c, unit, n0 + j)
                    if at is None or not 0 <= i < cu[b + 1] - cu[b]:
                        continue
                    c["k"][at], c["v"][at] = k[l, h, cu[b] + i], v[l, h, cu[b] + i]
                    c["mass"][at] = 0.0 if mass_in is None else mass_in[l, h, cu[b] + i]
                    c["positions"][at] = (0 if first_position is None else first_position[b]) + i
                out[unit] = n0 + len(idx)
    return c, out


def attention(c: dict, layer, q, lengths, scale, softcap=0.0, k_new=None, v_new=None, new_positions=None, accumulate=False,
              max_length=None):
    """q [batch][heads*g][d] bits, k_new / v_new [batch][heads][d] bits.  Returns (out, lse, cache, weights) with out and lse in
    fp64, the cache after the call (its mass as float64) and weights[h][b] = (slots' tokens, p [g][tokens], sum |v| p, A)."""
    c = copy_cache(c)
    c["mass"] = c["mass"].astype(np.float64)
    _, heads, batch = c["table"].shape[:3]
    g = q.shape[1] // heads
    d = q.shape[2]
    out = np.zeros((batch, heads * g, d))
    lse = np.full((batch, heads * g), -np.inf)
    info = {}
    limit = capacity(c) if max_length is None else min(max_length, capacity(c))
    for h in range(heads):
        for b in range(batch):
            unit = (layer, h, b)
            n = int(lengths[unit])
            if n < 0 or n + (k_new is not None) > limit:
                continue
            toks = [t for t in range(n) if slot_of(c, unit, t) is not None]
            at = [slot_of(c, unit, t) for t in toks]
            kk = [bf16_bits_to_f64(c["k"][a]) for a in at]
            vv = [bf16_bits_to_f64(c["v"][a]) for a in at]
            if k_new is not None:
                a = slot_of(c, unit, n)
                toks.append(n); at.append(a)
                kk.append(bf16_bits_to_f64(k_new[b, h])); vv.append(bf16_bits_to_f64(v_new[b, h]))
                if a is not None:
                    c["k"][a], c["v"][a] = k_new[b, h], v_new[b, h]
                    c["positions"][a] = n if new_positions is None else new_positions[b]
                    c["mass"][a] = 0.0
            if not toks:
                continue
            kk, vv = np.array(kk), np.array(vv)
            qq = bf16_bits_to_f64(q[b, h * g:(h + 1) * g])
            y = scale * (qq @ kk.T)
            mag = scale * (np.abs(qq) @ np.abs(kk).T)
            if softcap > 0:
                y = softcap * np.tanh(y / softcap)
            top = y.max(axis=1, keepdims=True)
            e = np.exp(y - top)
            z = e.sum(axis=1, keepdims=True)
            p = e / z
            out[b, h * g:(h + 1) * g] = p @ vv
            lse[b, h * g:(h + 1) * g] = (top + np.log(z))[:, 0]
            info[(h, b)] = (at, p, p @ np.abs(vv), mag.max())
            if accumulate:
                for j, a in enumerate(at):
                    if a is not None:
                        c["mass"][a] += p[:, j].sum()
    return out, lse, c, info


def evict(c: dict, units, lengths, budgets, recent=0, next_position=None, max_length=None):
    """Returns (cache, lengths) after the eviction of the given units."""
    c = copy_cache(c)
    out = lengths.copy()
    limit = capacity(c) if max_length is None else min(max_length, capacity(c))
    for unit in units:
        n, budget = int(lengths[unit]), int(budgets[unit])
        if n < 0 or budget < 0 or n <= budget or n > limit:
            continue
        at = [slot_of(c, unit, t) for t in range(n)]
        if budget > 0 and any(a is None for a in at):
            continue
        out[unit] = budget
        if budget == 0:
            continue

        def rank(t):
            w = c["mass"][at[t]]
            if recent > 0 and c["positions"][at[t]] >= next_position[unit[2]] - min(recent, budget):
                return (0, 0.0, t)
            if np.isnan(w):
                return (1, 0.0, t)
            return (2, -float(w), t)

        kept = set(sorted(range(n), key=rank)[:budget])
        holes = [t for t in range(budget) if t not in kept]
        movers = [t for t in range(budget, n) if t in kept]
        assert len(holes) == len(movers)
        for to, frm in zip(holes, movers):
            for name in ("k", "v", "mass", "positions"):
                c[name][at[to]] = c[name][at[frm]]
    return c, out
