"""More operators as measured: cases, inputs, plain forms and exact values.

They stand before, in and beside the paged cache that a compressed prefill is decoded from:

  norm     norms of queries and keys per head and the rotation by position in one pass: what a prefill is scored by (keys
           without rotation), held as (keys with it) and asked with (queries), and a decoding step's rows
  store    a compressed prefill into pages that hold 4 bits per channel, and read back from there as dense rows
  four     attention of one new token per sequence over such pages; the token's own row is appended as it is held
  bounds   the least and the greatest key of every page, channel by channel
  sparse   pages chosen for the step's queries by those bounds, and the attention over the chosen ones alone

A row of 128 channels in 4 bits is 80 bytes: for each group of 32 channels the least value `lo` (bf16) and a step s = (greatest -
least) / 15, rounded up to four significant bits; a channel is the whole number c nearest to (x - lo) / s (the lower of two)
and stands for lo + s c.  All of these operators are bound by memory; `work` counts every byte that has to be touched once."""
import math
import random

import torch

own = False

D = 128                                      # head dimension of every configuration here
GROUP = 32                                   # channels that share a step and a least value
ROW4 = D // 2 + 4 * (D // GROUP)             # bytes of a row in 4 bits


# --------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one decoding step of one sequence far into its context, 32 query heads and 8 KV heads: latency
        dict(name="norm step", op="norm", tokens=1, heads=8, g=4, rotary=128, interleaved=False, weights=True, plain=False, prefill=False),
        # an 8192-token prefill of one layer; the keys come with and without their rotation
        dict(name="norm c1", op="norm", tokens=8192, heads=8, g=4, rotary=128, interleaved=False, weights=True, plain=True, prefill=True),
        # 28 + 4 heads, a ragged pack of odd length, half of the channels rotated in neighbouring pairs, no norm
        dict(name="norm c2", op="norm", tokens=19661, heads=4, g=7, rotary=64, interleaved=True, weights=False, plain=False, prefill=True),
        # the small configuration's prefill at half retention
        dict(name="store c0", op="store", layers=1, heads=2, batch=1, lo=1024, hi=1024, r=0.5, page=16),
        # 32 layers x 8 heads of an 8192-token prefill at r = 0.3
        dict(name="store c1", op="store", layers=32, heads=8, batch=1, lo=8192, hi=8192, r=0.3, page=16),
        # one sequence of the small configuration, where latency counts
        dict(name="four c0", op="four", heads=2, batch=1, g=4, lo=511, hi=511, page=16, accumulate=False, softcap=0.0),
        # the longest uncompressed context, one sequence: the work of a few heads split over the whole GPU
        dict(name="four c3", op="four", heads=8, batch=1, g=5, lo=131071, hi=131071, page=64, accumulate=False, softcap=0.0),
        # a padded ragged batch of up to 32768 tokens, some rows empty, weights accumulated for a later eviction
        dict(name="four c4", op="four", heads=8, batch=16, g=4, lo=-1, hi=32768, page=16, accumulate=True, softcap=0.0),
        # all layers of a compressed 8192-token prefill
        dict(name="bounds c1", op="bounds", layers=32, heads=8, batch=1, lo=2457, hi=2457, page=16, bits=16),
        # two layers of a ragged batch held in 4 bits
        dict(name="bounds c4", op="bounds", layers=2, heads=8, batch=16, lo=409, hi=32768, page=64, bits=4),
        # 4096 of 131072 tokens asked for, one sequence
        dict(name="sparse c3", op="sparse", heads=8, batch=1, g=5, lo=131071, hi=131071, page=64, bits=16, blocks=64, accumulate=False),
        # at most 2048 tokens of each context of a ragged batch held in 4 bits
        dict(name="sparse c4", op="sparse", heads=8, batch=16, g=4, lo=409, hi=32768, page=32, bits=4, blocks=64, accumulate=True),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = 8 * 131072                        # tokens of a drawn case over all its heads: what the longest listed context has
    heads = rng.choice((1, 2, 4, 8))
    page = rng.choice((8, 16, 32, 64, 128))
    g = rng.choice((1, 2, 3, 4, 5, 6, 7, 8, 12, 16))
    op = rng.choice(("norm", "store", "four", "four", "bounds", "sparse"))
    if op == "norm":
        tokens = _log_uniform(rng, 1, 32768 * 8 // (heads * (1 + g) if heads * g > 8 else 16))
        return dict(op=op, tokens=tokens, heads=heads, g=g, rotary=rng.choice((128, 128, 64, 32, 96)), interleaved=rng.random() < 0.3,
                    weights=rng.random() < 0.7, plain=rng.random() < 0.5, prefill=tokens > 64 or rng.random() < 0.3)
    if op in ("four", "sparse"):
        batch = _log_uniform(rng, 1, 64)
        hi = _log_uniform(rng, 1, min(131071, most // (heads * batch)))
        lo = rng.choice((hi, max(0, hi // 16), -1))
        case = dict(op=op, heads=heads, batch=batch, g=g, lo=lo, hi=hi, page=page, accumulate=rng.random() < 0.6)
        if op == "four":
            return dict(case, softcap=rng.choice((0.0, 0.0, 30.0, 50.0)))
        return dict(case, bits=rng.choice((4, 16)), blocks=_log_uniform(rng, 2, max(2, hi // page)))
    layers = _log_uniform(rng, 1, 32)
    batch = _log_uniform(rng, 1, 16)
    hi = _log_uniform(rng, 16, min(131072, most // (layers * heads * batch)))
    lo = rng.choice((hi, max(1, hi // 16)))
    if op == "store":
        return dict(op=op, layers=layers, heads=heads, batch=batch, lo=lo, hi=hi, r=rng.choice((0.2, 0.3, 0.32, 0.5)), page=page)
    return dict(op=op, layers=layers, heads=heads, batch=batch, lo=lo, hi=hi, page=page, bits=rng.choice((4, 16)))


def _lengths(case):
    """One length per sequence between lo and hi, spread over the logarithm, the first of them hi; with lo = -1 a tenth of the
    sequences is empty and a tenth of the rows holds no sequence (-1).  The shapes are the case's, the values the seed's."""
    lo, hi = case["lo"], case["hi"]
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    lens = [hi]
    for _ in range(case["batch"] - 1):
        u, x = rng.random(), rng.uniform(math.log(max(1, lo)), math.log(max(1, hi)))
        lens.append((-1 if u < 0.1 else 0) if lo < 0 and u < 0.2 else hi if lo == hi else min(hi, int(math.exp(x))))
    return lens


def work(case):
    op, heads = case["op"], case["heads"]
    if op == "norm":
        rows = heads * (2 * (case["g"] + 1) + (1 if case["plain"] else 0))
        return {"bytes": case["tokens"] * (rows * 2 * D + 4), "flops": 0}
    lens = _lengths(case)
    if op == "store":
        kept = case["layers"] * heads * sum(max(1, math.ceil(case["r"] * n)) for n in lens)
        return {"bytes": kept * (2 * 2 * D + 4 + 4 + 8 + 2 * ROW4 + 2 * ROW4 + 2 * 2 * D), "flops": 0}
    if op == "bounds":
        pages = sum(-(-n // case["page"]) for n in lens)
        return {"bytes": case["layers"] * heads * (sum(lens) * (2 * D if case["bits"] == 16 else ROW4) + pages * 4 * D), "flops": 0}
    g, page, row = case["g"], case["page"], 2 * ROW4 if op == "four" or case["bits"] == 4 else 4 * D
    by = sum(2 * g * D * 2 + 4 * g + 4 * D for n in lens if n >= 0)
    tokens = 0
    for n in lens:
        if n < 0:
            continue
        pages = (n + page) // page
        if op == "sparse" and pages > case["blocks"]:
            by += 4 * D * pages + 4 * case["blocks"]
            tokens += page * (case["blocks"] - 1) + n % page + 1
        else:
            tokens += n + 1
    by += tokens * (row + (8 if case["accumulate"] else 0))
    return {"bytes": heads * by, "flops": 4.0 * heads * tokens * g * D}


# --------------------------------------------------------------------------------------------- rows in 4 bits
def _quantise(x):
    """Rows [..., 128] as 80 bytes: 64 of codes (channel 2 j in the low half of byte j), then (s, lo) of each group as bf16."""
    xg = x.float().unflatten(-1, (D // GROUP, GROUP))
    lo, hi = xg.amin(-1, keepdim=True), xg.amax(-1, keepdim=True)
    s = (hi - lo) / torch.full_like(hi, 15)                                     # (by a number it would be a product with 1 / 15)
    s = ((s.view(torch.int32) + 0xFFFFF) & ~0xFFFFF).view(torch.float32)          # up to four significant bits
    s = s.masked_fill(s < 2.0 ** -120, 0.0)
    bad = ~(torch.isfinite(xg).all(-1, keepdim=True) & (s <= 2.0 ** 120))
    c = torch.where(s > 0, torch.ceil((xg - lo) / s - 0.5), 0.0)
    c = torch.where(bad, 0.0, c).clamp(0, 15).to(torch.uint8).flatten(-2)
    params = torch.cat([s, lo], -1).masked_fill(bad, math.nan).bfloat16().flatten(-2)
    return torch.cat([c[..., 0::2] | (c[..., 1::2] << 4), params.view(torch.uint8)], -1)


def _values(rows):
    """What rows of 80 bytes stand for, in 32 bits."""
    codes = rows[..., :D // 2]
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).float().unflatten(-1, (D // GROUP, GROUP))
    p = rows[..., D // 2:].contiguous().view(torch.bfloat16).float().unflatten(-1, (D // GROUP, 2))
    return (p[..., 1:] + p[..., :1] * c).flatten(-2)


# --------------------------------------------------------------------------------------------- inputs
class State:
    pass


def _paged(g, capacity, page, n_pages):
    """A page table over a pool of n_pages in which the pages of all units lie in random order, some of them unused.
    capacity: tokens that each unit must be able to hold, [layers, heads, batch]."""
    pages = (capacity + page - 1) // page
    most, total = max(1, int(pages.max())), int(pages.sum())
    table = torch.full((*capacity.shape, most), -1, dtype=torch.int32, device="cuda")
    table[torch.arange(most, device="cuda") < pages.unsqueeze(-1)] = torch.randperm(n_pages, generator=g, device="cuda")[:total].to(torch.int32)
    return table


def _keys(g, *shape):
    """Keys with a few strong channels, as rotary models have them."""
    k = torch.randn(*shape, D, generator=g, device="cuda", dtype=torch.bfloat16)
    k[..., torch.randperm(D, generator=g, device="cuda")[:4]] *= 3
    return k


def _weights(g, *shape):
    """Accumulated attention weights: log-normal, a few tokens hold most of the mass."""
    return torch.exp(2 * torch.randn(*shape, generator=g, device="cuda"))


def _prepare_norm(s, c, g):
    t, heads, qh = c["tokens"], c["heads"], c["heads"] * c["g"]
    # queries, keys and values as one projection leaves them
    s.qkv = torch.randn(t, qh + 2 * heads, D, generator=g, device="cuda").mul_(2).bfloat16()
    s.q, s.k = s.qkv[:, :qh], s.qkv[:, qh:qh + heads]
    if c["prefill"]:                                                            # a pack of sequences, each from its own position on
        cut = max(1, t // 3)
        s.positions = (torch.arange(t, device="cuda") % cut + torch.randint(0, 65536, (1,), generator=g, device="cuda")).to(torch.int32)
        s.q_out, s.k_out = (torch.empty(n, t, D, dtype=torch.bfloat16, device="cuda").transpose(0, 1) for n in (qh, heads))
    else:
        s.positions = torch.randint(0, 131072, (t,), generator=g, device="cuda", dtype=torch.int32)
        s.q_out, s.k_out = (torch.empty(t, n, D, dtype=torch.bfloat16, device="cuda") for n in (qh, heads))
    s.k_plain = torch.empty_like(s.k_out) if c["plain"] else None
    s.inv_freq = (500000.0 ** (-torch.arange(0, c["rotary"], 2, device="cuda", dtype=torch.float64) / c["rotary"])).float()
    s.qw, s.kw = ((1 + 0.3 * torch.randn(D, generator=g, device="cuda")).bfloat16() if c["weights"] else None for _ in range(2))


def prepare(case, seed):
    s = State()
    s.case = case
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    if case["op"] == "norm":
        _prepare_norm(s, case, g)
        return s
    page, heads, batch, layers, op = case["page"], case["heads"], case["batch"], case.get("layers", 1), case["op"]
    s.lens = lens = _lengths(case)
    s.bits = 4 if op in ("store", "four") else case["bits"]
    per_seq = torch.tensor(lens, device="cuda")
    if op == "store":
        s.keep = [max(1, math.ceil(case["r"] * n)) for n in lens]
        total, kk = sum(lens), sum(s.keep)
        s.k, s.v = _keys(g, layers, heads, total), torch.randn(layers, heads, total, D, generator=g, device="cuda", dtype=torch.bfloat16)
        s.attn = _weights(g, layers, heads, total)
        idx = [torch.rand(layers, heads, n, generator=g, device="cuda").topk(k, dim=2).indices.sort(dim=2).values for n, k in zip(lens, s.keep)]
        s.idx = torch.cat(idx, 2).to(torch.int32).contiguous()
        s.lengths = torch.zeros(layers, heads, batch, dtype=torch.int32, device="cuda")
        s.k_out, s.v_out = (torch.zeros(layers, heads, kk, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        capacity = torch.tensor(s.keep, device="cuda").expand(layers, heads, batch)
    else:
        s.lengths = per_seq.to(torch.int32).expand(layers, heads, batch).contiguous()
        capacity = (s.lengths.long() + (op != "bounds")).clamp(min=0)
    n_pages = 1 + int(((capacity + page - 1) // page).sum()) * 9 // 8
    s.table = _paged(g, capacity, page, n_pages)
    s.max_length = max(lens) + 1
    k, v = _keys(g, n_pages, page), torch.randn(n_pages, page, D, generator=g, device="cuda", dtype=torch.bfloat16)
    if op == "sparse":                                                          # neighbouring tokens are alike
        k += 1.5 * torch.randn(n_pages, 1, D, generator=g, device="cuda", dtype=torch.bfloat16)
    s.k_pages, s.v_pages = (_quantise(k), _quantise(v)) if s.bits == 4 else (k, v)
    s.mass = _weights(g, n_pages, page)
    s.positions = torch.randint(0, 2 * max(1, max(lens)), (n_pages, page), generator=g, device="cuda", dtype=torch.int32)
    if op in ("bounds", "sparse"):
        s.bounds = torch.zeros(n_pages, 2, D, dtype=torch.bfloat16, device="cuda")
    if op in ("four", "sparse"):
        s.q = (1.5 * torch.randn(batch, heads * case["g"], D, generator=g, device="cuda")).bfloat16()
        s.k_new, s.v_new = _keys(g, batch, heads), torch.randn(batch, heads, D, generator=g, device="cuda").bfloat16()
        s.new_positions = per_seq.to(torch.int32).clamp(min=0)
        s.out = torch.empty_like(s.q)
        s.lse = torch.empty(batch, heads * case["g"], dtype=torch.float32, device="cuda")
    if op == "four":                                                            # the appended rows, as they are held
        s.after = torch.where(s.lengths >= 0, s.lengths + 1, -1)
        s.k_row, s.v_row = (torch.zeros(1, heads, batch, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    if op == "sparse":
        s.blocks = min(case["blocks"], s.table.shape[-1])
        s.last = min(2, s.blocks)                                               # the newest pages are always attended to, and the first
        s.first = min(1, s.blocks - s.last)
        s.chosen = torch.full((1, heads, batch, s.blocks), -1, dtype=torch.int32, device="cuda")
        s.chosen_lengths = torch.zeros(1, heads, batch, dtype=torch.int32, device="cuda")
        _plain_bounds(s)
    if own:
        from paper_2507_08143_b200 import binding as B
        Cache = B.PagedCache4 if s.bits == 4 else B.PagedCache
        s.cache = Cache(s.k_pages, s.v_pages, s.table, mass=s.mass, positions=s.positions)
        if op == "store":
            s.shape, s.kept_shape = B.Shape(layers, heads, D, 48, lens), B.Shape(layers, heads, D, 48, s.keep)
        if op == "four":
            s.opt = B.decode_options(case["g"], s.max_length, scale=D ** -0.5, softcap=case["softcap"], accumulate=case["accumulate"])
            s.ws = B.alloc_paged_attention_workspace(s.cache, s.opt)
            s.row_shape = B.Shape(1, heads, D, 48, [1] * batch)
        if op == "sparse":
            s.reduced = Cache(s.k_pages, s.v_pages, s.chosen, mass=s.mass, positions=s.positions)
            s.opt = B.decode_options(case["g"], s.blocks * page, scale=D ** -0.5, accumulate=case["accumulate"])
            s.ws = B.alloc_paged_attention_workspace(s.reduced, s.opt)
            s.select_ws = B.alloc_paged_select_workspace(s.cache, s.max_length)
    return s


# --------------------------------------------------------------------------------------------- plain forms
def _rotate(c, x, angle):
    """Rotation of the first `rotary` channels of x [tokens, heads, 128] (32 bits) by angle [tokens, rotary / 2] (64 bits)."""
    r = c["rotary"]
    cos, sin = angle.cos().float().unsqueeze(1), angle.sin().float().unsqueeze(1)
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if c["interleaved"] else (x[..., :r // 2], x[..., r // 2:r])
    a, b = a * cos - b * sin, b * cos + a * sin
    rotated = torch.stack([a, b], -1).flatten(-2) if c["interleaved"] else torch.cat([a, b], -1)
    return torch.cat([rotated, x[..., r:]], -1)


def _plain_norm(s):
    c = s.case
    angle = s.positions.double().unsqueeze(1) * s.inv_freq.double()
    q, k = s.q.float(), s.k.float()
    if c["weights"]:
        q = q * torch.rsqrt(q.square().mean(-1, keepdim=True) + 1e-6) * s.qw.float()
        k = k * torch.rsqrt(k.square().mean(-1, keepdim=True) + 1e-6) * s.kw.float()
    s.q_out.copy_(_rotate(c, q, angle))
    s.k_out.copy_(_rotate(c, k, angle))
    if c["plain"]:
        s.k_plain.copy_(k)


def _slot_rows(table, page, slot):
    """Row of the flattened pools of every slot, [..., slots]; -1 where the table has no page."""
    pid = table.long()[..., slot // page]
    return torch.where(pid >= 0, pid * page + slot % page, -1)


def _plain_store(s):
    c = s.case
    layers, heads, batch, page = c["layers"], c["heads"], c["batch"], c["page"]
    dev = s.k.device
    keep, start = torch.tensor(s.keep, device=dev), torch.tensor([0] + s.lens[:-1], device=dev).cumsum(0)
    of_b = torch.repeat_interleave(torch.arange(batch, device=dev), keep)
    slot = torch.arange(of_b.numel(), device=dev) - (keep.cumsum(0) - keep)[of_b]
    table = s.table.view(layers * heads, batch, -1).long()
    at = table[:, of_b, slot // page] * page + slot % page                      # [layers * heads, kept]
    idx = s.idx.long().view(layers * heads, -1)
    token = idx + start[of_b]
    rows = torch.arange(layers * heads, device=dev).unsqueeze(1)
    k, v = s.k_pages.view(-1, ROW4), s.v_pages.view(-1, ROW4)
    k[at] = _quantise(s.k.view(layers * heads, -1, D)[rows, token])
    v[at] = _quantise(s.v.view(layers * heads, -1, D)[rows, token])
    s.mass.view(-1)[at] = s.attn.view(layers * heads, -1)[rows, token]
    s.positions.view(-1)[at] = idx.to(torch.int32)
    s.lengths.copy_(keep.expand(layers, heads, batch))
    s.k_out.copy_(_values(k[at]).view(s.k_out.shape))
    s.v_out.copy_(_values(v[at]).view(s.v_out.shape))


def _plain_bounds(s):
    """Least and greatest key of every page of every unit, over its tokens, into s.bounds."""
    page = s.case["page"]
    tokens = (s.lengths.long().clamp(min=0).unsqueeze(-1) - page * torch.arange(s.table.shape[-1], device="cuda")).clamp(max=page)
    used = tokens > 0                                                           # [layers, heads, batch, pages]
    ids = s.table.long()[used]
    live = (torch.arange(page, device="cuda") < tokens[used].unsqueeze(1)).unsqueeze(-1)
    k = s.k_pages[ids]
    k = _values(k) if s.bits == 4 else k.float()
    s.bounds[ids, 0] = k.masked_fill(~live, math.inf).amin(1).bfloat16()
    s.bounds[ids, 1] = k.masked_fill(~live, -math.inf).amax(1).bfloat16()


def _plain_select(s):
    """The pages of each unit that the step's queries get: s.chosen, s.chosen_lengths; the new key enters its page's bounds."""
    c, page = s.case, s.case["page"]
    heads, batch, g = c["heads"], c["batch"], c["g"]
    n = s.lengths[0].long()                                                     # [heads, batch]
    alive = n >= 0
    slot = n.clamp(min=0)
    own_page = torch.gather(s.table[0].long(), 2, (slot // page).unsqueeze(-1)).squeeze(-1)[alive]
    k_new, begun = s.k_new.transpose(0, 1)[alive], (slot % page > 0)[alive].unsqueeze(1)
    s.bounds[own_page, 0] = torch.where(begun, torch.minimum(s.bounds[own_page, 0], k_new), k_new)
    s.bounds[own_page, 1] = torch.where(begun, torch.maximum(s.bounds[own_page, 1], k_new), k_new)
    pages = torch.where(alive, slot // page + 1, 0).unsqueeze(-1)
    block = torch.arange(s.table.shape[-1], device="cuda")
    there = block < pages
    b = s.bounds[s.table[0].long().clamp(min=0)].double()                       # [heads, batch, blocks, 2, D]
    q = s.q.double().view(batch, heads, g, D).transpose(0, 1)                   # [heads, batch, g, D]
    score = q.clamp(max=0) @ b[..., 0, :].transpose(-1, -2) + q.clamp(min=0) @ b[..., 1, :].transpose(-1, -2)
    score = score.amax(2).float()
    score = torch.where((block < s.first) | (block >= pages - s.last), math.inf, score).masked_fill(~there, -math.inf)
    best = score.sort(dim=-1, descending=True, stable=True).indices[..., :s.blocks]
    best = torch.where(torch.arange(s.blocks, device="cuda") < pages, best, 1 << 40).sort(dim=-1).values
    taken = best < 1 << 40
    s.chosen[0] = torch.where(taken, torch.gather(s.table[0].long(), 2, best.clamp(max=block.numel() - 1)), -1).to(torch.int32)
    count = pages.squeeze(-1).clamp(max=s.blocks)
    s.chosen_lengths[0] = torch.where(alive, (count - 1) * page + slot % page, n).to(torch.int32)


def _plain_attention(s, table, lengths, most, softcap):
    """The new token's row into its slot, then softmax(scale q K^T) V over a unit's slots, weights added to each token's."""
    c, page = s.case, s.case["page"]
    heads, batch, g = c["heads"], c["batch"], c["g"]
    n = lengths[0].long()                                                       # [heads, batch]
    alive = n >= 0
    slot = n.clamp(min=0)
    at = (torch.gather(table[0].long(), 2, (slot // page).unsqueeze(-1)).squeeze(-1) * page + slot % page)[alive]
    kp, vp, mass = s.k_pages.flatten(0, 1), s.v_pages.flatten(0, 1), s.mass.view(-1)
    held = _quantise if s.bits == 4 else (lambda x: x)
    kp[at], vp[at] = held(s.k_new.transpose(0, 1)[alive]), held(s.v_new.transpose(0, 1)[alive])
    s.positions.view(-1)[at] = s.new_positions.expand(heads, batch)[alive]
    mass[at] = 0
    n = torch.where(alive, n + 1, 0)
    slot = torch.arange(min(most, table.shape[-1] * page), device="cuda")
    rows = _slot_rows(table[0], page, slot).clamp(min=0)                        # [heads, batch, slots]
    live = slot < n.unsqueeze(-1)
    value = _values if s.bits == 4 else (lambda x: x.float())
    k = value(kp[rows]).masked_fill_(~live.unsqueeze(-1), 0.0)
    v = value(vp[rows]).masked_fill_(~live.unsqueeze(-1), 0.0)
    q = s.q.float().view(batch, heads, g, D).transpose(0, 1)                    # [heads, batch, g, D]
    y = (q * D ** -0.5) @ k.transpose(-1, -2)
    if softcap:
        y = softcap * torch.tanh(y / softcap)
    y = y.masked_fill(~live.unsqueeze(2), -math.inf)
    top = y.amax(-1, keepdim=True).clamp(min=-3e38)
    p = torch.exp(y - top)
    z = p.sum(-1, keepdim=True)
    p = p / z.clamp(min=1e-30)
    s.out.copy_((p @ v).transpose(0, 1).reshape(batch, heads * g, D))
    s.lse.copy_((top + torch.log(z)).squeeze(-1).transpose(0, 1).reshape(batch, heads * g))
    if c["accumulate"]:
        mass[rows[live]] += p.sum(2)[live]
    return at, alive


def run(s):
    c, op = s.case, s.case["op"]
    if own:
        from paper_2507_08143_b200 import binding as B
        new = {} if op not in ("four", "sparse") else dict(k_new=s.k_new, v_new=s.v_new, new_positions=s.new_positions, lse_out=s.lse)
        if op == "norm":
            B.norm_rope(s.q, s.k, s.positions, s.inv_freq, s.q_out, s.k_out, k_plain_out=s.k_plain, q_weight=s.qw, k_weight=s.kw, eps=1e-6,
                        interleaved=c["interleaved"])
        elif op == "store":
            B.paged_fill(s.cache, s.shape, s.k, s.v, s.keep, idx=s.idx, mass_in=s.attn, lengths_out=s.lengths)
            B.paged_read(s.cache, s.kept_shape, s.lengths, s.k_out, s.v_out)
        elif op == "four":
            B.paged_attention(s.cache, 0, s.opt, s.q, s.lengths, s.out, s.ws, **new)
            B.paged_read(s.cache, s.row_shape, s.after, s.k_row, s.v_row, first=s.lengths)
        elif op == "bounds":
            B.paged_bounds(s.cache, s.lengths, s.bounds, s.max_length)
        else:
            B.paged_select(s.cache, 0, c["g"], s.q, s.lengths, s.bounds, s.chosen, s.chosen_lengths, s.select_ws, s.max_length,
                           first_pages=s.first, last_pages=s.last, k_new=s.k_new)
            B.paged_attention(s.reduced, 0, s.opt, s.q, s.chosen_lengths, s.out, s.ws, **new)
    elif op == "norm":
        _plain_norm(s)
    elif op == "store":
        _plain_store(s)
    elif op == "four":
        at, alive = _plain_attention(s, s.table, s.lengths, s.max_length, c["softcap"])
        s.k_row[0][alive] = _values(s.k_pages.flatten(0, 1)[at]).bfloat16()
        s.v_row[0][alive] = _values(s.v_pages.flatten(0, 1)[at]).bfloat16()
    elif op == "bounds":
        _plain_bounds(s)
    else:
        _plain_select(s)
        _plain_attention(s, s.chosen, s.chosen_lengths, s.blocks * c["page"], 0.0)
    if op == "norm":
        return {"q": s.q_out, "k": s.k_out, "k_plain": s.k_plain}
    if op == "store":
        return {"k": s.k_out, "v": s.v_out, "mass": s.mass, "positions": s.positions, "lengths": s.lengths}
    if op == "bounds":
        return {"bounds": s.bounds}
    got = {"out": s.out, "lse": s.lse, "mass": s.mass, "positions": s.positions}
    if op == "four":
        return dict(got, k_row=s.k_row, v_row=s.v_row)
    return dict(got, bounds=s.bounds, chosen=s.chosen, lengths=s.chosen_lengths)


# --------------------------------------------------------------------------------------------- exact values
def _held64(x):
    """What rows x [n, 128] are held as in 4 bits, in 64 bits from the definition."""
    x = x.double().view(-1, D // GROUP, GROUP)
    lo = x.min(-1, keepdim=True).values
    step = torch.div(x.max(-1, keepdim=True).values - lo, torch.full_like(lo, 15))
    m, e = torch.frexp(step)                                                    # step = m 2^e, 1/2 <= m < 1
    step = torch.ldexp(torch.ceil(m * 16) / 16, e)
    c = torch.where(step > 0, torch.ceil((x - lo) / step - 0.5), torch.zeros_like(x))
    return (lo + c * step).view(-1, D)


def _stands_for64(rows):
    """What rows of 80 bytes [n, 80] stand for, in 64 bits."""
    shift = torch.tensor([0, 4], device=rows.device, dtype=torch.uint8)
    c = ((rows[:, :64, None] >> shift) & 15).reshape(-1, 4, 32).double()
    p = rows[:, 64:].contiguous().view(torch.bfloat16).double().view(-1, 4, 2)
    return (c * p[:, :, 0:1] + p[:, :, 1:2]).reshape(-1, D)


def _exact_norm(s):
    c = s.case
    r = c["rotary"]
    out = []
    for x, w in ((s.q, s.qw), (s.k, s.kw)):
        x = x.double()
        if w is not None:
            x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / D + 1e-6) * w.double()
        z = torch.polar(torch.ones_like(s.inv_freq, dtype=torch.float64), torch.zeros_like(s.inv_freq, dtype=torch.float64))
        angle = s.positions.double()[:, None, None] * s.inv_freq.double()
        turn = torch.polar(torch.ones_like(angle), angle) * z
        y = x.clone()
        even, odd = (slice(0, r, 2), slice(1, r, 2)) if c["interleaved"] else (slice(0, r // 2), slice(r // 2, r))
        z = torch.complex(x[..., even].contiguous(), x[..., odd].contiguous()) * turn
        y[..., even], y[..., odd] = z.real, z.imag
        out += [y, x]
    return {"q": out[0], "k": out[2], "k_plain": out[3] if c["plain"] else None}


def _exact_store(s):
    c = s.case
    start = 0
    ks, vs = [], []
    at = 0
    for n, keep in zip(s.lens, s.keep):
        idx = s.idx[:, :, at:at + keep].long() + start
        for x, to in ((s.k, ks), (s.v, vs)):
            rows = torch.gather(x, 2, idx.unsqueeze(-1).expand(-1, -1, -1, D))
            to.append(_held64(rows.reshape(-1, D)).view(rows.shape))
        start, at = start + n, at + keep
    return {"k": torch.cat(ks, 2), "v": torch.cat(vs, 2), "mass": None, "positions": None, "lengths": None}


def _exact_bounds(s):
    page = s.case["page"]
    want = torch.zeros(*s.bounds.shape, dtype=torch.float64, device="cuda")
    table = s.table.flatten(0, 2).tolist()
    last = []                                                                   # (page id, tokens in it)
    for row, n in zip(table, s.lengths.flatten().tolist()):
        last += [(row[j], min(page, n - j * page)) for j in range(-(-max(n, 0) // page))]
    for tokens in sorted({t for _, t in last}):                                 # pages with as many tokens together
        ids = torch.tensor([p for p, t in last if t == tokens], device="cuda")
        for part in ids.split(1 << 14):
            k = s.k_pages[part, :tokens]
            k = _stands_for64(k.reshape(-1, ROW4)).view(-1, tokens, D) if s.bits == 4 else k.double()
            want[part, 0], want[part, 1] = k.min(1).values, k.max(1).values
    return {"bounds": want}


def _exact_attention(s):
    """Unit by unit; for `sparse` over the pages that the definition chooses."""
    case = s.case
    page, heads, g, batch, op = case["page"], case["heads"], case["g"], case["batch"], case["op"]
    out = torch.zeros(batch, heads * g, D, dtype=torch.float64, device="cuda")
    lse = torch.full((batch, heads * g), -math.inf, dtype=torch.float64, device="cuda")
    mass = s.mass.double()
    rows = torch.zeros(2, 1, heads, batch, D, dtype=torch.float64, device="cuda")
    for h in range(heads):
        for b in range(batch):
            n = s.lens[b]
            if n < 0:
                continue
            used = s.table[0, h, b, : n // page + 1].long()
            q = s.q[b, h * g:(h + 1) * g].double()
            if op == "sparse" and used.numel() > s.blocks:
                lo, hi = s.bounds[used, 0].double(), s.bounds[used, 1].double()
                score = torch.maximum(q[:, None, :] * lo, q[:, None, :] * hi).sum(-1).max(0).values.float()
                score[: s.first] = math.inf
                score[used.numel() - s.last:] = math.inf
                used = used[torch.argsort(-score, stable=True)[: s.blocks].sort().values]
            new = [x[b, h][None] for x in (s.k_new, s.v_new)]
            if s.bits == 4:
                k, v = (_stands_for64(x[used].view(-1, ROW4)) for x in (s.k_pages, s.v_pages))
                new = [_held64(x) for x in new]
            else:
                k, v = (x[used].reshape(-1, D).double() for x in (s.k_pages, s.v_pages))
            m = (used.numel() - 1) * page + n % page
            k, v = torch.cat([k[:m], new[0].double()]), torch.cat([v[:m], new[1].double()])
            rows[0, 0, h, b], rows[1, 0, h, b] = new[0][0], new[1][0]
            y = torch.einsum("gd,nd->gn", q, k) / math.sqrt(D)
            if case.get("softcap"):
                y = case["softcap"] * torch.tanh(y / case["softcap"])
            lse[b, h * g:(h + 1) * g] = torch.logsumexp(y, 1)
            p = torch.softmax(y, 1)
            out[b, h * g:(h + 1) * g] = p @ v
            slots = torch.arange(p.shape[1], device="cuda")
            mass[used[m // page], m % page] = 0
            if case["accumulate"]:
                mass[used[slots // page], slots % page] += p.sum(0)
    got = {"out": out, "lse": lse, "mass": mass, "positions": None}
    if op == "four":
        return dict(got, k_row=rows[0], v_row=rows[1])
    return dict(got, bounds=None, chosen=None, lengths=None)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        return _exact_norm(s)
    if case["op"] == "store":
        return _exact_store(s)
    return _exact_bounds(s) if case["op"] == "bounds" else _exact_attention(s)
