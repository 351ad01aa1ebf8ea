"""The paged-cache operators as measured: cases, inputs, plain forms and exact values.

Three operators work on one cache of key and value pages in which every (layer, KV head, sequence)
unit owns a row of the page table and a length of its own, because a compressed prefill keeps
different tokens (and, across heads, different numbers of them) in every head:

  fill       the rows that a compression pass kept, gathered from the prefill's K and V into pages
  attention  one new token per sequence against its pages: softmax(scale q K^T) V, the token itself
             appended, the weights added to each cached token's accumulated attention weight
  evict      a cycle of a cache that has reached its budget: a block of tokens is appended, the tokens
             of least accumulated weight outside the recent window leave, and the holes they leave are
             filled from the tail

All three are memory-bound; `work` counts every byte that has to be touched once."""
import math
import random

import torch

own = False

D = 128                                      # head dimension of every configuration here


# --------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # the smallest call: one sequence of the 1 x 2 head configuration at half retention, where latency counts
        dict(name="attention c0", op="attention", heads=2, batch=1, g=4, lo=511, hi=511, page=16, accumulate=False, softcap=0.0, append=True),
        # 8192 tokens at r = 0.3 in one layer of 8 heads x 4 queries, weights accumulated for a later eviction
        dict(name="attention c1", op="attention", heads=8, batch=1, g=4, lo=2457, hi=2457, page=16, accumulate=True, softcap=0.0, append=True),
        # 4 heads x 7 queries, eight contexts of 32768 tokens at retentions of 0.2 to 0.6, odd lengths
        dict(name="attention c2", op="attention", heads=4, batch=8, g=7, lo=6553, hi=19661, page=32, accumulate=True, softcap=0.0, append=True),
        # the longest uncompressed context, one sequence: the work of a few heads split over the whole GPU
        dict(name="attention c3", op="attention", heads=8, batch=1, g=5, lo=131071, hi=131071, page=64, accumulate=False, softcap=0.0, append=True),
        # a ragged batch of sixteen compressed contexts of 2K to 64K tokens
        dict(name="attention c4", op="attention", heads=8, batch=16, g=4, lo=409, hi=32768, page=16, accumulate=True, softcap=0.0, append=True),
        # a padded batch of short conversations of a model that caps its scores; some rows hold no sequence, some no token yet
        dict(name="attention padded", op="attention", heads=8, batch=64, g=2, lo=-1, hi=2047, page=16, accumulate=True, softcap=50.0, append=True),
        # the small configuration's prefill into pages
        dict(name="fill c0", op="fill", layers=1, heads=2, batch=1, lo=1024, hi=1024, r=0.5, page=16, across=False),
        # 32 layers x 8 heads of an 8192-token prefill at r = 0.3
        dict(name="fill c1", op="fill", layers=32, heads=8, batch=1, lo=8192, hi=8192, r=0.3, page=16, across=False),
        # two layers of the ragged batch, budgets shared across the heads of a layer: every head its own length
        dict(name="fill c4", op="fill", layers=2, heads=8, batch=16, lo=2048, hi=65536, r=0.3, page=32, across=True),
        # every step one token in, one token out, all layers at once
        dict(name="evict c1", op="evict", layers=32, heads=8, batch=1, lo=2458, hi=2458, block=1, recent=64, page=16),
        # a block of 128 tokens in and out, four layers of the ragged batch
        dict(name="evict c4", op="evict", layers=4, heads=8, batch=16, lo=410, hi=32768, block=128, recent=256, page=32),
        # few long units: one layer at 0.32 of 131072 tokens, 8192 tokens of a new turn against as many old ones
        dict(name="evict c3", op="evict", layers=1, heads=8, batch=1, lo=41944, hi=41944, block=8192, recent=8192, page=64),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = 8 * 131072                        # tokens of a drawn case over all its heads: what the longest listed context has
    heads = rng.choice((1, 2, 4, 8))
    page = rng.choice((8, 16, 32, 64, 128))
    op = rng.choice(("attention", "attention", "fill", "evict"))
    if op == "attention":
        batch = _log_uniform(rng, 1, 64)
        hi = _log_uniform(rng, 1, min(131071, most // (heads * batch)))
        lo = rng.choice((hi, max(0, hi // 16), -1))
        return dict(op=op, heads=heads, batch=batch, g=rng.choice((1, 2, 3, 4, 5, 6, 7, 8, 12, 16)), lo=lo, hi=hi, page=page,
                    accumulate=rng.random() < 0.6, softcap=rng.choice((0.0, 0.0, 30.0, 50.0)), append=rng.random() < 0.8)
    layers = _log_uniform(rng, 1, 32)
    batch = _log_uniform(rng, 1, 16)
    if op == "fill":
        hi = _log_uniform(rng, 16, min(131072, 2 * most // (layers * heads * batch)))
        return dict(op=op, layers=layers, heads=heads, batch=batch, lo=rng.choice((hi, max(1, hi // 16))), hi=hi,
                    r=rng.choice((0.2, 0.3, 0.32, 0.5)), page=page, across=rng.random() < 0.5)
    hi = _log_uniform(rng, 64, min(131072, most // (layers * heads * batch)))
    lo = rng.choice((hi, max(32, hi // 16)))
    block = min(_log_uniform(rng, 1, 4096), max(1, lo // 4))
    return dict(op=op, layers=layers, heads=heads, batch=batch, lo=lo, hi=hi, block=block, recent=rng.randint(block, lo // 2) if block < lo // 2 else block, page=page)


def _mean_length(case):
    """Expected length of the sequences that prepare() makes, for `work`."""
    lo, hi, batch = case["lo"], case["hi"], case["batch"]
    if lo == hi or batch == 1:
        return float(hi)
    a = max(1, lo)
    mean = (hi - a) / math.log(hi / a) if hi > a else float(hi)
    return (hi + (batch - 1) * mean * (0.8 if lo < 0 else 1.0)) / batch


def work(case):
    row = 2 * 2 * D                          # a token's K and V in one head
    if case["op"] == "attention":
        units, n = case["heads"] * case["batch"], _mean_length(case) + case["append"]
        by = units * n * row + (units * n * 8 if case["accumulate"] else 0) + units * (2 * case["g"] * D * 2 + 4 * case["g"])
        by += units * 2 * row if case["append"] else 0
        return {"bytes": by, "flops": 4.0 * units * n * case["g"] * D}
    units = case["layers"] * case["heads"] * case["batch"]
    if case["op"] == "fill":
        kept = units * max(1.0, case["r"] * _mean_length(case))
        return {"bytes": kept * (2 * row + 4 + 4 + 8), "flops": 0}
    n, e = _mean_length(case) + case["block"], case["block"]
    # the block in (read and written, with weight and position), weights and positions of all read once, the block's rows moved into holes
    return {"bytes": units * (e * (2 * row + 12) + n * 8 + e * (2 * row + 16)), "flops": 0}


# --------------------------------------------------------------------------------------------- inputs
class State:
    pass


def _paged(g, layers, heads, batch, capacity, page, n_pages):
    """A page table over a pool of n_pages in which the pages of all units lie in random order, some of them unused.
    capacity: tokens that each unit must be able to hold, [layers, heads, batch]."""
    pages = (capacity + page - 1) // page
    most, total = int(pages.max()), int(pages.sum())
    ids = torch.randperm(n_pages, generator=g, device="cuda")[:total].to(torch.int32)
    table = torch.full((layers, heads, batch, max(1, most)), -1, dtype=torch.int32, device="cuda")
    used = torch.arange(max(1, most), device="cuda") < pages.unsqueeze(-1)
    table[used] = ids
    return table


def _keys(g, *shape):
    """Keys with a few strong channels, as rotary models have them."""
    k = torch.randn(*shape, D, generator=g, device="cuda", dtype=torch.bfloat16)
    k[..., torch.randperm(D, generator=g, device="cuda")[:4]] *= 3
    return k


def _weights(g, *shape):
    """Accumulated attention weights: log-normal, a few tokens hold most of the mass."""
    return torch.exp(2 * torch.randn(*shape, generator=g, device="cuda"))


def prepare(case, seed):
    s = State()
    s.case = case
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    page, heads, batch = case["page"], case["heads"], case["batch"]
    layers = case.get("layers", 1)
    # one length per sequence between lo and hi, spread over the logarithm, the first of them hi; with lo = -1 a
    # tenth of the sequences is empty and a tenth of the rows holds no sequence (-1)
    lo, hi = case["lo"], case["hi"]
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))    # the shapes are the case's, the values the seed's
    lens = [hi]
    for _ in range(batch - 1):
        u, x = rng.random(), rng.uniform(math.log(max(1, lo)), math.log(max(1, hi)))
        lens.append((-1 if u < 0.1 else 0) if lo < 0 and u < 0.2 else hi if lo == hi else min(hi, int(math.exp(x))))
    s.lens = lens
    per_seq = torch.tensor(lens, device="cuda")
    if case["op"] == "attention":
        s.lengths = per_seq.to(torch.int32).expand(1, heads, batch).contiguous()
        capacity = (s.lengths.long() + 1).clamp(min=1)
        s.q = (1.5 * torch.randn(batch, heads * case["g"], D, generator=g, device="cuda")).bfloat16()
        s.k_new, s.v_new = _keys(g, batch, heads), torch.randn(batch, heads, D, generator=g, device="cuda").bfloat16()
        s.new_positions = per_seq.to(torch.int32).clamp(min=0)
        s.max_length = max(lens) + 1
        n_pages = 1 + heads * sum((max(n, 0) + page) // page for n in lens)
        s.out = torch.empty_like(s.q)
        s.lse = torch.empty(batch, heads * case["g"], dtype=torch.float32, device="cuda")
    elif case["op"] == "fill":
        keep = [max(1, math.ceil(case["r"] * n)) for n in lens]
        s.keep, s.seqlens = keep, lens
        total, kk = sum(lens), sum(keep)
        s.k, s.v = _keys(g, layers, heads, total), torch.randn(layers, heads, total, D, generator=g, device="cuda", dtype=torch.bfloat16)
        s.attn = _weights(g, layers, heads, total)
        s.first_position = torch.zeros(batch, dtype=torch.int32, device="cuda")
        if case["across"]:
            # the heads * keep[b] best of all heads' scores, head by head, ascending within a head
            idx, offs = [], torch.zeros(layers, batch, heads + 1, dtype=torch.int32, device="cuda")
            for b, n in enumerate(lens):
                score = torch.rand(layers, heads, n, generator=g, device="cuda") * torch.linspace(0.5, 1.0, heads, device="cuda")[None, :, None]
                at = score.view(layers, heads * n).topk(heads * keep[b], dim=1).indices.sort(dim=1).values
                idx.append((at % n).to(torch.int32))
                offs[:, b, 1:] = torch.nn.functional.one_hot(at // n, heads).sum(1).cumsum(1)
            s.idx, s.head_offsets = torch.cat(idx, 1).contiguous(), offs
            capacity = (offs[:, :, 1:] - offs[:, :, :-1]).permute(0, 2, 1).long().contiguous()
        else:
            idx = [torch.rand(layers, heads, n, generator=g, device="cuda").topk(keep[b], dim=2).indices.sort(dim=2).values for b, n in enumerate(lens)]
            s.idx, s.head_offsets = torch.cat(idx, 2).to(torch.int32).contiguous(), None
            capacity = torch.tensor(keep, device="cuda").expand(layers, heads, batch).contiguous()
        s.lengths_out = torch.zeros(layers, heads, batch, dtype=torch.int32, device="cuda")
        n_pages = 1 + layers * sum(heads * n // page + heads for n in keep)          # enough whichever head keeps them
    else:
        e = case["block"]
        # every head its own budget, as a selection across heads leaves them: up to an eighth below its sequence's
        cut = (torch.rand(layers, heads, batch, generator=g, device="cuda") * (per_seq - case["recent"]).clamp(min=0) / 8).long()
        s.budgets = (per_seq - cut).clamp(min=case["recent"]).to(torch.int32)
        s.full = s.budgets + e
        capacity = s.full.long()
        s.max_length = max(lens) + e
        n_pages = layers * heads * sum((n + e) // page + 1 for n in lens)
        s.k_in = _keys(g, layers, heads, batch * e)
        s.v_in = torch.randn(layers, heads, batch * e, D, generator=g, device="cuda", dtype=torch.bfloat16)
        s.mass_in = 0.1 * _weights(g, layers, heads, batch * e)
        s.next_position = torch.full((batch,), 2 * max(lens), dtype=torch.int32, device="cuda")
        s.lengths_out = torch.zeros_like(s.budgets)
    s.table = _paged(g, layers, heads, batch, capacity, page, n_pages)
    s.k_pages = _keys(g, n_pages, page)
    s.v_pages = torch.randn(n_pages, page, D, generator=g, device="cuda", dtype=torch.bfloat16)
    s.mass = _weights(g, n_pages, page)
    s.positions = torch.randint(0, 2 * max(1, max(lens)), (n_pages, page), generator=g, device="cuda", dtype=torch.int32)
    if case["op"] == "evict":
        # a unit's tokens have distinct positions below the next one, in the order of their slots at first
        n = s.table.shape[-1] * page
        slot = torch.arange(n, device="cuda")
        rows = _slot_rows(s.table, page, slot)
        s.positions.view(-1)[rows[rows >= 0]] = (2 * slot).expand_as(rows)[rows >= 0].to(torch.int32) % (2 * max(lens))
    if own:
        from paper_2507_08143_b200 import binding as B
        s.cache = B.PagedCache(s.k_pages, s.v_pages, s.table, mass=s.mass, positions=s.positions)
        if case["op"] == "attention":
            s.opt = B.decode_options(case["g"], s.max_length, scale=D ** -0.5, softcap=case["softcap"], accumulate=case["accumulate"])
            s.ws = B.alloc_paged_attention_workspace(s.cache, s.opt)
        else:
            s.shape = B.Shape(layers, heads, D, 48, lens if case["op"] == "fill" else [case["block"]] * batch)
    return s


# --------------------------------------------------------------------------------------------- plain forms
def _slot_rows(table, page, slot):
    """Row of the flattened pools of every slot, [..., slots]; -1 where the table has no page."""
    pid = table.long()[..., slot // page]
    return torch.where(pid >= 0, pid * page + slot % page, -1)


def _plain_attention(s):
    c, page = s.case, s.case["page"]
    heads, batch, g = c["heads"], c["batch"], c["g"]
    dev = s.q.device
    n = s.lengths[0].long()                                                     # [heads, batch]
    kp, vp, mass, pos = s.k_pages.view(-1, D), s.v_pages.view(-1, D), s.mass.view(-1), s.positions.view(-1)
    if c["append"]:
        alive = n >= 0
        own_slot = n.clamp(min=0)
        at = torch.gather(s.table[0].long(), 2, (own_slot // page).unsqueeze(-1)).squeeze(-1) * page + own_slot % page
        at = at[alive]
        kp[at] = s.k_new.transpose(0, 1)[alive]
        vp[at] = s.v_new.transpose(0, 1)[alive]
        pos[at] = s.new_positions.expand(heads, batch)[alive]
        mass[at] = 0
        n = torch.where(alive, n + 1, 0)
    n = n.clamp(min=0)
    slot = torch.arange(s.max_length, device=dev)
    rows = _slot_rows(s.table[0], page, slot).clamp(min=0)                      # [heads, batch, slots]
    live = slot < n.unsqueeze(-1)
    k = torch.where(live.unsqueeze(-1), kp[rows].float(), 0.0)
    v = torch.where(live.unsqueeze(-1), vp[rows].float(), 0.0)
    q = s.q.float().view(batch, heads, g, D).transpose(0, 1)                    # [heads, batch, g, D]
    y = (q * D ** -0.5) @ k.transpose(-1, -2)
    if c["softcap"]:
        y = c["softcap"] * torch.tanh(y / c["softcap"])
    y = y.masked_fill(~live.unsqueeze(2), -math.inf)
    top = y.amax(-1, keepdim=True).clamp(min=-3e38)
    p = torch.exp(y - top)
    z = p.sum(-1, keepdim=True)
    p = p / z.clamp(min=1e-30)
    out = (p @ v).transpose(0, 1).reshape(batch, heads * g, D).to(torch.bfloat16)
    lse = (top + torch.log(z)).squeeze(-1).transpose(0, 1).reshape(batch, heads * g)
    if c["accumulate"]:
        mass[rows[live]] += p.sum(2)[live]
    return {"out": out, "lse": lse, "mass": s.mass, "positions": s.positions, "k_pages": s.k_pages, "v_pages": s.v_pages}


def _plain_put(s, k, v, weight, first, idx_rows, unit_of, slot_of, source_of):
    """Rows `source_of` of k / v [layers*heads, tokens, D] into the slots `slot_of` of the units `unit_of`."""
    page = s.case["page"]
    table = s.table.view(-1, s.table.shape[-1]).long()
    at = table[unit_of, slot_of // page] * page + slot_of % page
    lh = unit_of // s.case["batch"]
    s.k_pages.view(-1, D)[at] = k[lh, source_of]
    s.v_pages.view(-1, D)[at] = v[lh, source_of]
    s.mass.view(-1)[at] = weight[lh, source_of]
    s.positions.view(-1)[at] = (first[unit_of % s.case["batch"]] + idx_rows).to(torch.int32)


def _plain_fill(s):
    c = s.case
    layers, heads, batch = c["layers"], c["heads"], c["batch"]
    dev = s.k.device
    keep, start = torch.tensor(s.keep, device=dev), torch.tensor([0] + s.seqlens[:-1], device=dev).cumsum(0)
    of_b = torch.repeat_interleave(torch.arange(batch, device=dev), heads * keep if c["across"] else keep)
    head_of = None
    if c["across"]:
        within = torch.arange(of_b.numel(), device=dev) - (heads * (keep.cumsum(0) - keep))[of_b]
        offs = s.head_offsets.long()                                            # [layers, batch, heads + 1]
        mine = offs[:, of_b]                                                    # [layers, rows, heads + 1]
        head_of = (within[None, :, None] >= mine[..., 1:]).sum(-1)
        slot = within - torch.gather(mine, 2, head_of.unsqueeze(-1)).squeeze(-1)
        unit = (torch.arange(layers, device=dev)[:, None] * heads + head_of) * batch + of_b
        lengths = (offs[..., 1:] - offs[..., :-1]).permute(0, 2, 1)
    else:
        slot = (torch.arange(of_b.numel(), device=dev) - (keep.cumsum(0) - keep)[of_b]).expand(layers * heads, -1)
        unit = torch.arange(layers * heads, device=dev)[:, None] * batch + of_b
        lengths = keep.expand(layers, heads, batch)
    idx = s.idx.long().view(unit.shape)
    _plain_put(s, s.k.view(layers * heads, -1, D), s.v.view(layers * heads, -1, D), s.attn.view(layers * heads, -1), s.first_position.long(),
               idx.reshape(-1), unit.reshape(-1), slot.reshape(-1), (idx + start[of_b]).reshape(-1))
    s.lengths_out.copy_(lengths)


def _plain_evict(s):
    c = s.case
    layers, heads, batch, e, page = c["layers"], c["heads"], c["batch"], c["block"], c["page"]
    dev = s.k_in.device
    units = layers * heads * batch
    budget = s.budgets.view(-1).long()
    # the block is appended behind the unit's tokens
    unit = torch.arange(units, device=dev).repeat_interleave(e)
    j = torch.arange(e, device=dev).repeat(units)
    _plain_put(s, s.k_in.view(layers * heads, -1, D), s.v_in.view(layers * heads, -1, D), s.mass_in.view(layers * heads, -1),
               s.next_position.long(), j, unit, budget[unit] + j, (unit % batch) * e + j)
    s.next_position += e
    # rank: recent tokens first, then by weight, then by slot
    slot = torch.arange(min(s.max_length, s.table.shape[-1] * page), device=dev)
    rows = _slot_rows(s.table.view(units, -1), page, slot).clamp(min=0)
    live = slot < (budget + e).unsqueeze(1)
    w, pos = s.mass.view(-1)[rows], torch.where(live, s.positions.view(-1)[rows].long(), -1)
    recent = torch.minimum(torch.tensor(c["recent"], device=dev), budget).unsqueeze(1)
    w = torch.where(pos >= s.next_position.long().repeat(layers * heads).unsqueeze(1) - recent, math.inf, w)
    order = torch.where(live, w, -1.0).sort(dim=1, descending=True, stable=True).indices
    kept = torch.zeros_like(live).scatter_(1, order, slot < budget.unsqueeze(1))
    # the j-th hole among the first `budget` slots takes the j-th token that is kept behind them
    front = slot < budget.unsqueeze(1)
    holes, movers = live & front & ~kept, live & ~front & kept
    to, frm = rows[holes], rows[movers]                                         # both unit by unit, ascending
    for_all = (s.k_pages.view(-1, D), s.v_pages.view(-1, D), s.mass.view(-1), s.positions.view(-1))
    k, v, m, p = (x[frm] for x in for_all)
    for_all[0][to], for_all[1][to], for_all[2][to], for_all[3][to] = k, v, m, p
    s.lengths_out.copy_(s.budgets)


def run(s):
    c = s.case
    if own:
        from paper_2507_08143_b200 import binding as B
        if c["op"] == "attention":
            if c["append"]:
                B.paged_attention(s.cache, 0, s.opt, s.q, s.lengths, s.out, s.ws, k_new=s.k_new, v_new=s.v_new, new_positions=s.new_positions, lse_out=s.lse)
            else:
                B.paged_attention(s.cache, 0, s.opt, s.q, s.lengths, s.out, s.ws, lse_out=s.lse)
            return {"out": s.out, "lse": s.lse, "mass": s.mass, "positions": s.positions, "k_pages": s.k_pages, "v_pages": s.v_pages}
        if c["op"] == "fill":
            B.paged_fill(s.cache, s.shape, s.k, s.v, s.keep, idx=s.idx, head_offsets=s.head_offsets, mass_in=s.attn,
                         first_position=s.first_position, lengths_out=s.lengths_out)
        else:
            B.paged_fill(s.cache, s.shape, s.k_in, s.v_in, s.shape.seqlens, mass_in=s.mass_in, first_position=s.next_position, lengths=s.budgets)
            s.next_position += c["block"]
            B.paged_evict(s.cache, s.full, s.budgets, s.lengths_out, s.max_length, recent=c["recent"], next_position=s.next_position)
    elif c["op"] == "attention":
        return _plain_attention(s)
    elif c["op"] == "fill":
        _plain_fill(s)
    else:
        _plain_evict(s)
    return {"k_pages": s.k_pages, "v_pages": s.v_pages, "mass": s.mass, "positions": s.positions, "lengths": s.lengths_out}


# --------------------------------------------------------------------------------------------- exact values
def exact(case, seed):
    """The attention's values in 64 bits, unit by unit; the other operators only copy."""
    if case["op"] != "attention":
        return None
    s = prepare(case, seed)
    page, heads, g, batch = case["page"], case["heads"], case["g"], case["batch"]
    out = torch.zeros(batch, heads * g, D, dtype=torch.float64, device="cuda")
    lse = torch.full((batch, heads * g), -math.inf, dtype=torch.float64, device="cuda")
    mass = s.mass.double()
    for h in range(heads):
        for b in range(batch):
            n = s.lens[b]
            if n < 0 or n + case["append"] == 0:
                continue
            used = s.table[0, h, b, : (n + page) // page].long()
            k = s.k_pages[used].reshape(-1, D)[:n].double()
            v = s.v_pages[used].reshape(-1, D)[:n].double()
            if case["append"]:
                k, v = torch.cat([k, s.k_new[b, h][None].double()]), torch.cat([v, s.v_new[b, h][None].double()])
            q = s.q[b, h * g:(h + 1) * g].double()
            y = torch.einsum("gd,nd->gn", q, k) / math.sqrt(D)
            if case["softcap"]:
                y = case["softcap"] * torch.tanh(y / case["softcap"])
            lse[b, h * g:(h + 1) * g] = torch.logsumexp(y, 1)
            p = torch.softmax(y, 1)
            out[b, h * g:(h + 1) * g] = p @ v
            slots = torch.arange(p.shape[1], device="cuda")
            if case["append"]:
                mass[used[n // page], n % page] = 0
            if case["accumulate"]:
                mass[used[slots // page], slots % page] += p.sum(0)
    return {"out": out, "lse": lse, "mass": mass, "positions": None, "k_pages": None, "v_pages": None}
