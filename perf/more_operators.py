"""What a program with a long cache in pages asks of this framework: which parts of the cache a token reads, and which entries of it stay.

  bound    smallest and largest key element of every block of entries, kept up as entries are appended
  choose   the blocks that a token reads: by the largest logit that their bounds allow any head of the group
  attend   attention of a token over the entries of its chosen blocks alone, joined with another part or not
  weigh    the attention weight that every entry received, summed over tokens and the heads of its group
  evict    the entries that stay by these weights, beside the newest and the first, with their rows moved together

`own` false: elementary torch operations in 32 bits (scores that rank blocks in 64), rounded once at the end.  `own` true: the
framework's calls.
"""
import math

import torch

own = False

DEVICE = "cuda:0"


def _bound(name, seqs, tokens, kv_heads, dim, dtype, page, start, block):
    return {"name": name, "kind": "bound", "seqs": seqs, "tokens": tokens, "kv_heads": kv_heads, "dim": dim, "dtype": dtype,
            "page": page, "start": start, "block": block}


def _choose(name, seqs, tokens, q_heads, kv_heads, dim, dtype, length, block, chosen, sees):
    return {"name": name, "kind": "choose", "seqs": seqs, "tokens": tokens, "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim,
            "dtype": dtype, "length": length, "block": block, "chosen": chosen, "sees": sees, "first": 1, "last": 2}


def _attend(name, seqs, tokens, q_heads, kv_heads, dim, dtype, page, length, block, chosen, sees, joined):
    return {"name": name, "kind": "attend", "seqs": seqs, "tokens": tokens, "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim,
            "dtype": dtype, "page": page, "length": length, "block": block, "chosen": chosen, "sees": sees, "joined": joined}


def _weigh(name, seqs, tokens, q_heads, kv_heads, dim, dtype, page, length, sees, known, decay):
    return {"name": name, "kind": "weigh", "seqs": seqs, "tokens": tokens, "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim,
            "dtype": dtype, "page": page, "length": length, "sees": sees, "known": known, "decay": decay}


def _evict(name, seqs, kv_heads, dim, dtype, page, length, keep, recent, first, positions, ragged, ties):
    return {"name": name, "kind": "evict", "seqs": seqs, "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "page": page,
            "length": length, "keep": keep, "recent": recent, "first": first, "positions": positions, "ragged": ragged, "ties": ties}


def listed():
    return [
        # a decode step of the benchmark's batch: one new key of each sequence extends its block's bounds
        _bound("bound_step", 32, 1, 4, 128, "bf16", 16, 2055, 64),
        # a long prompt's keys, once
        _bound("bound_prompt", 1, 16384, 8, 128, "bf16", 64, 0, 64),
        # a decode step of the larger model's batch, every sequence with a whole book of its own behind it
        _choose("choose_step", 16, 1, 40, 8, 128, "bf16", 100003, 32, 64, "all"),
        # a stretch of new tokens after a long context, each sees its past
        _choose("choose_chunk", 1, 640, 28, 4, 128, "bf16", 32768, 64, 32, "past"),
        # a checking program's fp32 rows of 64, tokens that see a part or nothing
        _choose("choose_fp32", 3, 33, 32, 8, 64, "fp32", 5001, 16, 20, "some"),
        # a decode step over 2048 chosen entries of every sequence
        _attend("attend_step", 16, 1, 40, 8, 128, "bf16", 64, 32768, 32, 64, "all", False),
        # a stretch of new tokens, each over the blocks of its own choice
        _attend("attend_chunk", 1, 640, 28, 4, 128, "bf16", 32, 32768, 64, 32, "past", False),
        # fp32 rows of 64 in pages that end inside blocks, joined with what the tokens found elsewhere
        _attend("attend_fp32", 3, 5, 32, 8, 64, "fp32", 24, 701, 16, 20, "some", True),
        # a decode step's weights added to those before, older steps counting less
        _weigh("weigh_step", 16, 1, 40, 8, 128, "bf16", 64, 32768, "all", 32767, 0.99),
        # what a long prompt's entries received from the prompt itself
        _weigh("weigh_prompt", 1, 4096, 40, 8, 128, "bf16", 128, 4096, "past", 0, 1.0),
        # the benchmark's batch at the end of a window: 64 entries beyond the budget go
        _evict("evict_step", 32, 4, 128, "bf16", 16, 2112, 2048, 64, 4, True, False, False),
        # a long prompt brought down to the larger model's budget, sequences of several lengths, many equal weights
        _evict("evict_prompt", 4, 8, 128, "bf16", 64, 32768, 4096, 256, 4, False, True, True),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["bound", "choose", "choose", "attend", "attend", "weigh", "weigh", "evict", "evict"])
    dim, dtype = rng.choice([(128, "bf16")] * 4 + [(64, "bf16"), (64, "fp32"), (128, "fp32")])
    width = dim * (4 if dtype == "fp32" else 2) / 256.0
    slow = 8.0 if dtype == "fp32" else 1.0
    kv_heads = rng.choice([1, 2, 3, 4, 6, 8])
    q_heads = kv_heads * rng.choice([1, 2, 3, 4, 5, 6, 7, 8, 8, 16])
    seqs = rng.choice([1, 1, 2, 4, 8, 16])
    page = rng.choice([16, 16, 24, 32, 64, 128, 256])
    block = rng.choice([16, 32, 32, 64, 64, 128])
    if kind == "bound":
        tokens = _log_int(rng, 1, int(16384 * 8 / (seqs * kv_heads * width)))
        return _bound("", seqs, tokens, kv_heads, dim, dtype, page, rng.choice([0, rng.randint(1, 3000)]), block)
    if kind == "evict":
        length = _log_int(rng, 200, max(201, min(100003, int(4 * 8 * 32768 / (seqs * kv_heads * width)))))
        keep = max(1, min(length - 1, int(length * rng.choice([0.97, 0.5, 0.25, 0.1]))))
        recent = min(keep // 2, rng.choice([0, 1, 64, 256]))
        return _evict("", seqs, kv_heads, dim, dtype, page, length, keep, recent, min(keep - recent, rng.choice([0, 4])),
                      rng.random() < 0.5, rng.random() < 0.4, rng.random() < 0.4)
    many = rng.random() < 0.4
    if kind == "choose":
        seqs = min(seqs, 2) if many else seqs
        tokens = _log_int(rng, 33, 640) if many else rng.choice([1, 1, 1, 2, 5])
        most = min(100003 * 16 * 8 * block / 32 / (seqs * kv_heads * width), 2e9 * block / (slow * seqs * tokens * q_heads * dim))
        length = max(_log_int(rng, 300, max(301, min(262144, int(most)))), tokens)
        chosen = max(4, min(_log_int(rng, 4, 128), length // block))
        return _choose("", seqs, tokens, q_heads, kv_heads, dim, dtype, length, block, chosen, rng.choice(["all", "past", "some"]))
    if kind == "attend":
        seqs = min(seqs, 2) if many else seqs
        tokens = _log_int(rng, 33, 640) if many else rng.choice([1, 1, 1, 2, 5])
        length = max(_log_int(rng, 300, min(100003, int(16 * 8 * 32768 / (seqs * kv_heads * width)))), tokens)
        most = min(16 * 8 * 2048.0 / (seqs * tokens * kv_heads * width) if not many else 4096.0, 9e9 / (slow * seqs * tokens * q_heads * dim))
        chosen = max(1, min(_log_int(rng, 4, 256), length // block + 1, int(most / block)))
        return _attend("", seqs, tokens, q_heads, kv_heads, dim, dtype, page, length, block, chosen, rng.choice(["all", "past", "some"]),
                       rng.random() < 0.5)
    if many:
        seqs = min(seqs, 2)
        room = 40 * 4096.0 ** 2 / 2 / slow / (seqs * q_heads)
        tokens = _log_int(rng, 100, max(101, min(4096, int(math.sqrt(room)))))
        length = max(tokens, _log_int(rng, 100, max(101, min(16384, int(room / tokens)))))
        sees = rng.choice(["past", "past", "all"])
    else:
        tokens = rng.choice([1, 1, 1, 2, 5])
        most = min(16 * 8 * 32768 / (seqs * kv_heads * width), 16 * 40 * 32768 / (slow * seqs * tokens * q_heads))
        length = _log_int(rng, 100, max(101, min(262144, int(most))))
        sees = rng.choice(["all", "past", "some"]) if length >= tokens else "all"
    return _weigh("", seqs, tokens, q_heads, kv_heads, dim, dtype, page, length, sees, rng.choice([0, length - 1, rng.randint(0, length)]),
                  rng.choice([1.0, 0.99, 0.5]))


# ------------------------------------------------------------------------------------ inputs

def _dtype(case):
    return torch.float32 if case["dtype"] == "fp32" else torch.bfloat16


def _blocks(case):
    return (case["length"] + case["block"] - 1) // case["block"]


def _inputs(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    kind, dt, S, H, d = case["kind"], _dtype(case), case["seqs"], case["kv_heads"], case["dim"]

    def normal(*shape):
        return torch.empty(shape, device=DEVICE).normal_(generator=gen)

    def uniform(lo, hi, *shape):
        return torch.randint(lo, hi, shape, generator=gen, device=DEVICE)

    state = {"case": case}
    T, Hq = case.get("tokens"), case.get("q_heads")
    length = case["start"] + T if kind == "bound" else case["length"]
    if kind != "choose":
        page = case["page"]
        per_seq = (length + page - 1) // page
        n_pages = S * per_seq + 3
        state["table"] = torch.randperm(n_pages, generator=gen, device=DEVICE)[:S * per_seq].view(S, per_seq).to(torch.int32)
        # neighbouring entries are alike, as the parts of a text are
        drift = 0.7 * normal(n_pages, H, 1, d)
        state["k_pages"] = (normal(n_pages, H, page, d) + drift).to(dt)
        state["v_pages"] = normal(n_pages, H, page, d).to(dt)
    if kind in ("choose", "attend", "weigh"):
        state["visible"] = None
        if case["sees"] == "past":                 # the last tokens of the cache
            state["visible"] = torch.arange(length - T + 1, length + 1, dtype=torch.int32, device=DEVICE).expand(S, T).contiguous()
        if case["sees"] == "some":
            vis = uniform(0, length + 1, S, T).to(torch.int32)
            vis[:, ::7] = 0 if T > 1 else length // 2
            state["visible"] = vis
    if kind == "bound":
        block = case["block"]
        n_blocks = (length + block - 1) // block + 2
        state["bounds"] = normal(S, H, n_blocks, 2, d).to(dt)   # (what no entry has been counted in yet)
        if case["start"]:
            _plain_bound(state["k_pages"], state["table"], state["bounds"], 0, case["start"], block)
    if kind == "choose":
        n_blocks, G = _blocks(case), Hq // H
        middle = 0.8 * normal(S, H, n_blocks, d)
        state["bounds"] = torch.stack((middle - (2.0 + 0.4 * normal(S, H, n_blocks, d)).abs(),
                                       middle + (2.0 + 0.4 * normal(S, H, n_blocks, d)).abs()), 3).to(dt)
        # tokens look for something, neighbours for the like
        common = 0.5 * normal(S, 1, H, 1, d) + 0.5 * middle[:, :, :1, None].transpose(1, 2)
        state["q"] = (normal(S, T, H, G, d) + common).view(S, T, Hq, d).to(dt)
    if kind == "attend":
        n_blocks = _blocks(case)
        liked = normal(S, 1, H, n_blocks) + 0.5 * normal(S, T, H, n_blocks)
        seen = torch.full((S, T), length, device=DEVICE) if state["visible"] is None else state["visible"].long()
        first = min(1, case["chosen"] - 1)
        state["blocks"] = _listed_blocks(liked, (seen + case["block"] - 1) // case["block"], case["chosen"], first, 1)
        state["q"] = (1.3 * normal(S, T, Hq, d)).to(dt)
        state["joined"] = None
        if case["joined"]:                         # what the tokens found elsewhere
            state["joined"] = ((0.2 * normal(S, T, Hq, d)).to(dt), math.log(case["chosen"] * case["block"]) + normal(S, T, Hq))
    if kind == "weigh":
        state["q"] = (1.3 * normal(S, T, Hq, d)).to(dt)
        state["lse"] = _plain_lse(state["q"], state["k_pages"], state["table"], length, state["visible"])
        state["old"] = (normal(S, H, length + 5) - 2.0).exp()
        state["weights"] = torch.zeros((S, H, length + 5), device=DEVICE)
    if kind == "evict":
        weights = (2.0 * normal(S, H, length) - 4.0).exp()
        if case["ties"]:                           # sums of few weights above a threshold: many are alike
            weights = torch.floor(4.0 * weights) / 4.0
        state["weights"], state["positions"], state["lengths"] = weights, None, None
        if case["positions"]:                      # what stayed of a longer text stands in no order, the newest entries at the end
            old = torch.rand((S, H, length), generator=gen, device=DEVICE).argsort(-1).to(torch.int32) * 3
            tail = min(length, max(1, case["recent"]))
            old[..., length - tail:] = 3 * length + torch.arange(tail, dtype=torch.int32, device=DEVICE)
            state["positions"] = old
        if case["ragged"]:
            state["lengths"] = uniform(length // 4, length + 1, S).to(torch.int32)
            state["lengths"][0] = length
    return state


def prepare(case, seed):
    state = _inputs(case, seed)
    if own:
        from paper_2506_15969_amd import binding
        if "table" in state:                       # a layer's pages
            state["pages"] = binding.PagedCache(state["k_pages"], state["v_pages"], state["table"], n_q_heads=case.get("q_heads"))
        if "bounds" in state:                      # and the bounds of its blocks
            state["keys"] = binding.KeyBounds(state["bounds"], case["block"])
    return state


# ------------------------------------------------------------------------------------ plain forms

def _plain_bound(k_pages, table, bounds, start, n, block):
    S, H, _, _, d = bounds.shape
    page = k_pages.shape[2]
    first, end = start // block, start + n
    entry = torch.arange(first * block, end + (-end) % block, device=k_pages.device)
    here = ((entry >= start) & (entry < end))[:, None, None]
    at = entry.clamp(start, end - 1)
    k = k_pages[table[:, at // page].long(), :, at % page]                       # [S, entries, H, d]
    lo = k.masked_fill(~here, math.inf).view(S, -1, block, H, d).amin(2)
    hi = k.masked_fill(~here, -math.inf).view(S, -1, block, H, d).amax(2)
    new = torch.stack((lo, hi), 3).transpose(1, 2)                                # [S, H, blocks, 2, d]
    if start % block:                              # the first block had entries before
        new[:, :, 0, 0] = torch.minimum(new[:, :, 0, 0], bounds[:, :, first, 0])
        new[:, :, 0, 1] = torch.maximum(new[:, :, 0, 1], bounds[:, :, first, 1])
    bounds[:, :, first:first + new.shape[2]] = new
    return bounds


def _listed_blocks(score, n_seen, chosen, first, last):
    """The blocks that tokens read, [S, T, H, chosen]: of n_seen [S, T] blocks all, or the first, the last and those with the
    highest of the scores [S, T, H, blocks], equal ones the lowest first."""
    n = score.shape[-1]
    number = torch.arange(n, device=score.device)
    n_seen = n_seen[:, :, None, None]
    between = ((number >= first) & (number < n_seen - last)).expand(score.shape)
    order = torch.sort(score.nan_to_num(nan=math.inf, posinf=math.inf, neginf=-math.inf), dim=-1, descending=True, stable=True).indices
    rank = torch.sort(between.gather(-1, order).to(torch.int32), dim=-1, descending=True, stable=True).indices
    best = order.gather(-1, rank)[..., :chosen - first - last]
    taken = (number < n_seen) & ~between
    taken = taken.scatter(-1, best, True) & (number < n_seen)
    taken = torch.where(n_seen <= chosen, (number < n_seen).expand(score.shape), taken)
    blocks = torch.sort(torch.where(taken, number, n), dim=-1).values[..., :chosen]
    blocks = torch.nn.functional.pad(blocks, (0, chosen - blocks.shape[-1]), value=n)
    return torch.where(blocks < n, blocks, -1).to(torch.int32)


def _plain_choose(q, bounds, n_seen, chosen, first, last):
    S, T, Hq, d = q.shape
    H, n = bounds.shape[1:3]
    rows = q.double().view(S, T, H, Hq // H, d).transpose(1, 2).reshape(S, H, -1, d)
    lo, hi = (x.double().transpose(2, 3).contiguous() for x in bounds.unbind(3))
    score = torch.matmul(rows.clamp(min=0.0), hi) + torch.matmul(rows.clamp(max=0.0), lo)
    score = score.view(S, H, T, Hq // H, n).amax(3).transpose(1, 2)
    return _listed_blocks(score, n_seen, chosen, first, last)


def _plain_attend(q, k_pages, v_pages, table, blocks, block, length, visible, joined):
    S, T, Hq, d = q.shape
    H, page = k_pages.shape[1:3]
    G = Hq // H
    out = torch.zeros((S * T, Hq, d), device=q.device)
    lse = torch.zeros((S * T, Hq), device=q.device)
    head = torch.arange(H, device=q.device)[:, None]
    seq = torch.arange(S, device=q.device).repeat_interleave(T)
    step = max(1, 2 ** 28 // (H * blocks.shape[-1] * block * d))
    for t in range(0, S * T, step):
        mine, its = blocks.flatten(0, 1)[t:t + step].long(), seq[t:t + step, None, None]
        entry = (mine[..., None] * block + torch.arange(block, device=q.device)).flatten(2)              # [t, H, entries]
        there = entry >= 0
        there &= entry < (length if visible is None else visible.flatten()[t:t + step, None, None])
        entry = entry.clamp(0, length - 1)
        at = table.long()[its, entry // page]
        k, v = (x[at, head, entry % page].float() for x in (k_pages, v_pages))                            # [t, H, entries, d]
        rows = q.flatten(0, 1)[t:t + step].float().view(-1, H, G, d)
        logits = torch.matmul(rows, k.transpose(2, 3).contiguous()) * (1.0 / math.sqrt(d))
        logits.masked_fill_(~there[:, :, None], -math.inf)
        top = logits.amax(-1, keepdim=True)
        weights = (logits - top.clamp(min=-1e30)).exp_()
        total = weights.sum(-1, keepdim=True)
        out[t:t + step] = (torch.matmul(weights, v) / total.clamp(min=1e-30)).flatten(1, 2)
        lse[t:t + step] = (top + total.log()).flatten(1)
    out, lse = out.view(S, T, Hq, d), lse.view(S, T, Hq)
    if joined is not None:
        both = torch.logaddexp(lse, joined[1])
        out = out * (lse - both).exp()[..., None] + joined[0].float() * (joined[1] - both).exp()[..., None]
        lse = both
    return out.to(q.dtype), lse


def _plain_logits(q, k_pages, table, length, visible):
    """(sequences, their scaled logits [., H, T * G, length], -inf where a token does not see the entry), some sequences at a time."""
    S, T, Hq, d = q.shape
    H = k_pages.shape[1]
    G = Hq // H
    step = max(1, 2 ** 30 // (H * length * max(T * G, d)))
    for s in range(0, S, step):
        k = k_pages[table[s:s + step].long()].transpose(1, 2).flatten(2, 3)[:, :, :length].float()
        rows = q[s:s + step].float().view(-1, T, H, G, d).transpose(1, 2).reshape(-1, H, T * G, d)
        logits = torch.matmul(rows, k.transpose(2, 3).contiguous()) * (1.0 / math.sqrt(d))
        if visible is not None:
            hidden = torch.arange(length, device=q.device) >= visible[s:s + step].repeat_interleave(G, 1)[:, None, :, None]
            logits.masked_fill_(hidden, -math.inf)
        yield slice(s, s + step), logits


def _by_head(x, H):
    """Numbers of tokens and query heads [S, T, Hq] as [S, H, T * G]."""
    S, T, Hq = x.shape
    return x.view(S, T, H, Hq // H).transpose(1, 2).reshape(S, H, -1)


def _plain_lse(q, k_pages, table, length, visible):
    S, T, Hq, _ = q.shape
    H = k_pages.shape[1]
    lse = torch.empty((S, H, T * (Hq // H)), device=q.device)
    for s, logits in _plain_logits(q, k_pages, table, length, visible):
        top = logits.amax(-1, keepdim=True).clamp(min=-1e30)
        lse[s] = (top + (logits - top).exp_().sum(-1, keepdim=True).log())[..., 0]
    return lse.view(S, H, T, -1).transpose(1, 2).reshape(S, T, Hq)


def _plain_weigh(q, lse, k_pages, table, length, visible, old, known, decay, weights):
    by_head = _by_head(lse, k_pages.shape[1])[..., None]
    for s, logits in _plain_logits(q, k_pages, table, length, visible):
        its = by_head[s]
        got = (logits - its).masked_fill_(its == -math.inf, -math.inf).exp_().sum(2)
        got[:, :, :known] += decay * old[s, :, :known]
        weights[s, :, :length] = got
    return weights


def _plain_evict(state, case):
    weights, length, keep = state["weights"], case["length"], case["keep"]
    S, H, _ = weights.shape
    page = case["page"]
    place = torch.arange(length, device=weights.device)
    position = place.to(torch.int32).expand(S, H, length) if state["positions"] is None else state["positions"]
    lengths = torch.full((S,), length, device=weights.device) if state["lengths"] is None else state["lengths"].long()
    there = (place < lengths[:, None])[:, None].expand(S, H, length)
    newest = torch.where(there, position, -1).amax(-1, keepdim=True)
    safe = there & ((position > newest - case["recent"]) | (position < case["first"]))
    # by weight, the safe ones before the others, what is no entry behind all; equal ones in their order
    order = torch.sort(weights, dim=-1, descending=True, stable=True).indices
    class_ = there.to(torch.int32) + safe
    order = order.gather(-1, torch.sort(class_.gather(-1, order), dim=-1, descending=True, stable=True).indices)
    by_place = torch.sort(class_, dim=-1, descending=True, stable=True).indices                         # (safe ones: in their order)
    n_safe = safe.sum(-1, keepdim=True)
    order = torch.where(place < n_safe, by_place, order)
    stays = torch.zeros_like(there).scatter(-1, order[..., :keep], True) & there
    # kept entries from `keep` on, in their order, go to the places below it that became free
    low, high = stays[..., :keep], stays[..., keep:]
    free = torch.sort((~low).to(torch.int32), dim=-1, descending=True, stable=True).indices             # free places first
    late = torch.sort(high.to(torch.int32), dim=-1, descending=True, stable=True).indices + keep        # kept late entries first
    n_moved = high.sum(-1, keepdim=True)
    source = torch.where(low, place[:keep], -1)
    nth = place[:keep].expand(S, H, keep)
    late = torch.nn.functional.pad(late, (0, max(0, keep - late.shape[-1])), value=-1)[..., :keep]
    source.scatter_(-1, free, torch.where(nth < n_moved, late, source.gather(-1, free)))
    moved = source > place[:keep]
    s, h, to = moved.nonzero(as_tuple=True)
    come = source[s, h, to]
    for x in (state["k_pages"], state["v_pages"]):
        x[state["table"][s, to // page].long(), h, to % page] = x[state["table"][s, come // page].long(), h, come % page]
    at = source.clamp(min=0)
    return {"sources": source.to(torch.int32), "weights": torch.where(source >= 0, weights.gather(-1, at), 0.0),
            "positions": torch.where(source >= 0, position.gather(-1, at), -1).to(torch.int32)}


def run(state):
    case = state["case"]
    kind = case["kind"]
    if kind == "bound":
        if own:
            state["keys"].update(state["pages"], case["start"], case["tokens"])
        else:
            _plain_bound(state["k_pages"], state["table"], state["bounds"], case["start"], case["tokens"], case["block"])
        return {"bounds": state["bounds"]}
    if kind == "choose":
        if own:
            blocks = state["keys"].choose(case["length"], state["q"], case["chosen"], visible=state["visible"], first=case["first"],
                                          last=case["last"])
        else:
            seen = torch.full(state["q"].shape[:2], case["length"], device=DEVICE) if state["visible"] is None else state["visible"].long()
            blocks = _plain_choose(state["q"], state["bounds"], (seen + case["block"] - 1) // case["block"], case["chosen"], case["first"],
                                   case["last"])
        return {"blocks": blocks}
    if kind == "attend":
        if own:
            out, lse = state["pages"].attend_blocks(case["length"], state["q"], state["blocks"], case["block"], visible=state["visible"],
                                                    joined=state["joined"])
        else:
            out, lse = _plain_attend(state["q"], state["k_pages"], state["v_pages"], state["table"], state["blocks"], case["block"],
                                     case["length"], state["visible"], state["joined"])
        return {"out": out, "lse": lse}
    if kind == "weigh":
        if own:
            weights = state["pages"].weigh(case["length"], state["q"], state["lse"].contiguous(), visible=state["visible"], old=state["old"],
                                           known=case["known"], decay=case["decay"], weights=state["weights"])
        else:
            weights = _plain_weigh(state["q"], state["lse"], state["k_pages"], state["table"], case["length"], state["visible"],
                                   state["old"], case["known"], case["decay"], state["weights"])
        return {"weights": weights}
    if own:
        sources, weights, positions = state["pages"].evict(case["length"], state["weights"], case["keep"], recent=case["recent"],
                                                           first=case["first"], positions=state["positions"], lengths=state["lengths"])
        got = {"sources": sources, "weights": weights, "positions": positions}
    else:
        got = _plain_evict(state, case)
    got.update(k_pages=state["k_pages"], v_pages=state["v_pages"])
    return got


# ------------------------------------------------------------------------------------ 64 bits

def _exact_choose(case, state):
    """Row by row: the bound of every head's logit as a sum of maxima, and a pick of the best one after the other's border."""
    q, bounds = state["q"].double(), state["bounds"].double()
    S, T, Hq, d = q.shape
    H, n = bounds.shape[1:3]
    G = Hq // H
    blocks = torch.full((S, T, H, case["chosen"]), -1, dtype=torch.int32, device=q.device)
    for s in range(S):
        seen = [case["length"]] * T if state["visible"] is None else state["visible"][s].tolist()
        for h in range(H):
            lo, hi = bounds[s, h, :, 0], bounds[s, h, :, 1]
            step = max(1, 2 ** 26 // (G * n * d))
            for t0 in range(0, T, step):
                rows = q[s, t0:t0 + step, h * G:(h + 1) * G, None]
                score = torch.maximum(rows * lo, rows * hi).sum(-1).amax(1)
                for t in range(score.shape[0]):
                    m = -(-seen[t0 + t] // case["block"])
                    if m <= case["chosen"]:
                        mine = torch.arange(m, device=q.device)
                    else:
                        between = score[t, case["first"]:m - case["last"]]
                        best = torch.argsort(between, descending=True, stable=True)[:case["chosen"] - case["first"] - case["last"]]
                        mine = torch.cat((torch.arange(case["first"], device=q.device), best + case["first"],
                                          torch.arange(m - case["last"], m, device=q.device))).sort().values
                    blocks[s, t0 + t, h, :mine.numel()] = mine.to(torch.int32)
    return {"blocks": blocks}


def _exact_attend(case, state):
    q, page, block, length = state["q"].double(), case["page"], case["block"], case["length"]
    S, T, Hq, d = q.shape
    H = case["kv_heads"]
    G = Hq // H
    out = torch.zeros((S, T, Hq, d), dtype=torch.float64, device=q.device)
    lse = torch.zeros((S, T, Hq), dtype=torch.float64, device=q.device)
    for s in range(S):
        for h in range(H):
            k, v = (state[x][state["table"][s].long(), h].flatten(0, 1)[:length].double() for x in ("k_pages", "v_pages"))
            for t in range(T):
                end = length if state["visible"] is None else int(state["visible"][s, t])
                mine = state["blocks"][s, t, h].tolist()
                entries = [torch.arange(b * block, min((b + 1) * block, end), device=q.device) for b in mine if 0 <= b * block < end]
                if not entries:
                    lse[s, t, h * G:(h + 1) * G] = -math.inf
                    continue
                at = torch.cat(entries)
                logits = q[s, t, h * G:(h + 1) * G] @ k[at].T.contiguous() / d ** 0.5
                whole = torch.logsumexp(logits, 1)
                lse[s, t, h * G:(h + 1) * G] = whole
                out[s, t, h * G:(h + 1) * G] = torch.exp(logits - whole[:, None]) @ v[at]
    if state["joined"] is not None:
        found, its = state["joined"][0].double(), state["joined"][1].double()
        share = torch.sigmoid(lse - its)[..., None]
        out, lse = share * out + (1.0 - share) * found, torch.logaddexp(lse, its)
    return {"out": out, "lse": lse}


def _exact_weigh(case, state):
    q, lse, length, page = state["q"].double(), state["lse"].double(), case["length"], case["page"]
    S, T, Hq, d = q.shape
    G = Hq // case["kv_heads"]
    weights = state["weights"].double()
    entry = torch.arange(length, device=q.device)
    for s in range(S):
        at = state["table"][s].long()[entry // page]
        for h in range(case["kv_heads"]):
            k = state["k_pages"][at, h, entry % page].double()
            sum_ = torch.zeros(length, dtype=torch.float64, device=q.device)
            for g in range(h * G, (h + 1) * G):
                for t0 in range(0, T, 1024):
                    share = torch.exp(q[s, t0:t0 + 1024, g] @ k.T.contiguous() / d ** 0.5 - lse[s, t0:t0 + 1024, g, None])
                    if state["visible"] is not None:
                        share = torch.where(entry < state["visible"][s, t0:t0 + 1024, None], share, 0.0)
                    sum_ += share.sum(0)
            sum_[:case["known"]] += float(torch.tensor(case["decay"])) * state["old"][s, h, :case["known"]].double()
            weights[s, h, :length] = sum_
    return {"weights": weights}


def _exact_evict(case, state):
    """Unit by unit on the host: a sort of tuples, then the moves one after the other."""
    import numpy as np
    weights, keep, page = state["weights"].cpu().numpy(), case["keep"], case["page"]
    S, H, length = weights.shape
    positions = None if state["positions"] is None else state["positions"].cpu().numpy()
    sources, to_w, to_p = np.full((S, H, keep), -1, np.int32), np.zeros((S, H, keep), np.float64), np.full((S, H, keep), -1, np.int32)
    pools = {x: state[x].double() for x in ("k_pages", "v_pages")}
    table = state["table"].cpu().numpy()
    for s in range(S):
        n = length if state["lengths"] is None else int(state["lengths"][s])
        for h in range(H):
            position = np.arange(n) if positions is None else positions[s, h, :n]
            newest = position.max() if n else 0
            safe = (position > newest - case["recent"]) | (position < case["first"])
            rank = np.lexsort((np.arange(n), np.where(safe, 0.0, -weights[s, h, :n].astype(np.float64)), ~safe))
            stays = np.zeros(n, bool)
            stays[rank[:keep]] = True
            source = np.where(stays[:keep], np.arange(min(n, keep)), -1)
            free, late = np.flatnonzero(~stays[:keep]), keep + np.flatnonzero(stays[keep:])
            source[free[:len(late)]] = late
            sources[s, h, :len(source)] = source
            to_w[s, h, :len(source)], to_p[s, h, :len(source)] = weights[s, h, source], position[source]
            to = torch.tensor(free[:len(late)], device=DEVICE)
            come = torch.tensor(late, device=DEVICE)
            row = torch.tensor(table[s].astype(np.int64), device=DEVICE)
            for x in pools.values():
                x[row[to // page], h, to % page] = x[row[come // page], h, come % page]
    return {"sources": torch.tensor(sources, device=DEVICE), "weights": torch.tensor(to_w, device=DEVICE),
            "positions": torch.tensor(to_p, device=DEVICE), **pools}


def exact(case, seed):
    state = _inputs(case, seed)
    if case["kind"] == "bound":
        bounds, block, start = state["bounds"].double(), case["block"], case["start"]
        end = start + case["tokens"]
        for s in range(case["seqs"]):
            at = state["table"][s].long()
            for b in range(start // block, (end + block - 1) // block):
                entry = torch.arange(max(start, b * block), min(end, (b + 1) * block), device=DEVICE)
                k = state["k_pages"][at[entry // case["page"]], :, entry % case["page"]].double()
                lo, hi = k.min(0).values, k.max(0).values
                if b * block < start:
                    lo, hi = torch.minimum(lo, bounds[s, :, b, 0]), torch.maximum(hi, bounds[s, :, b, 1])
                bounds[s, :, b, 0], bounds[s, :, b, 1] = lo, hi
        return {"bounds": bounds}
    return {"choose": _exact_choose, "attend": _exact_attend, "weigh": _exact_weigh, "evict": _exact_evict}[case["kind"]](case, state)


def work(case):
    S, H, d = case["seqs"], case["kv_heads"], case["dim"]
    size = 4 if case["dtype"] == "fp32" else 2
    row, kind = d * size, case["kind"]
    if kind == "bound":
        first, end = case["start"] // case["block"], case["start"] + case["tokens"]
        touched = (end + case["block"] - 1) // case["block"] - first
        known = 1 if case["start"] % case["block"] else 0
        return {"bytes": S * H * row * (case["tokens"] + 2 * touched + 2 * known), "flops": 2 * S * H * case["tokens"] * d}
    length = case["length"]
    if kind == "evict":
        keep, loose = case["keep"], max(1, length - case["recent"] - case["first"])
        rest = keep - case["recent"] - case["first"]
        moved = min(case["recent"], length - keep) + rest * max(0, length - keep - case["recent"]) / loose
        mean = 0.625 if case["ragged"] else 1.0    # (lengths from a quarter on)
        entry = 8 if case["positions"] else 4
        return {"bytes": int(S * H * (length * mean * entry + 12 * keep + mean * moved * 4 * row)), "flops": int(S * H * length * mean)}
    T, Hq = case["tokens"], case["q_heads"]
    rows = S * T * Hq
    seen = length - (T - 1) / 2 if case["sees"] == "past" else length / 2 if case["sees"] == "some" else length
    if kind == "choose":
        scored = max(0.0, seen / case["block"] - case["first"] - case["last"])
        return {"bytes": int(rows * row + S * H * _blocks(case) * 2 * row + 4 * S * T * H * case["chosen"]),
                "flops": int(2 * rows * scored * d)}
    if kind == "attend":
        read = min(case["chosen"] * case["block"], seen)
        union = min(length, T * read)
        moved = 2 * S * H * union * row + 4 * S * T * H * case["chosen"] + 2 * rows * row + 4 * rows
        if case["joined"]:
            moved += rows * (row + 4)
        return {"bytes": int(moved), "flops": int(4 * rows * d * read)}
    return {"bytes": int(S * H * length * (row + 4) + 4 * S * H * case["known"] + rows * (row + 4)), "flops": int(2 * rows * d * seen)}
