"""What stands around a decode step of this framework: rows made ready for it, a prefix kept in pages, and the
attention that reads those pages.

  rotate   norms of the query and key heads and the rotation by the token's position, in one pass
  append   keys (normed and rotated on the way) and values written into the pages of a cache
  attend   attention of the tokens that share a context over its pages: single tokens of a batch over
           their common prefix, joined with what they found in their own caches; a prompt over the prefix
           before it; a prompt over itself (every token sees the entries up to its own)

`own` false: elementary torch operations in 32 bits (angles in 64), rounded once at the end.  `own` true: the
framework's calls.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
EPS = 1e-6


def _rotate(name, seqs, tokens, q_heads, kv_heads, dim, dtype, layout, dims, norm, joint, far):
    return {"name": name, "kind": "rotate", "seqs": seqs, "tokens": tokens, "q_heads": q_heads, "kv_heads": kv_heads,
            "dim": dim, "dtype": dtype, "layout": layout, "dims": dims, "norm": norm, "joint": joint, "far": far}


def _append(name, seqs, tokens, kv_heads, dim, dtype, page, start, layout, dims, norm):
    return {"name": name, "kind": "append", "seqs": seqs, "tokens": tokens, "kv_heads": kv_heads, "dim": dim,
            "dtype": dtype, "page": page, "start": start, "layout": layout, "dims": dims, "norm": norm}


def _attend(name, seqs, tokens, q_heads, kv_heads, dim, dtype, page, length, sees, joined):
    return {"name": name, "kind": "attend", "seqs": seqs, "tokens": tokens, "q_heads": q_heads, "kv_heads": kv_heads,
            "dim": dim, "dtype": dtype, "page": page, "length": length, "sees": sees, "joined": joined}


def listed():
    return [
        # the rows of a decode step of the benchmark's batch: one token of each of 32 sequences, far into the generation
        _rotate("rotate_step", 1, 32, 28, 4, 128, "bf16", "halves", 128, True, False, 32768),
        # the prompts of a batch, queries and keys lying in one joint projection
        _rotate("rotate_prompts", 4, 2048, 40, 8, 128, "bf16", "halves", 128, True, True, 0),
        # a checking program's fp32 prompt: heads of 64, half of them rotated, neighbours as pairs, no norm
        _rotate("rotate_fp32_pairs", 3, 499, 32, 8, 64, "fp32", "pairs", 32, False, False, 0),
        # a prefix that grows by one token
        _append("append_one", 1, 1, 4, 128, "bf16", 16, 1000, "halves", 128, True),
        # a long shared prefix written at once
        _append("append_prefix", 1, 16384, 8, 128, "bf16", 64, 0, "halves", 128, True),
        # several contexts continued by a stretch that begins and ends inside a page
        _append("append_fp32", 4, 601, 8, 64, "fp32", 24, 77, "pairs", 64, False),
        # one user's token over a short prefix: as long as its latency
        _attend("attend_one", 1, 1, 28, 4, 128, "bf16", 16, 1003, "all", False),
        # the benchmark's batch over a common prefix, joined with the sequences' own caches
        _attend("attend_batch", 1, 32, 28, 4, 128, "bf16", 64, 8192, "all", True),
        # the larger model's batch over a whole book
        _attend("attend_book", 1, 16, 40, 8, 128, "bf16", 64, 100003, "all", True),
        # a prompt read after the prefix that it shares with others
        _attend("attend_prompt", 1, 640, 28, 4, 128, "bf16", 32, 4096, "all", False),
        # a long prompt's attention over itself
        _attend("attend_causal", 1, 4096, 40, 8, 128, "bf16", 128, 4096, "causal", False),
        # fp32 heads of 64, several contexts, tokens that see a part of it or nothing
        _attend("attend_fp32", 3, 33, 32, 8, 64, "fp32", 48, 701, "some", True),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["rotate", "append", "attend", "attend", "attend"])
    dim, dtype = rng.choice([(128, "bf16")] * 4 + [(64, "bf16"), (64, "fp32"), (128, "fp32")])
    width = dim * (4 if dtype == "fp32" else 2) / 256.0
    kv_heads = rng.choice([1, 2, 3, 4, 6, 8])
    layout = rng.choice(["halves", "halves", "pairs"])
    dims = rng.choice([dim, dim, dim // 2])
    norm = rng.random() < 0.7
    seqs = rng.choice([1, 1, 1, 2, 4])
    page = rng.choice([16, 16, 24, 32, 64, 128, 256])
    if kind == "rotate":
        q_heads = kv_heads * rng.randint(1, 8)
        tokens = _log_int(rng, 1, int(4 * 2048 * 48 / (seqs * (q_heads + kv_heads) * width)))
        return _rotate("", seqs, tokens, q_heads, kv_heads, dim, dtype, layout, dims, norm, rng.random() < 0.5,
                       rng.choice([0, 4096, 131072]))
    if kind == "append":
        tokens = _log_int(rng, 1, int(16384 * 8 / (seqs * kv_heads * width)))
        return _append("", seqs, tokens, kv_heads, dim, dtype, page, rng.choice([0, rng.randint(1, 2000)]), layout, dims, norm)
    group = rng.choice([1, 2, 3, 4, 5, 6, 7, 8, 8, 16])
    q_heads = kv_heads * group
    form = rng.choice(["tokens", "tokens", "prompt", "causal"])
    slow = 8.0 if dtype == "fp32" else 1.0
    if form == "tokens":
        tokens = _log_int(rng, 1, 48)
        most = min(100003 * 8 / (seqs * kv_heads * width), 16 * 40 * 100003 / slow / (seqs * tokens * q_heads))
        length = _log_int(rng, 100, max(101, int(most)))
        sees = rng.choice(["all", "all", "all", "some"])
    else:
        room = 40 * 4096.0 ** 2 / 2 / slow / (seqs * q_heads)
        tokens = _log_int(rng, 100, max(101, min(4096, int(math.sqrt(room)))))
        length = tokens if form == "causal" else _log_int(rng, 100, max(101, min(16384, int(room / tokens))))
        sees = "causal" if form == "causal" else "all"
    return _attend("", seqs, tokens, q_heads, kv_heads, dim, dtype, page, length, sees, form == "tokens" and rng.random() < 0.6)


# ------------------------------------------------------------------------------------ inputs

def _dtype(case):
    return torch.float32 if case["dtype"] == "fp32" else torch.bfloat16


def _inv_freq(dims):
    return torch.tensor([10000.0 ** (-2.0 * j / dims) for j in range(dims // 2)], dtype=torch.float32, device=DEVICE)


def _paged(dense, table, n_pages, page, gen):
    """Rows [S, T, H, d] in pages [n_pages, H, page, d] as the table says; what no row fills holds other numbers."""
    S, T, H, d = dense.shape
    pool = torch.empty((n_pages, H, page, d), device=DEVICE).normal_(generator=gen).to(dense.dtype)
    at = torch.arange(T, device=DEVICE)
    pages = table[:, at // page].long()
    pool[pages, :, (at % page).expand(S, T)] = dense
    return pool


def _inputs(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    dt, S, T, d, H = _dtype(case), case["seqs"], case["tokens"], case["dim"], case["kv_heads"]

    def normal(*shape):
        return torch.empty(shape, device=DEVICE).normal_(generator=gen)

    def weight():
        return (1.0 + 0.1 * normal(d)).to(dt)

    state = {"case": case}
    if case["kind"] == "rotate":
        Hq = case["q_heads"]
        if case["joint"]:                          # [query heads | key heads | value heads] of a token
            rows = normal(S, T, Hq + 2 * H, d).to(dt)
            state["q"], state["k"] = rows[:, :, :Hq], rows[:, :, Hq:Hq + H]
        else:
            state["q"], state["k"] = normal(S, T, Hq, d).to(dt), normal(S, T, H, d).to(dt)
        if case["far"]:                            # every token at a place of its own
            state["positions"] = torch.randint(0, case["far"], (S, T), generator=gen, device=DEVICE).to(torch.int32)
        else:
            state["positions"] = torch.arange(T, dtype=torch.int32, device=DEVICE).expand(S, T).contiguous()
        state["q_weight"], state["k_weight"] = (weight(), weight()) if case["norm"] else (None, None)
    if case["kind"] == "append":
        state["k"], state["v"] = normal(S, T, H, d).to(dt), normal(S, T, H, d).to(dt)
        state["q_weight"], state["k_weight"] = None, weight() if case["norm"] else None
    if case["kind"] in ("rotate", "append"):
        state["inv_freq"] = _inv_freq(case["dims"])
    if case["kind"] in ("append", "attend"):
        page = case["page"]
        length = case["length"] if case["kind"] == "attend" else case["start"] + T
        per_seq = (length + page - 1) // page
        n_pages = S * per_seq + 3
        table = torch.randperm(n_pages, generator=gen, device=DEVICE)[:S * per_seq].view(S, per_seq).to(torch.int32)
        state["table"] = table
        if case["kind"] == "append":
            state["k_pages"], state["v_pages"] = (normal(n_pages, H, page, d).to(dt) for _ in range(2))
        else:
            Hq, G = case["q_heads"], case["q_heads"] // H
            k, v = normal(S, length, H, d).to(dt), normal(S, length, H, d).to(dt)
            # every query reads the first entry, and one more of its own
            read = torch.randint(0, length, (S, T), generator=gen, device=DEVICE)
            seen = torch.stack([k[s][read[s]] for s in range(S)]).float()
            q = normal(S, T, H, G, d) + 0.25 * k[:, :1, :, None].float() + 0.5 * seen[:, :, :, None]
            state["q"] = q.view(S, T, Hq, d).to(dt)
            state["k_pages"], state["v_pages"] = (_paged(x, table, n_pages, page, gen) for x in (k, v))
            state["visible"] = None
            if case["sees"] == "causal":
                state["visible"] = torch.arange(1, T + 1, dtype=torch.int32, device=DEVICE).expand(S, T).contiguous()
            if case["sees"] == "some":
                vis = torch.randint(0, length + 1, (S, T), generator=gen, device=DEVICE).to(torch.int32)
                vis[:, ::7] = 0
                state["visible"] = vis
            state["joined"] = None
            if case["joined"]:                     # what the tokens found in their own caches
                state["joined"] = ((0.2 * normal(S, T, Hq, d)).to(dt), math.log(length) + normal(S, T, Hq))
    return state


def prepare(case, seed):
    state = _inputs(case, seed)
    if own:
        from paper_2506_15969_amd import binding
        if "inv_freq" in state:                    # a layer's norms and rotation
            layout = binding.ROPE_HALVES if case["layout"] == "halves" else binding.ROPE_PAIRS
            state["rope"] = binding.NormRope(case["dim"], _dtype(case), q_weight=state["q_weight"], k_weight=state["k_weight"],
                                             eps=EPS, inv_freq=state["inv_freq"], layout=layout)
        if "table" in state:                       # a layer's pages
            state["pages"] = binding.PagedCache(state["k_pages"], state["v_pages"], state["table"],
                                                n_q_heads=case.get("q_heads"))
    return state


# ------------------------------------------------------------------------------------ plain forms

def _turned(x, positions, weight, inv_freq, layout):
    """The heads x [S, T, H, d] normed (where there is a weight) and rotated, in 32 bits."""
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()
    angle = positions.double()[:, :, None, None] * inv_freq.double()
    cos, sin = angle.cos().float(), angle.sin().float()
    r = 2 * inv_freq.numel()
    if layout == "halves":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    else:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    return torch.cat((turned, x[..., r:]), -1)


def _plain_attend(q, k_pages, v_pages, table, length, visible, joined):
    S, T, Hq, d = q.shape
    n_pages, H, page, _ = k_pages.shape
    G = Hq // H
    k, v = (x[table.long()].transpose(1, 2).reshape(S, H, -1, d)[:, :, :length].float() for x in (k_pages, v_pages))
    rows = q.float().view(S, T, H, G, d).transpose(1, 2).reshape(S, H, T * G, d)
    logits = torch.matmul(rows, k.transpose(2, 3).contiguous()) * (1.0 / math.sqrt(d))
    if visible is not None:
        hidden = torch.arange(length, device=q.device) >= visible.repeat_interleave(G, 1)[:, None, :, None]
        logits.masked_fill_(hidden, -math.inf)
    top = logits.amax(-1, keepdim=True)
    weights = (logits - top.clamp(min=-1e30)).exp_()
    total = weights.sum(-1, keepdim=True)
    out = torch.matmul(weights, v) / total.clamp(min=1e-30)
    lse = top + total.log()

    def by_token(x):
        return x.view(S, H, T, G, -1).transpose(1, 2).reshape(S, T, Hq, -1)
    out, lse = by_token(out), by_token(lse)[..., 0]
    if joined is not None:
        both = torch.logaddexp(lse, joined[1])
        out = out * (lse - both).exp()[..., None] + joined[0].float() * (joined[1] - both).exp()[..., None]
        lse = both
    return out.to(q.dtype), lse


def run(state):
    case = state["case"]
    if case["kind"] == "rotate":
        if own:
            q, k = state["rope"](state["q"], state["k"], positions=state["positions"])
        else:
            q, k = (_turned(state[x], state["positions"], state[x + "_weight"], state["inv_freq"], case["layout"])
                    .to(state[x].dtype) for x in ("q", "k"))
        return {"q": q, "k": k}
    if case["kind"] == "append":
        start, T, page = case["start"], case["tokens"], case["page"]
        if own:
            state["pages"].append(start, state["k"], state["v"], rope=state["rope"])
        else:
            at = start + torch.arange(T, device=DEVICE)
            pages, places = state["table"][:, at // page].long(), (at % page).expand(case["seqs"], T)
            state["k_pages"][pages, :, places] = _turned(state["k"], at.expand(case["seqs"], T), state["k_weight"],
                                                         state["inv_freq"], case["layout"]).to(state["k"].dtype)
            state["v_pages"][pages, :, places] = state["v"]
        return {"k_pages": state["k_pages"], "v_pages": state["v_pages"]}
    if own:
        out, lse = state["pages"].attend(case["length"], state["q"], visible=state["visible"], joined=state["joined"])
    else:
        out, lse = _plain_attend(state["q"], state["k_pages"], state["v_pages"], state["table"], case["length"],
                                 state["visible"], state["joined"])
    return {"out": out, "lse": lse}


# ------------------------------------------------------------------------------------ 64 bits

def _exact_turn(x, positions, weight, inv_freq, layout):
    """Rotation as the product with a complex number of length one."""
    x = x.double()
    if weight is not None:
        x = x / (x.square().sum(-1, keepdim=True) / x.shape[-1] + EPS).sqrt() * weight.double()
    half = inv_freq.numel()
    unit = torch.polar(torch.ones((), dtype=torch.float64, device=x.device),
                       torch.einsum("st,j->stj", positions.double(), inv_freq.double()))[:, :, None]
    first, second = (range(half), range(half, 2 * half)) if layout == "halves" else (range(0, 2 * half, 2), range(1, 2 * half, 2))
    first, second = torch.tensor(list(first), device=x.device), torch.tensor(list(second), device=x.device)
    z = torch.complex(x[..., first], x[..., second]) * unit
    y = x.clone()
    y[..., first], y[..., second] = z.real, z.imag
    return y


def exact(case, seed):
    state = _inputs(case, seed)
    S, T, H, d = case["seqs"], case["tokens"], case["kv_heads"], case["dim"]
    if case["kind"] == "rotate":
        return {x: _exact_turn(state[x], state["positions"], state[x + "_weight"], state["inv_freq"], case["layout"]) for x in ("q", "k")}
    page = case["page"]
    if case["kind"] == "append":
        entry = case["start"] + torch.arange(T, device=DEVICE)
        k = _exact_turn(state["k"], entry.expand(S, T), state["k_weight"], state["inv_freq"], case["layout"])
        pools = {}
        for name, rows in (("k_pages", k), ("v_pages", state["v"].double())):
            pool = state[name].double()
            for s in range(S):
                by_page = state["table"][s].long()[entry // page]
                pool.transpose(1, 2)[by_page, entry % page] = rows[s]
            pools[name] = pool
        return pools
    Hq, G, length = case["q_heads"], case["q_heads"] // H, case["length"]
    out = torch.zeros((S, T, Hq, d), dtype=torch.float64, device=DEVICE)
    lse = torch.zeros((S, T, Hq), dtype=torch.float64, device=DEVICE)
    entry = torch.arange(length, device=DEVICE)
    for s in range(S):
        by_page = state["table"][s].long()[entry // page]
        limit = torch.full((T,), length, device=DEVICE) if state["visible"] is None else state["visible"][s].long()
        for h in range(Hq):
            k, v = (state[x][by_page, h // G, entry % page].double() for x in ("k_pages", "v_pages"))
            logits = state["q"][s, :, h].double() @ k.T.contiguous() / d ** 0.5
            logits[entry[None] >= limit[:, None]] = -math.inf
            whole = torch.logsumexp(logits, 1)
            share = torch.exp(logits - whole[:, None]).nan_to_num(0.0)
            out[s, :, h], lse[s, :, h] = share @ v, whole
    if state["joined"] is not None:
        found, its = state["joined"][0].double(), state["joined"][1].double()
        share = torch.sigmoid(lse - its)[..., None]
        out, lse = share * out + (1.0 - share) * found, torch.logaddexp(lse, its)
    return {"out": out, "lse": lse}


def work(case):
    S, T, H, d = case["seqs"], case["tokens"], case["kv_heads"], case["dim"]
    size = 4 if case["dtype"] == "fp32" else 2
    if case["kind"] == "rotate":
        rows = S * T * (case["q_heads"] + H)
        return {"bytes": 2 * rows * d * size + 4 * S * T, "flops": rows * (3 * case["dims"] + (4 * d if case["norm"] else 0))}
    if case["kind"] == "append":
        return {"bytes": 4 * S * T * H * d * size, "flops": S * T * H * (3 * case["dims"] + (4 * d if case["norm"] else 0))}
    length, rows = case["length"], S * T * case["q_heads"]
    seen = (T + 1) / 2 if case["sees"] == "causal" else length / 2 * 6 / 7 if case["sees"] == "some" else length
    moved = 2 * S * length * H * d * size + 2 * rows * d * size + 4 * rows
    if case["joined"]:
        moved += rows * (d * size + 4)
    return {"bytes": int(moved), "flops": int(4 * rows * d * seen)}
