"""The calls around a long cache in pages together, as a program makes them: a prompt, its weights, an eviction, steps over chosen blocks; captured and
replayed; on other streams; in a pool beyond 2^32 bytes; and the cases of perf/more_operators.py at their own sizes."""
import importlib.util
import math
import os
import random

import pytest
import torch

import long64
import plain64
import test_gpu_blocks as blocks_
import test_gpu_weights as weights_
from plain64 import U
from test_gpu_blocks import TYPES, Cache

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
_spec = importlib.util.spec_from_file_location("more_operators_cases", os.path.join(ROOT, "perf", "more_operators.py"))
more = importlib.util.module_from_spec(_spec)
_spec.loader.exec_module(more)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("page,block", [(16, 32), (24, 16), (64, 64)])
def test_a_generation(lazyev_lib, dtype, d, page, block):
    """A prompt of 200 entries brought down to 128, then 40 steps that read 4 chosen blocks each, with an eviction to 128 every 16: every call against
    64 bits, from the state that the calls before it left."""
    S, H, Hq, budget, window = 2, 2, 14, 128, 16
    c = Cache(lazyev_lib, dtype, d, S, H, page, 256, seed=30)
    keys = lazyev_lib.KeyBounds.of(c.cache, block)
    assert keys.bounds.shape[2] == -(-c.cache.entries // block)
    k, v = c.randn(S, 200, H, d).to(c.dt), c.randn(S, 200, H, d).to(c.dt)
    c.cache.append(0, k, v)
    assert torch.equal(c.rows(c.k_pages)[:, :200], k)
    q = c.randn(S, 200, Hq, d).to(c.dt)
    seen = torch.arange(1, 201, device="cuda").int().expand(S, 200).contiguous()
    lse = c.cache.attend(200, q, visible=seen)[1]
    weights = torch.zeros((S, H, 256), device="cuda")
    weights_._weigh(c, 200, q, lse, visible=seen, weights=weights)
    positions = torch.arange(256, device="cuda").int().expand(S, H, 256).contiguous()
    weights_._evict(c, 200, weights, budget, window, 4, positions=positions, in_place=True)
    length = budget
    keys.update(c.cache, 0, length)
    for t in range(200, 240):
        k, v = c.randn(S, 1, H, d).to(c.dt), c.randn(S, 1, H, d).to(c.dt)
        c.cache.append(length, k, v, position0=t)
        keys.update(c.cache, length, 1)
        positions[:, :, length] = t
        length += 1
        now = blocks_._bounds_of(c.rows(c.k_pages)[:, :length], block)
        assert torch.equal(keys.bounds[:, :, :now.shape[2]], now)
        token = c.randn(S, 1, Hq, d).to(c.dt)
        chosen = keys.choose(length, token, 4, first=1, last=1)
        for s in range(S):
            want = long64.choose(long64.scores(token[s], now[s]), [length], block, 1, 1, 4)
            assert torch.equal(chosen[s].cpu(), want)
        _, lse = blocks_._attend(c, length, token, chosen, block)
        # (weights beside the chosen blocks alone: of entries of others they are what their logits make beside those)
        weights_._weigh(c, length, token, lse, old=weights, known=length - 1, decay=0.95, weights=weights)
        if length == budget + window:
            weights_._evict(c, length, weights, budget, window, 4, positions=positions, in_place=True)
            length = budget
            keys.update(c.cache, 0, length)
    assert length == budget + 8


class Step:
    """One step of everything, on buffers of its own."""

    def __init__(self, b, dtype, d, S, n, H, Hq, length, keep, seed):
        self.c = c = Cache(b, dtype, d, S, H, 32, length, seed=seed)
        self.n, self.length, self.keep = n, length, keep
        self.keys = b.KeyBounds.of(c.cache, 32)
        self.keys.update(c.cache, 0, length - n)
        self.q = c.randn(S, n, Hq, d).to(c.dt)
        self.vis = torch.arange(length - n + 1, length + 1, device="cuda").int().expand(S, n).contiguous()
        self.old = c.randn(S, H, length).exp()
        self.tensors = [c.k_pages, c.v_pages, self.keys.bounds, self.q, self.old]

    def __call__(self):
        c = self.c
        self.keys.update(c.cache, self.length - self.n, self.n)
        chosen = self.keys.choose(self.length, self.q, 6, visible=self.vis, first=1, last=2)
        out, lse = c.cache.attend_blocks(self.length, self.q, chosen, 32, visible=self.vis)
        weights = c.cache.weigh(self.length, self.q, lse, old=self.old, decay=0.9, visible=self.vis)
        sources, kept, positions = c.cache.evict(self.length, weights, self.keep, recent=16, first=4)
        return [chosen, out, lse, weights, sources, kept, positions]

    def load(self, other, scale):
        for x, y in zip(self.tensors, other.tensors):
            x.copy_(y)
        self.q.mul_(scale)


@pytest.mark.parametrize("dtype,d,S,n,H,Hq,length,keep", [
    ("bf16", 128, 2, 1, 4, 28, 900, 500), ("fp32", 64, 1, 40, 8, 16, 700, 690), ("bf16", 64, 1, 300, 2, 14, 1500, 400), ("fp32", 128, 2, 3, 2, 6, 40000, 5000)])
def test_captured_and_replayed(lazyev_lib, dtype, d, S, n, H, Hq, length, keep):
    """Three replays on contents of their own, eager work and synchronizations between them, each against the eager calls."""
    first = Step(lazyev_lib, dtype, d, S, n, H, Hq, length, keep, seed=40)
    step, eager = (Step(lazyev_lib, dtype, d, S, n, H, Hq, length, keep, seed=40) for _ in range(2))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()                                     # (allocations of this stream)
        step.load(first, 1.0)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        captured = step()
    for scale in (1.0, 0.5, 1.75):
        step.load(first, scale)
        eager.load(first, scale)
        want = eager()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(captured + step.tensors, want + eager.tensors):
            assert torch.equal(x, y)


def test_on_two_streams_at_once(lazyev_lib):
    shapes = [("bf16", 128, 2, 1, 4, 28, 3000, 2000), ("bf16", 128, 1, 200, 4, 28, 2000, 1000)]
    steps = [Step(lazyev_lib, *x, seed=50) for x in shapes]
    alone = [Step(lazyev_lib, *x, seed=50) for x in shapes]
    want = [s() for s in alone]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in steps]
    got = []
    for s, stream in zip(steps, streams):
        with torch.cuda.stream(stream):
            got.append(s())
    torch.cuda.synchronize()
    for g, w, s, a in zip(got, want, steps, alone):
        assert all(torch.equal(x, y) for x, y in zip(g + s.tensors, w + a.tensors))


def test_sequences_of_a_batch_do_not_see_one_another(lazyev_lib):
    """The bits of a sequence are those of a batch with another sequence beside it (the sizes of the call being the same)."""
    a, b = (Step(lazyev_lib, "bf16", 128, 2, 3, 4, 28, 1200, 700, seed=60) for _ in range(2))
    with torch.no_grad():
        b.q[1].mul_(-2.0)
        b.old[1].add_(1.0)
    x, y = a(), b()
    for g, w in zip(x, y):
        assert torch.equal(g[0], w[0])


def test_entries_beyond_2_32_bytes(lazyev_lib):
    """A pool of 6 GB of keys and of values whose last pages hold the cache."""
    H, page, d, n_pages = 8, 256, 128, 12000
    k_pages, v_pages = (torch.empty((n_pages, H, page, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    assert 8200 * H * page * d * 2 > 2 ** 32
    c = Cache(lazyev_lib, "bf16", d, 1, H, page, 1000, seed=70)
    table = torch.tensor([[n_pages - 1, 11990, 9000, 8200]], device="cuda").int()
    for t, small in zip(table[0].tolist(), c.table[0].tolist()):
        k_pages[t], v_pages[t] = c.k_pages[small], c.v_pages[small]
    big = lazyev_lib.PagedCache(k_pages, v_pages, table)
    q = c.randn(1, 5, 40, d).bfloat16()
    blocks = blocks_._some_blocks(c, 5, 1000, 16, 20)
    out = big.attend_blocks(1000, q, blocks, 16), big.attend(1000, q)
    want = c.cache.attend_blocks(1000, q, blocks, 16), c.cache.attend(1000, q)
    assert all(torch.equal(x, y) for g, w in zip(out, want) for x, y in zip(g, w))
    lse = out[1][1]
    weights = big.weigh(1000, q, lse)
    assert torch.equal(weights, c.cache.weigh(1000, q, lse))
    keys = [lazyev_lib.KeyBounds.of(x, 64) for x in (big, c.cache)]
    for x, cache in zip(keys, (big, c.cache)):
        x.update(cache, 0, 1000)
    assert torch.equal(keys[0].bounds[:, :, :15], keys[1].bounds[:, :, :15])
    got, want = (x.evict(1000, weights, 300, recent=10) for x in (big, c.cache))
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    for t, small in zip(table[0].tolist(), c.table[0].tolist()):
        assert torch.equal(k_pages[t], c.k_pages[small]) and torch.equal(v_pages[t], c.v_pages[small])


CASES = {c["name"]: c for c in more.listed()}
CASES.update(("drawn_%d" % i, more.draw(random.Random(i))) for i in range(20))


@pytest.mark.parametrize("name", CASES)
def test_case(lazyev_lib, monkeypatch, name):
    monkeypatch.setattr(more, "own", True)
    case, seed = CASES[name], 78
    state = more.prepare(case, seed)
    got = more.run(state)
    kind = case["kind"]
    if kind in ("bound", "choose", "evict"):
        exact = more.exact(case, seed)
        for x in exact:
            assert torch.equal(got[x].to(exact[x].dtype), exact[x]), x
        return
    S, T, H, d, length = case["seqs"], case["tokens"], case["kv_heads"], case["dim"], case["length"]
    for s in range(S):
        k, v = (state[x][state["table"][s].long()].transpose(1, 2).flatten(0, 1)[:length] for x in ("k_pages", "v_pages"))
        vis = torch.full((T,), length, device="cuda") if state["visible"] is None else state["visible"][s].long()
        if kind == "weigh":
            want, bound = long64.weigh(state["q"][s], state["lse"][s], k, vis, d ** -0.5)
            known = case["known"]
            kept = float(torch.tensor(case["decay"])) * state["old"][s, :, :known].double()
            want[:, :known] += kept
            bound[:, :known] += 2 * U * kept.abs()
            off = (got["weights"][s, :, :length].double() - want).abs()
            assert bool((off <= bound + U * want.abs() + 1e-30).all())
            continue
        G = case["q_heads"] // H
        for i in sorted({0, 1, T // 2, T - 1} & set(range(T)) | set(range(0, T, max(1, T // 12)))):
            for h in range(H):
                end, block = int(vis[i]), case["block"]
                at = [torch.arange(x * block, min((x + 1) * block, end), device="cuda") for x in state["blocks"][s, i, h].tolist() if 0 <= x * block < end]
                at = torch.cat(at) if at else torch.zeros(0, dtype=torch.long, device="cuda")
                mine = slice(h * G, (h + 1) * G)
                joined = None if state["joined"] is None else tuple(x[s, i:i + 1, mine] for x in state["joined"])
                want = plain64.attend(state["q"][s, i:i + 1, mine], k[at, h:h + 1], v[at, h:h + 1], torch.full((1,), len(at), device="cuda"), d ** -0.5, joined)
                plain64.check_out(got["out"][s, i:i + 1, mine], want[0], want[2])
                plain64.check_lse(got["lse"][s, i:i + 1, mine], want[1], want[3])
