"""lazyev_decode_step_shared and the calls around it, together as they are used: a prefix made ready (norm and rotation) and kept in
pages, queries and keys of every step made ready likewise, decode steps over prefix and own cache with evictions.  Outputs and weights
against 64 bits; recurrence state and survivors exactly the oracle's, which thresholds the weights beside the prefix."""
import numpy as np
import pytest
import torch

import plain64
from oracle.lazyev_oracle import OracleUnit

pytestmark = pytest.mark.gpu

TYPES = [("bf16", 128), ("bf16", 64), ("fp32", 128), ("fp32", 64)]
S, HQ, H, B, W, P, STEPS, PRE = 3, 14, 2, 60, 10, 25, 75, 150
ALPHA = 8.0 / (B + PRE)


class World:
    """Raw rows of a prefix, of prompts and of steps, and what a model would make of them."""

    def __init__(self, b, dtype, d, pre=PRE, seed=0):
        self.b, self.d, self.pre = b, d, pre
        self.dt = torch.float32 if dtype == "fp32" else torch.bfloat16
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def randn(*shape):
            return torch.randn(shape, generator=gen, device="cuda").to(self.dt)
        self.rope = b.NormRope(d, self.dt, q_weight=1 + 0.1 * randn(d), k_weight=1 + 0.1 * randn(d),
                               inv_freq=torch.logspace(0, -4, d // 2, device="cuda"))
        self.prefix_k, self.prefix_v = randn(max(pre, 1), H, d), randn(max(pre, 1), H, d)
        self.prompt_k, self.prompt_v = randn(S, P, H, d), randn(S, P, H, d)
        self.q, self.k, self.v = randn(STEPS, S, HQ, d), randn(STEPS, S, H, d), randn(STEPS, S, H, d)
        # a step's queries look for an older key of the sequence now and then
        for t in range(STEPS):
            self.q[t] += 1.5 * self.k[max(0, t - 7 - t % 5)].repeat_interleave(HQ // H, 1)

    def prefix(self, page=16):
        m = -(-max(self.pre, 1) // page)
        pools = [torch.full((m + 1, H, page, self.d), 3.0, dtype=self.dt, device="cuda") for _ in range(2)]
        table = torch.randperm(m + 1, device="cuda")[:m].int()[None]
        cache = self.b.PagedCache(*pools, table, n_q_heads=HQ)
        half = self.pre // 3                       # in two pieces, the second from inside a page
        cache.append(0, self.prefix_k[:half], self.prefix_v[:half], rope=self.rope)
        cache.append(half, self.prefix_k[half:self.pre], self.prefix_v[half:self.pre], rope=self.rope)
        return cache

    def engine(self, **kw):
        eng = self.b.LazyEviction(1, S, HQ, H, self.d, B, W, P, ALPHA, dtype=self.dt, **kw)
        own = self.b.PagedCache(eng.k_cache[0], eng.v_cache[0], torch.arange(S, device="cuda").int()[:, None])
        own.append(0, self.prompt_k, self.prompt_v, rope=self.rope, position0=self.pre)
        return eng.init()

    def step(self, t):
        """Queries and keys of step t (1-based) at the position they have behind prefix and prompt."""
        pos = torch.full((S,), self.pre + P + t - 1, dtype=torch.int32, device="cuda")
        q, k = self.rope(self.q[t - 1], self.k[t - 1], positions=pos)
        return q, k, self.v[t - 1]

    def prefix_rows(self, cache):
        at = torch.arange(self.pre, device="cuda")
        page = cache.table[0].long()[at // cache.pages.page_size]
        return tuple(x[page, :, at % cache.pages.page_size] for x in (cache.k_pages, cache.v_pages))


@pytest.mark.parametrize("dtype,d", TYPES)
def test_steps_over_prefix_and_own_cache(lazyev_lib, dtype, d):
    w = World(lazyev_lib, dtype, d)
    cache = w.prefix()
    pk, pv = w.prefix_rows(cache)
    want, bound = plain64.turn(w.prefix_k, torch.arange(PRE, device="cuda"), w.rope.k_weight, 1e-6, w.rope.inv_freq, "halves")
    plain64.check_out(pk, want, bound)
    assert torch.equal(pv, w.prefix_v)
    eng, quiet = w.engine(), w.engine()            # one asks for the weights, one does not
    G = HQ // H
    units = [(s, h, OracleUnit(eng.k_cache[0, s, h, :P].double().cpu().numpy(), eng.v_cache[0, s, h, :P].double().cpu().numpy(), G, B, W, ALPHA))
             for s in range(S) for h in range(H)]
    out, out2 = (torch.empty((S, HQ, d), dtype=w.dt, device="cuda") for _ in range(2))
    p_out = torch.zeros((S, HQ, eng.capacity), device="cuda")
    acts, prefix_share = 0, 0.0
    for t in range(1, STEPS + 1):
        q, k, v = w.step(t)
        eng.decode_step_shared(0, t, q, k, v, out, cache, PRE, p_out=p_out)
        quiet.decode_step_shared(0, t, q, k, v, out2, cache, PRE)
        assert torch.equal(out, out2), t
        n = len(units[0][2]) + 1
        p = p_out[:, :, :n].cpu().numpy()
        for s in range(S):
            rows = [torch.cat((x, y[0, s, :, :n].transpose(0, 1))) for x, y in ((pk, eng.k_cache), (pv, eng.v_cache))]
            both = plain64.attend(q[s][None], *rows, torch.tensor([PRE + n], device="cuda"), d ** -0.5)
            # both parts are rounded to the rows' type before they are joined, the logarithms of their sums to 32 bits
            extra = plain64.HALF_STEP[w.dt] * (both[2] * 0 + rows[1].double().abs().amax())
            plain64.check_out(out[s][None], both[0], both[2] + extra + 2e-5 * rows[1].double().abs().amax())
            kh = rows[0].double()
            for h in range(HQ):
                logit = kh[PRE:, h // G] @ q[s, h].double() * d ** -0.5
                joint = torch.exp(logit - both[1][0, h])
                prefix_share += float(1 - joint.sum()) / (STEPS * S * HQ)
                assert float((joint.cpu() - torch.from_numpy(p[s, h]).double()).abs().max()) < 2e-5 * float(joint.max())
        for s, h, u in units:
            _, _, act = u.decode_step(t, q[s, h * G:(h + 1) * G].double().cpu().numpy(), k[s, h].double().cpu().numpy(),
                                      v[s, h].double().cpu().numpy(), p_override=p[s, h * G:(h + 1) * G])
            acts += int(act.sum())
        gone = eng.evict_all(t)
        assert quiet.evict_all(t) == gone
        for s, h, u in units:
            assert len(u.evict(t)) == gone
        if gone or t % 7 == 0:
            eng.stats()
            for s, h, u in units:
                m = len(u)
                assert np.array_equal(eng.pos[0, s, h, :m].cpu().numpy(), u.pos) and np.array_equal(eng.ts[0, s, h, :m].cpu().numpy(), u.TS)
                assert np.array_equal(eng.mri[0, s, h, :m].cpu().numpy(), u.MRI)
    assert 0.2 < prefix_share < 0.98               # the prefix has a part in it, and so have the own entries
    st, st2 = eng.stats(), quiet.stats()
    assert st == st2 and st["n_activations"] == [acts] and st["n_evict_events"][0] >= 3
    n = st["len"][0]
    for x, y in ((eng.ts, quiet.ts), (eng.mri, quiet.mri), (eng.pos, quiet.pos), (eng.k_cache, quiet.k_cache)):
        assert torch.equal(x[:, :, :, :n], y[:, :, :, :n])


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("fp32", 64)])
def test_without_a_prefix_and_with_one_of_no_pages(lazyev_lib, dtype, d):
    """prefix_len 0, or a table that leads nowhere, is lazyev_decode_step, bit by bit."""
    w = World(lazyev_lib, dtype, d)
    cache = w.prefix()
    runs = []
    for how in ("plain", "zero", "nowhere"):
        eng, res = w.engine(), []
        if how == "nowhere":
            cache.table.fill_(-1)
        for t in range(1, 31):
            q, k, v = w.step(t)
            out = torch.empty_like(q)
            if how == "plain":
                eng.decode_step(0, t, q, k, v, out)
            else:
                eng.decode_step_shared(0, t, q, k, v, out, cache, 0 if how == "zero" else PRE)
            eng.evict_all(t)
            res.append(out)
        st = eng.stats()
        n = st["len"][0]
        runs.append((torch.stack(res), eng.ts[:, :, :, :n].clone(), eng.mri[:, :, :, :n].clone(), eng.pos[:, :, :, :n].clone(), st))
    for r in runs[1:]:
        assert all(torch.equal(x, y) for x, y in zip(r[:4], runs[0][:4])) and r[4] == runs[0][4]


def test_ranking_by_the_steps_own_weights(lazyev_lib):
    """Evictions that rank by the weights of their own step take those beside the prefix: each query head's weights are scaled by a
    share of its own, so the largest of a group's heads may be another one than without the prefix."""
    w = World(lazyev_lib, "bf16", 128)
    cache, G = w.prefix(), HQ // H
    eng = w.engine(score_flags=lazyev_lib.SCORE_CURRENT_ATTENTION)
    out = torch.empty((S, HQ, 128), dtype=w.dt, device="cuda")
    p_out = torch.zeros((S, HQ, eng.capacity), device="cuda")
    pos = None
    for t in range(1, STEPS + 1):
        q, k, v = w.step(t)
        eng.decode_step_shared(0, t, q, k, v, out, cache, PRE, p_out=p_out)
        n = eng.stats()["len"][0]
        pos = eng.pos[0, :, :, :n].clone()
        if eng.evict(0, t):
            p = p_out[:, :, :n].view(S, H, G, n).amax(2)
            eng.stats()
            for s in range(S):
                for h in range(H):
                    score = p[s, h, :n - W].cpu().numpy().astype(np.float64)
                    order = sorted(range(n - W), key=lambda i: (score[i], i))[-(B - W):]
                    keep = sorted(order) + list(range(n - W, n))
                    got = eng.pos[0, s, h, :B].tolist()
                    assert got == [int(pos[s, h, i]) for i in keep], (t, s, h)
    assert eng.stats()["n_evict_events"][0] >= 3


def test_sequences_that_take_no_part_are_left_alone(lazyev_lib):
    w = World(lazyev_lib, "bf16", 128)
    cache = w.prefix()
    eng, all_in = w.engine(), w.engine()
    eng.retire(1)
    for t in range(1, 25):
        if t == 12:
            eng.admit(1, 0, 13)                    # from step 14 on
        q, k, v = w.step(t)
        out = torch.full_like(q, 5.0)
        eng.decode_step_shared(0, t, q, k, v, out, cache, PRE)
        eng.evict_all(t)
        want = torch.empty_like(q)
        all_in.decode_step_shared(0, t, q, k, v, want, cache, PRE)
        all_in.evict_all(t)
        for s in (0, 2):
            assert float((out[s].float() - want[s].float()).abs().max()) <= 2.0 ** -7 * float(want.abs().max())
        assert bool((out[1] == 5).all()) == (t < 14)
    eng.stats()


def test_replayed_and_on_a_stream_of_its_own(lazyev_lib):
    """A captured step is replayed with new inputs; the context's stream is not the current one."""
    w = World(lazyev_lib, "bf16", 128)
    cache = w.prefix()
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        eager = w.engine(stream=stream)
        captured = w.engine(stream=stream)
    ins = [w.step(t) for t in range(1, 9)]
    torch.cuda.synchronize()
    wants = []
    for q, k, v in ins:                            # each as the first step of a fresh context
        eager.init()
        out = torch.empty_like(q)
        eager.decode_step_shared(0, 1, q, k, v, out, cache, PRE)
        wants.append(out)
    torch.cuda.synchronize()
    bufs = [x.clone() for x in ins[0]]
    out = torch.empty_like(bufs[0])
    work = torch.empty(cache.workspace_bytes(PRE, S, HQ) + 1, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        captured.decode_step_shared(0, 1, *bufs, out, cache, PRE, workspace=work)
    for r in range(16):
        for b, x in zip(bufs, ins[r % 8]):
            b.copy_(x)
        if r % 3 == 0:
            torch.cuda.synchronize()
            work.fill_(171)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, wants[r % 8]), r


def test_refusals(lazyev_lib):
    """Nothing happens to the context: the step can still be taken."""
    b = lazyev_lib
    w = World(b, "bf16", 128)
    cache, eng = w.prefix(), w.engine()
    q, k, v = w.step(1)
    out = torch.empty_like(q)

    def fails(code, *a, **kw):
        with pytest.raises(b.LazyevError) as e:
            eng.decode_step_shared(*a, **kw)
        assert e.value.code == code
    two = b.PagedCache(cache.k_pages, cache.v_pages, cache.table.expand(2, -1).contiguous())
    other = b.PagedCache(cache.k_pages.float(), cache.v_pages.float(), cache.table)
    heads = b.PagedCache(cache.k_pages[:, :1].contiguous(), cache.v_pages[:, :1].contiguous(), cache.table)
    for bad in (two, other, heads):
        fails(b.EINVAL, 0, 1, q, k, v, out, bad, 100)
    fails(b.EINVAL, 0, 1, q, k, v, out, cache, 100000)
    fails(b.EINVAL, 0, 1, q, k, v, out, cache, -1)
    fails(b.EINVAL, 0, 1, q, k, v, q, cache, PRE)
    fails(b.EINVAL, 0, 2, q, k, v, out, cache, PRE)
    fails(b.EINVAL, 1, 1, q, k, v, out, cache, PRE)
    eng.set_variant(0)
    fails(b.EINVAL, 0, 1, q, k, v, out, cache, PRE)
    eng.set_variant(1)
    eng.decode_step_shared(0, 1, q, k, v, out, cache, PRE)
    assert eng.stats()["len"] == [P + 1]


def test_binding_checks_its_tensors(lazyev_lib):
    b = lazyev_lib
    q = torch.zeros((4, 8, 128), dtype=torch.bfloat16, device="cuda")
    rope = b.NormRope(128, inv_freq=torch.ones(64, device="cuda"))
    pages = torch.zeros((3, 2, 16, 128), dtype=torch.bfloat16, device="cuda")
    table = torch.zeros((1, 2), dtype=torch.int32, device="cuda")
    cache = b.PagedCache(pages, pages.clone(), table, n_q_heads=8)
    kv = torch.zeros((4, 2, 128), dtype=torch.bfloat16, device="cuda")
    pos = torch.zeros(4, dtype=torch.int32, device="cuda")
    for bad in (lambda: rope(q.float()), lambda: rope(q.cpu()), lambda: rope(q[..., ::2]), lambda: rope(q, kv[:3]), lambda: rope(),
                lambda: rope(q, positions=pos.long()), lambda: rope(q, positions=pos[:3]), lambda: rope(q, q_out=torch.empty_like(q[:3])),
                lambda: rope(q.transpose(1, 2)), lambda: rope(q, start=1 << 40), lambda: b.NormRope(96), lambda: b.NormRope(64, torch.float16),
                lambda: b.NormRope(128, inv_freq=torch.ones(63, device="cuda")), lambda: b.NormRope(128, q_weight=q[0, 0].float()),
                lambda: b.PagedCache(pages, pages[:2], table), lambda: b.PagedCache(pages, pages, table.long()),
                lambda: b.PagedCache(pages[..., :32], pages[..., :32], table), lambda: cache.append(30, kv, kv), lambda: cache.append(-1, kv, kv),
                lambda: cache.append(0, kv, kv[:3]), lambda: cache.append(0, q, q), lambda: cache.append(0, kv.float(), kv.float()),
                lambda: cache.attend(33, q), lambda: cache.attend(5, q[:, :4].contiguous()), lambda: cache.attend(5, q.transpose(0, 1)),
                lambda: cache.attend(5, q, visible=pos.long()), lambda: cache.attend(5, q, joined=(q, torch.zeros(4, 7, device="cuda"))),
                lambda: cache.attend(5, q, out=q.float()), lambda: cache.attend(5, q, workspace=pos)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(b.LazyevError) as e:
        cache.attend(5, q, out=q)
    assert e.value.code == b.EINVAL
