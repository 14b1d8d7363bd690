"""Calls around a decode step that no other test makes: queries that are no numbers beside others, a norm for one kind of heads only, the most rows a call
takes, results that nobody asked for, a shared step whose own caches are empty or whose weights the caller hands in."""
import math

import pytest
import torch

import plain64
from test_gpu_pages import TYPES, Case, _dt

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("n,length,Hq,H", [(2, 200, 7, 1), (40, 700, 28, 4), (300, 400, 2, 1), (900, 300, 7, 1), (9000, 130, 1, 1)])
@pytest.mark.parametrize("some", [False, True])
def test_a_query_that_is_no_number_has_no_influence_on_others(lazyev_lib, dtype, d, n, length, Hq, H, some):
    c = Case(lazyev_lib, dtype, d, 1, n, Hq, H, 16, length, seed=41)
    vis = torch.randint(1, length + 1, (1, n), generator=c.gen, device="cuda").int() if some else None
    clean = c.cache.attend(length, c.q, visible=vis)
    bad = torch.zeros(n, dtype=torch.bool, device="cuda")
    bad[1::3] = True
    c.q[:, 1::3, :, 5] = math.nan
    c.q[:, 1::6, :, 5] = math.inf
    out, lse = c.cache.attend(length, c.q, visible=vis)
    assert torch.equal(out[:, ~bad], clean[0][:, ~bad]) and torch.equal(lse[:, ~bad], clean[1][:, ~bad])
    # NaN everywhere, but where an infinite query meets entries of the other sign only: its logits are all minus infinity, the weights zero, and the
    # token has seen nothing
    k5 = c.rows(c.k_pages)[0, :, :, 5].float()     # [length, H]
    seen = torch.arange(length, device="cuda")[None] < (torch.full((n,), length, device="cuda") if vis is None else vis[0].long())[:, None]
    against = ~(seen[:, :, None] & (k5 >= 0)[None]).any(1).repeat_interleave(Hq // H, 1)     # [n, Hq]
    nothing = torch.zeros_like(against)
    nothing[1::6] = against[1::6]
    assert bool((out[0][nothing] == 0).all()) and bool((lse[0][nothing] == -math.inf).all())
    assert bool(out[0][bad[:, None] & ~nothing].isnan().all())


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("n", [5, 4500])
@pytest.mark.parametrize("normed", ["q", "k"])
def test_a_norm_for_queries_or_keys_only(lazyev_lib, dtype, d, n, normed):
    dt, gen = _dt(dtype), torch.Generator(device="cuda").manual_seed(n)
    w = (1.0 + 0.2 * torch.randn(d, generator=gen, device="cuda")).to(dt)
    freq = torch.logspace(0, -4, d // 4, device="cuda")
    rope = lazyev_lib.NormRope(d, dt, q_weight=w if normed == "q" else None, k_weight=w if normed == "k" else None, inv_freq=freq)
    q, k = (3 * torch.randn((n, h, d), generator=gen, device="cuda").to(dt) for h in (3, 2))
    got = rope(q, k)
    for x, y, weight in ((q, got[0], rope.q_weight), (k, got[1], rope.k_weight)):
        want, bound = plain64.turn(x, torch.arange(n, device="cuda"), weight, 1e-6, freq, "halves")
        plain64.check_out(y, want, bound)


@pytest.mark.parametrize("dtype,d,G,n", [("bf16", 64, 1, 65535 * 32), ("fp32", 64, 64, 65535 // 2)])
def test_the_most_rows_of_a_table_row(lazyev_lib, dtype, d, G, n):
    c = Case(lazyev_lib, dtype, d, 1, n, G, 1, 16, 33, seed=42)
    vis = torch.randint(0, 34, (1, n), generator=c.gen, device="cuda").int()
    c.check(c.cache.attend(33, c.q, visible=vis), visible=vis)
    more = torch.zeros((1, n + 65536 * 32 // G, G, d), dtype=c.dt, device="cuda")
    with pytest.raises(lazyev_lib.LazyevError):
        c.cache.attend(33, more)


@pytest.mark.parametrize("dtype,d", TYPES)
def test_many_table_rows(lazyev_lib, dtype, d):
    """A few thousand sequences of a token each."""
    c = Case(lazyev_lib, dtype, d, 3000, 1, 4, 2, 16, 19, seed=43)
    out, lse = c.cache.attend(19, c.q)
    k, v = c.rows(c.k_pages), c.rows(c.v_pages)
    for s in range(0, 3000, 157):
        want = plain64.attend(c.q[s], k[s], v[s], torch.full((1,), 19, device="cuda"), d ** -0.5)
        plain64.check_out(out[s], want[0], want[2])
        plain64.check_lse(lse[s], want[1], want[3])


@pytest.mark.parametrize("n,length", [(1, 9000), (700, 300)])
def test_no_lse_asked_for(lazyev_lib, n, length):
    b = lazyev_lib
    c = Case(b, "bf16", 128, 1, n, 8, 2, 16, length, seed=44)
    joined = ((0.3 * c.randn(1, n, 8, 128)).to(c.dt), math.log(length) + c.randn(1, n, 8))
    want = c.cache.attend(length, c.q, joined=joined)[0]
    out, need = torch.empty_like(c.q), c.cache.workspace_bytes(length, n)
    work = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
    code = b.lib.lazyev_pages_attend(c.cache.pages, length, n, 8, None, c.q.data_ptr(), joined[0].data_ptr(), joined[1].data_ptr(), out.data_ptr(), None,
                                     0.0, work.data_ptr(), need, torch.cuda.current_stream().cuda_stream)
    assert code == b.OK and torch.equal(out, want)


@pytest.mark.parametrize("dtype,d", TYPES)
def test_a_shared_step_of_empty_caches_and_of_weights_handed_in(lazyev_lib, dtype, d):
    b, S, H, Hq, pre, B, W = lazyev_lib, 2, 2, 6, 90, 12, 4
    dt, gen = _dt(dtype), torch.Generator(device="cuda").manual_seed(7)

    def randn(*shape):
        return torch.randn(shape, generator=gen, device="cuda").to(dt)
    m = -(-pre // 16)
    cache = b.PagedCache(randn(m, H, 16, d), randn(m, H, 16, d), torch.randperm(m, generator=gen, device="cuda").int()[None])
    rows = [x[cache.table[0].long()].transpose(1, 2).flatten(0, 1)[:pre] for x in (cache.k_pages, cache.v_pages)]
    ask, told = (b.LazyEviction(1, S, Hq, H, d, B, W, 0, 0.01, dtype=dt).init() for _ in range(2))
    p_out = torch.zeros((S, Hq, ask.capacity), device="cuda")
    for t in range(1, 31):
        q, k, v = randn(S, Hq, d), randn(S, H, d), randn(S, H, d)
        out, again = torch.empty_like(q), torch.empty_like(q)
        ask.decode_step_shared(0, t, q, k, v, out, cache, pre, p_out=p_out)
        told.decode_step_shared(0, t, q, k, v, again, cache, pre, p_override=p_out)
        assert torch.equal(out, again)
        n = ask.stats()["len"][0]
        for s in range(S):
            both = [torch.cat((x, y[0, s, :, :n].transpose(0, 1))) for x, y in zip(rows, (ask.k_cache, ask.v_cache))]
            want = plain64.attend(q[s][None], *both, torch.tensor([pre + n], device="cuda"), d ** -0.5)
            # (both parts rounded to the rows' type before they are joined, the logarithms of their sums to 32 bits)
            size = both[1].double().abs().amax()
            plain64.check_out(out[s][None], want[0], want[2] + (plain64.HALF_STEP[dt] + 2e-5) * size)
        assert ask.evict_all(t) == told.evict_all(t)
    assert ask.stats() == told.stats()
    n = ask.stats()["len"][0]
    for x, y in ((ask.ts, told.ts), (ask.mri, told.mri), (ask.pos, told.pos)):
        assert torch.equal(x[..., :n], y[..., :n])
