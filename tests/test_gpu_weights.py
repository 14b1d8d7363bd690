"""The weights that a cache's entries received and the eviction by them, against their definitions: head groups, page sizes, what tokens see, ties,
infinities and NaN, lengths of one's own, places that are no page."""
import math

import numpy as np
import pytest
import torch

import long64
from plain64 import U
from test_gpu_blocks import TYPES, Cache, _off_by_one

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------ weights

def _weigh(c, length, q, lse, visible=None, old=None, known=None, decay=1.0, scale=0.0, there=None, weights=None):
    before = None if old is None else old.clone()
    got = c.cache.weigh(length, q, lse, weights=weights, old=old, known=known, decay=decay, visible=visible, scale=scale)
    k = c.rows(c.k_pages)
    S, n, Hq, d = q.shape
    known = (0 if old is None else length) if known is None else known
    for s in range(S):
        vis = torch.full((n,), length, device="cuda") if visible is None else visible[s].long().clamp(0, length)
        want, bound = long64.weigh(q[s], lse[s], k[s, :length], vis, scale or d ** -0.5, None if there is None else there[s][:length])
        if known:
            kept = float(np.float32(decay)) * before[s, :, :known].double()
            want[:, :known] += kept
            bound[:, :known] += 2 * U * kept.abs()
        off = (got[s, :, :length].double() - want).abs()
        most = bound + U * want.abs() + 1e-30
        assert bool((off <= most).all()), (s, float((off / most).max()))
    return got


def _lse(c, length, q, visible=None):
    return c.cache.attend(length, q, visible=visible)[1]


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("S,n,Hq,H,page,length", [
    (1, 1, 1, 1, 16, 1), (2, 1, 28, 4, 16, 333), (1, 1, 8, 1, 24, 5000), (3, 5, 8, 8, 1, 77), (1, 4, 64, 1, 64, 600), (2, 33, 33, 1, 48, 500), (1, 130, 6, 2, 100, 130),
    (1, 600, 7, 1, 32, 700), (2, 70, 32, 8, 16, 129), (1, 1000, 2, 1, 4096, 128)])
def test_weights(lazyev_lib, dtype, d, S, n, Hq, H, page, length):
    c = Cache(lazyev_lib, dtype, d, S, H, page, length, seed=6)
    q = (1.3 * c.randn(S, n, Hq, d)).to(c.dt)
    lse = _lse(c, length, q)
    first = _weigh(c, length, q, lse)
    assert first.shape == (S, H, length)
    total = first.double().sum((1, 2))             # every row's weights add up to one
    assert bool(((total - n * Hq).abs() <= 1e-3 * n * Hq).all())
    vis = c.randint(0, length + 1, S, n).int()
    vis[:, ::4], vis[:, 1::6] = length, 0
    if n > 2:
        vis[:, 2::7] = -5
    lse = _lse(c, length, q, vis)
    old = c.randn(S, H, length + 3).exp()
    tail = old[:, :, length:].clone()
    for known, decay in ((length, 1.0), (length // 2, 0.9), (0, 0.5), (length, 0.0), (length, -2.5)):
        junk = torch.full_like(old, math.nan)
        got = _weigh(c, length, q, lse, visible=vis, old=old, known=known, decay=decay, weights=junk)
        assert got is junk and bool(torch.isnan(got[:, :, length:]).all())
    want = c.cache.weigh(length, q, lse, old=old, decay=0.9, visible=vis)[:, :, :length]
    got = _weigh(c, length, q, lse, visible=vis, old=old, decay=0.9, weights=old)       # in place
    assert got is old and torch.equal(got[:, :, :length], want) and torch.equal(got[:, :, length:], tail)
    # joined with much else the weights are small, with a scale of one's own others
    _weigh(c, length, q, lse + 5.0, visible=vis)
    _weigh(c, length, q, c.cache.attend(length, q, scale=0.3)[1], scale=0.3)


@pytest.mark.parametrize("dtype,d", TYPES)
def test_a_prompts_own_weights_then_steps(lazyev_lib, dtype, d):
    """A prompt of 300 tokens, each over its past, and ten steps of one token: the sum of all weights is the number of rows."""
    c = Cache(lazyev_lib, dtype, d, 2, 2, 24, 310, seed=7)
    q = c.randn(2, 310, 14, d).to(c.dt)
    vis = torch.arange(1, 311, device="cuda").int().expand(2, 310).contiguous()
    prompt, seen = q[:, :300].contiguous(), vis[:, :300].contiguous()
    weights = torch.full((2, 2, 310), math.nan, device="cuda")
    _weigh(c, 300, prompt, _lse(c, 300, prompt, seen), visible=seen, weights=weights)
    for t in range(300, 310):
        token = q[:, t:t + 1].contiguous()
        _weigh(c, t + 1, token, _lse(c, t + 1, token), old=weights, known=t, weights=weights)
    once = c.cache.weigh(310, q, _lse(c, 310, q, vis), visible=vis)
    assert bool(((once - weights).abs() <= 1e-4 * once + 1e-6).all())
    assert bool(((weights.double().sum((1, 2)) - 310 * 14).abs() < 1.0).all())


@pytest.mark.parametrize("dtype,d", TYPES)
def test_weights_of_what_is_not_seen(lazyev_lib, dtype, d):
    """Keys that no token sees hold NaN and infinities; queries that see nothing hold them too; entries of no page."""
    c = Cache(lazyev_lib, dtype, d, 1, 2, 16, 200, seed=8)
    q = c.randn(1, 40, 14, d).to(c.dt)
    vis = c.randint(1, 150, 1, 40).int()
    vis[0, 7] = vis[0, 39] = 0
    lse = _lse(c, 200, q, vis)
    clean = c.cache.weigh(200, q, lse, visible=vis)
    dense = c.rows(c.k_pages).clone()
    q[0, 7], q[0, 39, 3] = math.nan, math.inf
    for at in range(150, 200):
        c.k_pages[c.table[0, at // 16].long(), :, at % 16] = (math.nan, math.inf, -math.inf)[at % 3]
    got = c.cache.weigh(200, q, lse, visible=vis)
    assert torch.equal(got, clean) and bool((got[:, :, 150:] == 0).all())
    # a token that sees a NaN has it, in that entry alone
    c.k_pages[c.table[0, 2].long(), 1, 5, 3] = math.nan
    got = c.cache.weigh(200, q, lse, visible=vis)
    assert bool(torch.isnan(got[0, 1, 37]))
    got[0, 1, 37] = clean[0, 1, 37]
    assert torch.equal(got, clean)
    c.k_pages[c.table[0, 2].long(), 1, 5, 3] = dense[0, 37, 1, 3]
    c.table[0, 3], c.table[0, 5] = -1, 10 ** 6
    old = torch.ones(1, 2, 200, device="cuda")
    got = c.cache.weigh(200, q, lse, visible=vis, old=old, decay=0.5)
    none = (torch.arange(200, device="cuda") // 16 == 3) | (torch.arange(200, device="cuda") // 16 == 5)
    assert bool((got[:, :, none] == 0.5).all())
    assert torch.equal(got[:, :, ~none], (clean + 0.5)[:, :, ~none])


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("n", [2, 40])
def test_a_row_whose_logsumexp_is_no_number(lazyev_lib, dtype, d, n):
    """It says nothing of the entries that it does not see."""
    c = Cache(lazyev_lib, dtype, d, 1, 2, 16, 200, seed=16)
    q = c.randn(1, n, 14, d).to(c.dt)
    vis = c.randint(100, 200, 1, n).int()
    vis[0, 1] = 33
    lse = _lse(c, 200, q, vis)
    clean = c.cache.weigh(200, q, lse, visible=vis)
    for odd in (math.nan, math.inf):
        lse[0, 1, 5] = odd
        got = c.cache.weigh(200, q, lse, visible=vis)
        assert torch.equal(got[0, 1], clean[0, 1]) and torch.equal(got[0, 0, 33:], clean[0, 0, 33:])
        assert bool(torch.isnan(got[0, 0, :33]).all()) if math.isnan(odd) else bool((got[0, 0, :33] <= clean[0, 0, :33]).all())


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("n", [1, 40])
def test_weights_with_rows_at_odd_addresses(lazyev_lib, dtype, d, n):
    c = Cache(lazyev_lib, dtype, d, 2, 2, 16, 500, seed=18)
    q = c.randn(2, n, 14, d).to(c.dt)
    lse, old = _lse(c, 500, q), c.randn(2, 2, 500).exp()
    want = c.cache.weigh(500, q, lse, old=old, decay=0.5)
    got = c.cache.weigh(500, _off_by_one(q), _off_by_one(lse), old=_off_by_one(old), decay=0.5, weights=_off_by_one(old))
    assert torch.equal(got, want)


def test_weights_of_nothing(lazyev_lib):
    c = Cache(lazyev_lib, "bf16", 128, 2, 4, 16, 100, seed=9)
    q = c.randn(2, 3, 28, 128).bfloat16()
    lse = _lse(c, 100, q)
    old = c.randn(2, 4, 100)
    assert torch.equal(c.cache.weigh(100, q[:, :0], lse[:, :0], old=old, decay=0.5), 0.5 * old)        # no token
    junk = torch.full_like(old, math.nan)
    assert torch.equal(c.cache.weigh(100, q, lse, old=junk, decay=0.0, weights=junk), c.cache.weigh(100, q, lse))   # nothing of what was before
    assert torch.equal(c.cache.weigh(100, q[:, :0], lse[:, :0], old=junk.fill_(math.inf), decay=0.0), torch.zeros_like(old))
    assert c.cache.weigh(0, q, lse).shape == (2, 4, 0)                                                 # no entry
    assert torch.equal(c.cache.weigh(100, q, torch.full_like(lse, -math.inf), old=old), old)           # nothing seen
    assert bool((c.cache.weigh(100, q, torch.full_like(lse, math.inf)) == 0).all())


def test_weights_from_very_many_rows(lazyev_lib):
    """66400 rows of a KV head (more stages than a block lists at once), which see the first 300 of 32768 entries at most."""
    c = Cache(lazyev_lib, "bf16", 64, 1, 8, 256, 32768, seed=15)
    q = c.randn(1, 8300, 64, 64).bfloat16()
    vis = c.randint(0, 301, 1, 8300).int()
    vis[0, 100:5000] = 0
    lse = _lse(c, 300, q, vis)
    got = c.cache.weigh(32768, q, lse, visible=vis)
    assert bool((got[:, :, 300:] == 0).all())
    want, bound = long64.weigh(q[0], lse[0], c.rows(c.k_pages)[0, :300], vis[0].long(), 0.125)
    assert bool(((got[0, :, :300].double() - want).abs() <= bound + U * want.abs() + 1e-30).all())


# ------------------------------------------------------------------------------------ eviction

def _evict(c, length, weights, keep, recent=0, first=0, positions=None, lengths=None, in_place=False, no_page=()):
    before = [x.clone() for x in (c.k_pages, c.v_pages)]
    w0, p0 = weights.clone(), None if positions is None else positions.clone()
    more = dict(weights_out=weights, positions_out=positions) if in_place else {}
    sources, w, p = c.cache.evict(length, weights, keep, recent=recent, first=first, positions=positions, lengths=lengths, **more)
    S, H = weights.shape[:2]
    page = c.k_pages.shape[2]
    host_w, host_p, table = w0.cpu().numpy(), None if p0 is None else p0.cpu().numpy(), c.table.cpu().numpy()
    moves = 0
    for s in range(S):
        n = length if lengths is None else min(max(int(lengths[s]), 0), length)
        for h in range(H):
            want = long64.evict(host_w[s, h], None if host_p is None else host_p[s, h], n, keep, recent, first)
            assert np.array_equal(sources[s, h].cpu().numpy(), want), (s, h, n)
            some = torch.tensor(want >= 0, device="cuda")
            at = torch.tensor(np.maximum(want, 0), device="cuda")
            assert torch.equal(w[s, h, :keep], torch.where(some, w0[s, h][at], 0.0)) or bool(torch.isnan(w0[s, h]).any())
            assert torch.equal(w[s, h, :keep].nan_to_num(nan=3.5), torch.where(some, w0[s, h][at], 0.0).nan_to_num(nan=3.5))
            assert torch.equal(p[s, h, :keep], torch.where(some, at.int() if p0 is None else p0[s, h][at], -1))
            to = np.flatnonzero(want > np.arange(keep))
            to = np.array([x for x in to if x // page not in no_page and want[x] // page not in no_page], dtype=np.int64)
            come = want[to]
            for x in before:
                x[table[s, to // page].astype(np.int64), h, to % page] = x[table[s, come // page].astype(np.int64), h, come % page]
            moves += len(to)
    # rows that nothing moved to, those behind `keep` among them, are as they were
    assert torch.equal(c.k_pages, before[0]) and torch.equal(c.v_pages, before[1])
    if in_place:
        assert torch.equal(weights[:, :, keep:].nan_to_num(), w0[:, :, keep:].nan_to_num())
    return moves


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("S,H,page,length,keep,recent,first", [
    (1, 1, 16, 1, 1, 0, 0), (1, 1, 16, 2, 1, 0, 0), (1, 2, 16, 2, 1, 1, 0), (2, 4, 16, 130, 64, 8, 4), (1, 3, 24, 65, 64, 64, 0), (2, 2, 1, 40, 39, 0, 39), (1, 8, 500, 1025, 1024, 64, 4),
    (3, 2, 48, 2112, 2048, 64, 0), (1, 2, 128, 5000, 1000, 100, 10), (1, 1, 64, 100, 64, 20, 3), (1, 1, 4096, 4097, 4096, 4095, 1)])
def test_eviction(lazyev_lib, dtype, d, S, H, page, length, keep, recent, first):
    c = Cache(lazyev_lib, dtype, d, S, H, page, length, seed=10)
    weights = c.randn(S, H, length + 2).exp()
    assert _evict(c, length, weights, keep, recent, first) >= min(recent, length - keep)
    coarse = torch.floor(2 * weights) / 2          # many alike
    _evict(c, length, coarse, keep, recent, first)
    positions = torch.rand((S, H, length + 2), generator=c.gen, device="cuda").argsort(-1).int() * 2
    _evict(c, length, coarse, keep, recent, first, positions=positions)
    lengths = c.randint(0, length + 1, S).int()
    lengths[0] = length
    _evict(c, length, weights, keep, recent, first, lengths=lengths)
    _evict(c, length, coarse, keep, recent, first, positions=positions, lengths=lengths, in_place=True)


@pytest.mark.parametrize("length,keep", [(12000, 3000), (16384, 16000), (20000, 6000), (32768, 32000), (32769, 300), (50000, 49000), (65536, 30000), (65537, 30000), (40001, 5000), (100003, 90000)])
def test_eviction_of_long_caches(lazyev_lib, length, keep):
    c = Cache(lazyev_lib, "bf16", 64, 1, 2, 256, length, seed=11)
    weights = torch.floor(4 * c.randn(1, 2, length).exp()) / 4
    _evict(c, length, weights, keep, 256, 4)
    _evict(c, length, weights, keep, 256, 4, positions=torch.rand((1, 2, length), generator=c.gen, device="cuda").argsort(-1).int(), in_place=True)


def test_odd_weights(lazyev_lib):
    c = Cache(lazyev_lib, "bf16", 128, 1, 2, 16, 300, seed=12)
    weights = c.randn(1, 2, 300)
    weights[0, 0, ::7], weights[0, 0, 1::11], weights[0, 0, 2::13] = math.nan, math.inf, -math.inf
    weights[0, 1] = 0.0
    weights[0, 1, ::2] = -0.0                      # (one value)
    for keep in (1, 43, 60, 150, 290):
        _evict(c, 300, weights, keep, recent=1 if keep > 1 else 0)
    weights[:] = math.nan
    _evict(c, 300, weights, 100, 3, 3)
    _evict(c, 300, torch.full_like(weights, -math.inf), 100, 3, 3)


def test_eviction_from_nothing(lazyev_lib):
    c = Cache(lazyev_lib, "bf16", 128, 2, 4, 16, 100)
    for weights in (torch.zeros(2, 4, 0, device="cuda"), torch.zeros(2, 4, 7, device="cuda")):
        sources, w, p = c.cache.evict(0, weights, 5)
        assert bool((sources == -1).all()) and bool((w == 0).all()) and bool((p == -1).all())


def test_positions_of_all_kinds(lazyev_lib):
    c = Cache(lazyev_lib, "fp32", 64, 2, 2, 16, 200, seed=13)
    weights = c.randn(2, 2, 200).exp()
    for positions in (torch.full((2, 2, 200), 5), torch.arange(200, 0, -1).expand(2, 2, 200), torch.arange(200).expand(2, 2, 200) - 2 ** 31,
                      torch.arange(200).expand(2, 2, 200) + (2 ** 31 - 200)):
        positions = positions.to(torch.int32).cuda().contiguous()
        for recent, first in ((0, 0), (70, 0), (0, 70), (30, 40)):
            _evict(c, 200, weights, 70, recent, first, positions=positions)


def test_places_of_no_page(lazyev_lib):
    c = Cache(lazyev_lib, "bf16", 128, 1, 2, 16, 320, seed=14)
    c.table[0, 1], c.table[0, 15] = -1, 10 ** 6
    _evict(c, 320, c.randn(1, 2, 320), 100, 5, 2, no_page=(1, 15))


def test_the_binding_refuses(lazyev_lib):
    c = Cache(lazyev_lib, "bf16", 128, 2, 4, 16, 100)
    q = c.randn(2, 3, 28, 128).bfloat16()
    lse, w = torch.zeros(2, 3, 28, device="cuda"), torch.zeros(2, 4, 100, device="cuda")
    for bad in (dict(length=200), dict(q=q.float()), dict(lse=lse[:1]), dict(lse=lse.double()), dict(weights=w[:, :, :99]), dict(weights=w.double()),
                dict(old=w[:1]), dict(known=5), dict(old=w, known=101), dict(old=w, known=-1), dict(weights=w, old=torch.zeros(2, 4, 101, device="cuda")),
                dict(visible=torch.zeros(2, 3, device="cuda")), dict(weights=w.transpose(0, 1))):
        with pytest.raises(ValueError):
            c.cache.weigh(**{"length": 100, "q": q, "lse": lse, **bad})
    for bad in (dict(length=200), dict(keep=0), dict(recent=51), dict(recent=30, first=30), dict(recent=-1), dict(weights=w[:, :, :99]), dict(weights=w.int()),
                dict(positions=w), dict(positions=w.int()[:, :, :100].repeat(1, 1, 2)), dict(lengths=torch.zeros(2, device="cuda")),
                dict(lengths=torch.zeros(3, device="cuda").int()), dict(sources=torch.zeros(2, 4, 49, device="cuda").int()),
                dict(weights_out=torch.zeros(2, 4, 49, device="cuda")), dict(positions_out=torch.zeros(2, 4, 50, device="cuda"))):
        with pytest.raises(ValueError):
            c.cache.evict(**{"length": 100, "weights": w, "keep": 50, **bad})
