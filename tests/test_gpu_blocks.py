"""Bounds of a cache's blocks, the choice of blocks and attention over them, against their definitions in 64 bits: head groups, block and page
sizes, what a token sees, blocks that nearly tie, infinities and NaN, numbers that are no block."""
import math

import pytest
import torch

import long64
import plain64

pytestmark = pytest.mark.gpu

TYPES = [("bf16", 128), ("bf16", 64), ("fp32", 128), ("fp32", 64)]


def _dt(name):
    return torch.float32 if name == "fp32" else torch.bfloat16


class Cache:
    """Random pages with a table whose rows share none, and the dense rows."""

    def __init__(self, b, dtype, d, S, H, page, entries, seed=0):
        self.b, self.dt, self.S, self.H, self.d, self.entries = b, _dt(dtype), S, H, d, entries
        self.gen = torch.Generator(device="cuda").manual_seed(1000 * seed + 7 * entries + page)
        m = max(1, -(-entries // page))
        self.table = torch.randperm(S * m + 2, generator=self.gen, device="cuda")[:S * m].view(S, m).int()
        self.k_pages, self.v_pages = (self.randn(S * m + 2, H, page, d).to(self.dt) for _ in range(2))
        self.cache = b.PagedCache(self.k_pages, self.v_pages, self.table)

    def randn(self, *shape):
        return torch.randn(shape, generator=self.gen, device="cuda")

    def randint(self, lo, hi, *shape):
        return torch.randint(lo, hi, shape, generator=self.gen, device="cuda")

    def rows(self, pages):                         # [S, entries, H, d]
        return pages[self.table.long()].transpose(2, 3).flatten(1, 2)[:, :self.entries]


# ------------------------------------------------------------------------------------ bounds

def _bounds_of(k, block):
    """k [S, n, H, d] -> [S, H, blocks, 2, d]"""
    n = k.shape[1]
    return torch.stack([torch.stack((k[:, i:i + block].amin(1), k[:, i:i + block].amax(1)), 2) for i in range(0, n, block)], 2)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("S,H,page,entries,block", [(1, 1, 16, 1, 16), (2, 3, 16, 17, 16), (1, 8, 24, 200, 32), (3, 2, 1, 70, 16), (2, 4, 500, 700, 64),
                                                    (1, 2, 64, 1000, 128), (1, 5, 4096, 333, 128)])
def test_bounds(lazyev_lib, dtype, d, S, H, page, entries, block):
    c = Cache(lazyev_lib, dtype, d, S, H, page, entries)
    want = _bounds_of(c.rows(c.k_pages), block)
    n_blocks = want.shape[2]
    junk = c.randn(S, H, n_blocks + 2, 2, d).to(c.dt)
    whole = lazyev_lib.KeyBounds(junk.clone(), block)
    whole.update(c.cache, 0, entries)
    assert torch.equal(whole.bounds[:, :, :n_blocks], want) and torch.equal(whole.bounds[:, :, n_blocks:], junk[:, :, n_blocks:])
    whole.update(c.cache, 0, 0)                    # nothing
    # in pieces, as entries are appended: lengths from one on
    pieces = lazyev_lib.KeyBounds(junk.clone(), block)
    at = 0
    for n in [1, 1, 3, block, 2 * block + 1, 7] * 50:
        n = min(n, entries - at)
        pieces.update(c.cache, at, n)
        at += n
        if n:
            seen = _bounds_of(c.rows(c.k_pages)[:, :at], block)
            assert torch.equal(pieces.bounds[:, :, :seen.shape[2]], seen)
            assert torch.equal(pieces.bounds[:, :, seen.shape[2]:], junk[:, :, seen.shape[2]:])
    assert at == entries


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_bounds_of_odd_keys(lazyev_lib, dtype):
    c = Cache(lazyev_lib, dtype, 64, 1, 2, 16, 160, seed=1)
    c.k_pages[c.table[0, 0].long(), 0, 3, 5] = math.nan
    c.k_pages[c.table[0, 1].long(), 1, 2, 7] = math.inf
    c.k_pages[c.table[0, 1].long(), 1, 9, 7] = -math.inf
    c.table[0, 4] = -1                             # no page: entries 64 .. 79, half of the block 2, and a whole block
    c.table[0, 6:8] = 10 ** 6
    x = lazyev_lib.KeyBounds.of(c.cache, 32)
    x.bounds.fill_(7)
    x.update(c.cache, 0, 160)
    k = c.k_pages[c.table.long().clamp(0, c.k_pages.shape[0] - 1)].transpose(2, 3).flatten(1, 2)
    want = _bounds_of(k, 32)
    want[:, :, 2] = _bounds_of(k[:, 80:96], 32)[:, :, 0]
    want[:, :, 3, 0], want[:, :, 3, 1] = math.inf, -math.inf
    assert torch.equal(torch.isnan(x.bounds), torch.isnan(want))
    assert torch.equal(x.bounds.nan_to_num(nan=5.0), want.nan_to_num(nan=5.0))
    x.update(c.cache, 33, 1)                       # a NaN or infinity stays when its block is extended
    x.update(c.cache, 5, 1)
    assert torch.equal(x.bounds.nan_to_num(nan=5.0), want.nan_to_num(nan=5.0))


# ------------------------------------------------------------------------------------ choice

def _choose(c, bounds, block, length, q, chosen, visible=None, first=0, last=1):
    S, n, Hq, d = q.shape
    x = c.KeyBounds(bounds, block)
    got = x.choose(length, q, chosen, visible=visible, first=first, last=last)
    for s in range(S):
        seen = torch.full((n,), length) if visible is None else visible[s].clamp(0, length)
        want = long64.choose(long64.scores(q[s], bounds[s]), seen.tolist(), block, first, last, chosen)
        assert torch.equal(got[s].cpu(), want), (s, (got[s].cpu() != want).nonzero()[:5])
    return got


def _bounds(gen, S, H, n, d, dt):
    x = torch.randn((2, S, H, n, d), generator=gen, device="cuda")
    mid = torch.randn((S, H, n, d), generator=gen, device="cuda")
    return torch.stack((mid - x[0].abs(), mid + x[1].abs()), 3).to(dt)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("S,n,Hq,H,length,block,chosen,first,last", [
    (1, 1, 1, 1, 1, 16, 1, 0, 1), (1, 1, 1, 1, 33, 16, 2, 0, 1), (2, 1, 28, 4, 5003, 16, 20, 1, 2), (1, 3, 8, 8, 700, 32, 5, 0, 1), (1, 33, 6, 2, 2000, 16, 9, 2, 3),
    (2, 5, 32, 1, 1000, 16, 8, 0, 2), (1, 2, 64, 1, 900, 16, 3, 1, 1), (1, 7, 33, 1, 900, 16, 30, 1, 1), (1, 9, 9, 3, 1111, 128, 3, 0, 1), (1, 70, 5, 1, 640, 64, 4, 1, 1),
    (3, 17, 32, 2, 300, 16, 7, 3, 4), (1, 40, 2, 1, 4000, 16, 250, 0, 1), (1, 2, 12, 1, 40000, 16, 600, 1, 2), (1, 1, 4, 4, 1000, 16, 1000, 1, 1), (1, 600, 2, 2, 500, 32, 6, 1, 1)])
def test_choice(lazyev_lib, dtype, d, S, n, Hq, H, length, block, chosen, first, last):
    gen = torch.Generator(device="cuda").manual_seed(length + n)
    dt = _dt(dtype)
    bounds = _bounds(gen, S, H, -(-length // block) + 1, d, dt)
    q = torch.randn((S, n, Hq, d), generator=gen, device="cuda").to(dt)
    _choose(lazyev_lib, bounds, block, length, q, chosen, first=first, last=last)
    vis = torch.randint(0, length + 1, (S, n), generator=gen, device="cuda").int()
    vis[:, ::5], vis[:, 1::5] = 0, length + 100
    vis[:, 2::9] = -4
    _choose(lazyev_lib, bounds, block, length, q, chosen, visible=vis, first=first, last=last)
    past = torch.arange(length - n + 1, length + 1, device="cuda").clamp(min=0).int().expand(S, n).contiguous()
    _choose(lazyev_lib, bounds, block, length, q, chosen, visible=past, first=first, last=last)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("n_blocks", [40, 400, 700, 1500, 3000, 5000, 12000])
def test_scores_that_nearly_tie(lazyev_lib, dtype, d, n_blocks):
    """One large sum in all blocks and a difference that sums in 32 bits lose (2^15 and multiples of 2^-12); equal blocks among them."""
    gen = torch.Generator(device="cuda").manual_seed(n_blocks)
    dt = _dt(dtype)
    bounds = torch.full((1, 2, n_blocks, 2, d), 256.0, device="cuda")
    bounds[..., d // 2] = torch.randint(-100, 100, (1, 2, n_blocks, 1), generator=gen, device="cuda") * 2.0 ** -12
    bounds[..., 3] = 32768.0 - 256.0 * (d - 2)
    q = torch.ones((1, 3, 4, d), device="cuda")
    q[:, 1, ::2] = -1.0                            # (both signs in one group)
    q[:, 2, :] = torch.randn((4, d), generator=gen, device="cuda")
    for chosen in (2, n_blocks // 2, n_blocks - 2):
        _choose(lazyev_lib, bounds.to(dt), 16, 16 * n_blocks, q.to(dt), chosen)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("n_blocks", [30, 400, 900, 1500, 3000, 6000, 9000])
def test_equal_scores_go_by_their_numbers(lazyev_lib, dtype, d, n_blocks):
    gen = torch.Generator(device="cuda").manual_seed(5)
    dt = _dt(dtype)
    few = _bounds(gen, 1, 2, 7, d, dt)
    bounds = few[:, :, torch.randint(0, 7, (n_blocks,), generator=gen, device="cuda")].contiguous()
    q = torch.randn((1, 4, 6, d), generator=gen, device="cuda").to(dt)
    q[:, 1] = 0                                    # every score is zero
    q[:, 2, 3:] = -0.0
    for chosen in (5, n_blocks - 3):
        got = _choose(lazyev_lib, bounds, 16, 16 * n_blocks, q, chosen, first=1, last=2)
        assert got[0, 1, 0].tolist() == list(range(chosen - 2)) + [n_blocks - 2, n_blocks - 1]
    _choose(lazyev_lib, few[:, :, :1].expand(1, 2, n_blocks, 2, d).contiguous(), 16, 16 * n_blocks, q, 8)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_choice_of_very_many_blocks(lazyev_lib, dtype):
    """More blocks than a row's registers hold; then many tokens, whose scores come in several turns."""
    gen = torch.Generator(device="cuda").manual_seed(9)
    dt = _dt(dtype)
    bounds = _bounds(gen, 1, 2, 17000, 64, dt)
    bounds[:, :, 5000:5300] = bounds[:, :, 100:400]
    q = torch.randn((1, 3, 4, 64), generator=gen, device="cuda").to(dt)
    q[:, 2] = 0
    for chosen in (7, 900):
        _choose(lazyev_lib, bounds, 16, 16 * 17000, q, chosen, first=2, last=2)
    bounds = _bounds(gen, 1, 8, 4100, 64, dt)
    q = torch.randn((1, 300, 8, 64), generator=gen, device="cuda").to(dt)
    size = lazyev_lib.lib.lazyev_blocks_choose_workspace(lazyev_lib.KeyBounds(bounds, 16).blocks, 16 * 4100, 300, 8, 1, 33)
    assert size < 300 * 8 * 4098 * 12              # (not for all of them at once)
    _choose(lazyev_lib, bounds, 16, 16 * 4100, q, 33)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("n_blocks", [250, 500, 1000, 2000, 4000])
def test_choice_of_many_tokens(lazyev_lib, dtype, d, n_blocks):
    gen = torch.Generator(device="cuda").manual_seed(n_blocks)
    dt = _dt(dtype)
    bounds = _bounds(gen, 2, 2, n_blocks, d, dt)
    bounds[:, :, 100:120] = bounds[:, :, 150:170]
    q = torch.randn((2, 150, 6, d), generator=gen, device="cuda").to(dt)
    q[:, 5] = q[:, 6, :1]
    vis = torch.randint(0, 16 * n_blocks + 1, (2, 150), generator=gen, device="cuda").int()
    for visible in (None, vis):
        _choose(lazyev_lib, bounds, 16, 16 * n_blocks, q, 33, visible=visible, first=1, last=2)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_choice_by_odd_numbers(lazyev_lib, dtype):
    """Infinities, NaN, blocks of nothing, sums that leave the range of 32 bits, elements too small for a product of 32 bits."""
    gen = torch.Generator(device="cuda").manual_seed(6)
    dt, d = _dt(dtype), 64
    bounds = _bounds(gen, 1, 2, 60, d, dt)
    q = torch.randn((1, 6, 4, d), generator=gen, device="cuda").to(dt)
    q[:, 1, 0, 5] = math.nan
    q[:, 2, 0, 5] = math.inf
    q[:, 3] *= 1e-25
    q[:, 4, :, 9] = 0.0
    q[:, 5, :, ::2] = 0.0
    odd = bounds.clone()
    odd[0, 0, 7, 1, 3], odd[0, 0, 9, 0, 3] = math.inf, -math.inf
    odd[0, 0, 11, :, 4] = math.nan
    odd[0, 1, 13, 0], odd[0, 1, 13, 1] = math.inf, -math.inf          # a block of no entries
    odd[0, 1, 20, 1, :] = 3e38                                          # sums beyond fp32 ...
    odd[0, 1, 21, 1, :] = 2.9e38                                        # ... that differ
    tiny = (bounds.float() * 1e-25).to(dt)
    for x in (bounds, odd, tiny):
        for chosen in (3, 20, 57):
            _choose(lazyev_lib, x, 16, 960, q, chosen, first=1, last=1)


def test_blocks_that_nobody_ranks_have_no_influence(lazyev_lib):
    gen = torch.Generator(device="cuda").manual_seed(7)
    bounds = _bounds(gen, 2, 4, 100, 128, torch.bfloat16)
    q = torch.randn((2, 3, 28, 128), generator=gen, device="cuda").bfloat16()
    vis = torch.tensor([[500, 16 * 60, 700], [16 * 60, 3, 950]], device="cuda").int()
    x = lazyev_lib.KeyBounds(bounds, 16)
    want = x.choose(1600, q, 9, visible=vis, first=1, last=1)
    bounds[:, :, 59:] = math.nan                   # the last one of those seen is not ranked
    assert torch.equal(x.choose(1600, q, 9, visible=vis, first=1, last=1), want)
    # a call of its own for one token has the same answer
    alone = x.choose(960, q[:, 1:2].contiguous(), 9, visible=vis[:, 1:2].contiguous(), first=1, last=1)
    assert torch.equal(alone, want[:, 1:2])


def test_choice_with_queries_at_odd_addresses(lazyev_lib):
    gen = torch.Generator(device="cuda").manual_seed(8)
    for dt, d in ((torch.bfloat16, 128), (torch.float32, 64)):
        bounds = _bounds(gen, 1, 2, 50, d, dt)
        flat = torch.randn(1 + 4 * 6 * d, generator=gen, device="cuda").to(dt)
        q = flat[1:].view(1, 4, 6, d)
        _choose(lazyev_lib, bounds, 16, 800, q, 7)


# ------------------------------------------------------------------------------------ attention

def _attend(c, length, q, blocks, block, visible=None, joined=None, scale=0.0, there=None, **more):
    out, lse = c.cache.attend_blocks(length, q, blocks, block, visible=visible, joined=joined, scale=scale, **more)
    k, v = c.rows(c.k_pages), c.rows(c.v_pages)
    S, n, Hq, d = q.shape
    G = Hq // c.H
    # (of many tokens the first and the last ones, and every eleventh)
    for s in range(S):
        for i in range(n) if n <= 60 else sorted({*range(12), *range(n - 12, n), *range(0, n, 11)}):
            end = length if visible is None else min(max(int(visible[s, i]), 0), length)
            for h in range(c.H):
                at = [torch.arange(x * block, min(x * block + block, end), device="cuda") for x in blocks[s, i, h].tolist() if 0 <= x and x * block < end]
                at = torch.cat(at) if at else torch.zeros(0, dtype=torch.long, device="cuda")
                if there is not None:
                    at = at[there[s][at]]
                mine = slice(h * G, (h + 1) * G)
                want = plain64.attend(q[s, i:i + 1, mine], k[s, at, h:h + 1], v[s, at, h:h + 1], torch.full((1,), len(at), device="cuda"), scale or d ** -0.5,
                                      None if joined is None else (joined[0][s, i:i + 1, mine], joined[1][s, i:i + 1, mine]))
                plain64.check_out(out[s, i:i + 1, mine], want[0], want[2])
                plain64.check_lse(lse[s, i:i + 1, mine], want[1], want[3])
    return out, lse


def _some_blocks(c, n, length, block, m):
    """Ascending numbers, some of them -1 at the end."""
    n_blocks = -(-length // block)
    order = torch.rand((c.S, n, c.H, n_blocks), generator=c.gen, device="cuda").argsort(-1)[..., :m]
    blocks = torch.full((c.S, n, c.H, m), n_blocks, device="cuda")
    blocks[..., :order.shape[-1]] = order
    blocks = blocks.sort(-1).values
    return torch.where(blocks < n_blocks, blocks, -1).int()


SHAPES = [  # tables, tokens, query and KV heads, page, length, block, chosen
    (1, 1, 1, 1, 16, 1, 16, 1), (2, 1, 28, 4, 16, 333, 16, 5), (1, 1, 7, 1, 24, 1000, 32, 9), (3, 5, 8, 8, 1, 77, 16, 4), (1, 4, 64, 1, 64, 600, 64, 3),
    (2, 3, 33, 1, 48, 500, 16, 12), (1, 2, 6, 2, 4096, 3000, 128, 20), (1, 33, 10, 2, 32, 900, 64, 6), (1, 1, 8, 1, 128, 9000, 16, 300), (1, 2, 5, 1, 100, 2000, 128, 3),
    # many units: tiles of tokens share their lists; tiles that the tokens do not fill, pages that end inside blocks, groups of 1 to 64 heads
    (1, 259, 7, 1, 64, 700, 64, 4), (2, 71, 6, 2, 32, 900, 32, 9), (3, 5, 160, 20, 16, 500, 16, 6), (1, 300, 1, 1, 24, 333, 16, 7), (1, 131, 32, 2, 1, 130, 16, 3),
    (1, 270, 64, 1, 128, 600, 128, 2), (4, 2, 99, 33, 48, 1000, 64, 12), (1, 33, 40, 8, 64, 5000, 32, 50), (1, 257, 4, 1, 256, 2100, 128, 17),
    # runs of single entries: more of them than a block looks up at once
    (1, 2, 4, 1, 5, 4000, 16, 100), (1, 200, 8, 2, 3, 3000, 16, 10)]


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("S,n,Hq,H,page,length,block,m", SHAPES)
def test_attention(lazyev_lib, dtype, d, S, n, Hq, H, page, length, block, m):
    c = Cache(lazyev_lib, dtype, d, S, H, page, length, seed=2)
    q = (1.5 * c.randn(S, n, Hq, d)).to(c.dt)
    blocks = _some_blocks(c, n, length, block, m)
    plain = _attend(c, length, q, blocks, block)
    vis = c.randint(0, length + 1, S, n).int()
    vis[:, ::4] = length
    if n > 1:
        vis[:, 1::6], vis[:, 2::7], vis[:, 3::7] = 0, -3, length + 50
    joined = ((0.3 * c.randn(S, n, Hq, d)).to(c.dt), 2 * c.randn(S, n, Hq))
    joined[1][:, ::3, ::2] = -math.inf             # nothing there ...
    joined[0][:, ::3, ::2] = math.nan              # ... whatever it says
    got = _attend(c, length, q, blocks, block, visible=vis, joined=joined, scale=0.2)
    same = c.cache.attend_blocks(length, q, blocks, block, visible=vis, joined=joined, out=joined[0], lse=joined[1], scale=0.2)
    assert torch.equal(same[0], got[0]) and torch.equal(same[1], got[1]) and same[0] is joined[0]
    assert all(torch.equal(x, y) for x, y in zip(c.cache.attend_blocks(length, q, blocks, block), plain))


def _off_by_one(x):
    """The same elements, one element behind an aligned address."""
    flat = torch.empty(1 + x.numel(), dtype=x.dtype, device="cuda")
    flat[1:] = x.flatten()
    return flat[1:].view(x.shape)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("n,H", [(3, 2), (40, 7)])
def test_attention_with_rows_at_odd_addresses(lazyev_lib, dtype, d, n, H):
    c = Cache(lazyev_lib, dtype, d, 1, H, 16, 300, seed=17)
    q = c.randn(1, n, 3 * H, d).to(c.dt)
    blocks = _some_blocks(c, n, 300, 16, 5)
    joined = (c.randn(1, n, 3 * H, d).to(c.dt), c.randn(1, n, 3 * H))
    want = c.cache.attend_blocks(300, q, blocks, 16, joined=joined)
    odd = tuple(_off_by_one(x) for x in joined)
    got = c.cache.attend_blocks(300, _off_by_one(q), _off_by_one(blocks), 16, joined=odd, out=_off_by_one(q), lse=_off_by_one(joined[1]))
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    got = c.cache.attend_blocks(300, q, blocks, 16, joined=odd, out=odd[0], lse=odd[1])
    assert all(torch.equal(x, y) for x, y in zip(got, want))


# (one token's lists on their own; 40 tokens of 7 KV heads and so on: tiles of tokens)
@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("n,H", [(4, 2), (40, 7)])
def test_numbers_that_are_no_block_and_numbers_twice(lazyev_lib, dtype, d, n, H):
    c = Cache(lazyev_lib, dtype, d, 2, H, 16, 300, seed=3)
    q = c.randn(2, n, 3 * H, d).to(c.dt)
    blocks = _some_blocks(c, n, 300, 16, 11)
    blocks[:, 0] = -1                              # no block at all
    blocks[:, 1, :, ::2] = torch.tensor([19, 2 ** 31 - 1, -2 ** 31, 10 ** 6, -7, 1 << 27], device="cuda").int()     # 0 .. 18 are blocks
    blocks[:, 2, :, 3] = blocks[:, 2, :, 4]        # twice
    blocks[:, 3] = blocks[:, 3].flip(-1)           # in another order
    if n > 20:
        blocks[:, 20, :, :] = 5                    # eleven times
    first = _attend(c, 300, q, blocks, 16)
    again = c.cache.attend_blocks(300, q, blocks, 16)
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    vis = c.randint(0, 300, 2, n).int()
    vis[0, :4], vis[1, :4] = torch.tensor([295, 200, 290, 17], device="cuda").int(), torch.tensor([1, 16, 289, 0], device="cuda").int()
    _attend(c, 295, q, blocks, 16, visible=vis)
    _attend(c, 0, q, blocks, 16)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("n,H", [(3, 2), (50, 6)])
@pytest.mark.parametrize("block,page", [(16, 16), (64, 24), (32, 64)])
def test_entries_of_no_page(lazyev_lib, dtype, d, block, page, n, H):
    c = Cache(lazyev_lib, dtype, d, 1, H, page, 700, seed=4)
    dense = c.rows(c.k_pages), c.rows(c.v_pages)
    c.table[0, 1], c.table[0, -2] = -1, 10 ** 6
    there = [(torch.arange(700, device="cuda") // page != 1) & (torch.arange(700, device="cuda") // page != c.table.shape[1] - 2)]
    c.rows = lambda pages: dense[0] if pages is c.k_pages else dense[1]
    q = c.randn(1, n, 3 * H, d).to(c.dt)
    blocks = _some_blocks(c, n, 700, block, 8)
    blocks[:, :, :, 0] = page // block
    _attend(c, 700, q, blocks, block, there=there)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("many", [1, 30])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_what_a_token_does_not_see_has_no_influence(lazyev_lib, dtype, d, value, many):
    """Entries of other blocks, those of a listed block behind what the token sees, and those behind the length."""
    c = Cache(lazyev_lib, dtype, d, 1, 2, 24, 500, seed=5)
    n = 6 * many                                   # (30: tiles of tokens)
    q = c.randn(1, n, 14, d).to(c.dt)
    blocks = torch.tensor([0, 3, 7, 12, -1], device="cuda").int().expand(1, n, 2, 5).contiguous()
    blocks[:, ::2, :, 4] = 10
    vis = torch.tensor([[500, 402, 385, 120, 7, 397]], device="cuda").int().repeat(1, many)
    clean = c.cache.attend_blocks(450, q, blocks, 32, visible=vis)
    for at in list(range(32, 96)) + list(range(416, 500)) + list(range(402, 416)):
        if at >= 416 or at < 402:
            c.k_pages[c.table[0, at // 24].long(), :, at % 24] = value
        c.v_pages[c.table[0, at // 24].long(), :, at % 24] = value
    got = c.cache.attend_blocks(450, q, blocks, 32, visible=vis)
    low = vis[0] <= 402
    assert torch.equal(got[0][:, low], clean[0][:, low]) and torch.equal(got[1], clean[1])
    assert bool((~torch.isfinite(got[0][:, ~low])).all())
    only = c.cache.attend_blocks(450, q, blocks[..., :3].contiguous(), 32)       # (none of them listed)
    assert bool(torch.isfinite(only[0]).all())
    # a value that some tokens of a tile read, in a column of its own: theirs and nobody else's
    c.v_pages[c.table[0, 321 // 24].long(), :, 321 % 24, 5] = value               # (of block 10)
    got = c.cache.attend_blocks(400, q, blocks, 32)
    assert bool((~torch.isfinite(got[0][:, ::2, :, 5])).all()) and bool(torch.isfinite(got[0][:, 1::2]).all())
    others = torch.arange(d, device="cuda") != 5
    assert bool(torch.isfinite(got[0][..., others]).all())


def test_tokens_that_share_a_tile_do_not_see_one_another(lazyev_lib):
    """A token's bits depend on its own list and queries alone: other tokens' lists, values and order in the tile change nothing."""
    for dtype, d in TYPES:
        c = Cache(lazyev_lib, dtype, d, 1, 4, 32, 2000, seed=20)
        n = 90
        q = c.randn(1, n, 28, d).to(c.dt)
        blocks = _some_blocks(c, n, 2000, 32, 12)
        vis = c.randint(1500, 2001, 1, n).int()
        want = c.cache.attend_blocks(2000, q, blocks, 32, visible=vis)
        other_q, other_b = c.randn(1, n, 28, d).to(c.dt) * 3, blocks.clone()
        keep = torch.arange(n, device="cuda") % 3 == 1
        other_q[:, keep] = q[:, keep]
        mine = other_b[:, keep].clone()
        got = c.cache.attend_blocks(2000, other_q, other_b, 32, visible=vis)
        assert torch.equal(got[0][:, keep], want[0][:, keep]) and torch.equal(got[1][:, keep], want[1][:, keep]) and torch.equal(mine, blocks[:, keep])


def test_the_binding_refuses(lazyev_lib):
    c = Cache(lazyev_lib, "bf16", 128, 2, 4, 16, 100)
    q = c.randn(2, 3, 28, 128).bfloat16()
    x = lazyev_lib.KeyBounds.of(c.cache, 16)
    with pytest.raises(ValueError):
        lazyev_lib.KeyBounds.of(c.cache, 0)
    blocks = x.choose(0, q, 3)
    assert bool((blocks == -1).all())
    for bad in (dict(length=200), dict(length=-1), dict(q=q.float()), dict(q=q[:1]), dict(q=q.transpose(1, 2)), dict(n=0), dict(first=3), dict(last=0),
                dict(first=-1), dict(visible=torch.zeros(2, 3, device="cuda")), dict(visible=torch.zeros(2, 2, device="cuda").int()),
                dict(out=blocks[:, :, :, :2]), dict(workspace=torch.zeros(100, device="cuda"))):
        with pytest.raises(ValueError):
            x.choose(**{"length": 100, "q": q, "n": 3, **bad})
    for bad in (dict(blocks=blocks.long()), dict(blocks=blocks[:1]), dict(blocks=blocks[..., :2]), dict(block=24), dict(length=200), dict(q=q.float()),
                dict(out=q[:1]), dict(lse=torch.zeros(2, 3, device="cuda")), dict(joined=(q, torch.zeros(2, 3, device="cuda")))):
        with pytest.raises(ValueError):
            c.cache.attend_blocks(**{"length": 100, "q": q, "blocks": blocks, "block": 16, **bad})
    for bad in (dict(bounds=x.bounds[:, :, :, :1]), dict(bounds=x.bounds.half()), dict(bounds=x.bounds.transpose(1, 2)), dict(block=20)):
        with pytest.raises(ValueError):
            lazyev_lib.KeyBounds(**{"bounds": x.bounds, "block": 16, **bad})
    for start, n in ((-1, 2), (100, 30), (0, -1)):
        with pytest.raises(ValueError):
            x.update(c.cache, start, n)
    other = Cache(lazyev_lib, "bf16", 64, 2, 4, 16, 100)
    with pytest.raises(lazyev_lib.LazyevError):
        x.update(other.cache, 0, 10)
