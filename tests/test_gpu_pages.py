"""lazyev_pages_attend against 64 bits: single tokens and long prompts, head groups, page sizes, what a token sees (all, its past,
nothing), contexts joined with another part, and the places that a token does not see."""
import math

import pytest
import torch

import plain64

pytestmark = pytest.mark.gpu

TYPES = [("bf16", 128), ("bf16", 64), ("fp32", 128), ("fp32", 64)]


def _dt(name):
    return torch.float32 if name == "fp32" else torch.bfloat16


class Case:
    """Random pages with a table, queries of which each reads one entry strongly, and the dense rows."""

    def __init__(self, b, dtype, d, S, n, Hq, H, page, length, seed=0, extra=2):
        self.dt, self.S, self.n, self.Hq, self.H, self.length = _dt(dtype), S, n, Hq, H, length
        self.gen = torch.Generator(device="cuda").manual_seed(seed + 31 * n + length)
        m = max(1, -(-length // page))
        self.table = torch.randperm(S * m + extra, generator=self.gen, device="cuda")[:S * m].view(S, m).int()
        self.k_pages, self.v_pages = (self.randn(S * m + extra, H, page, d).to(self.dt) for _ in range(2))
        self.q = self.randn(S, n, Hq, d).to(self.dt)
        k = self.rows(self.k_pages)
        if length:
            read = torch.randint(0, length, (S, n), generator=self.gen, device="cuda")
            for s in range(S):
                self.q[s] += (0.4 * k[s][read[s]].float().repeat_interleave(Hq // H, 1)).to(self.dt)
        self.cache = b.PagedCache(self.k_pages, self.v_pages, self.table, n_q_heads=Hq)

    def randn(self, *shape):
        return torch.randn(shape, generator=self.gen, device="cuda")

    def rows(self, pages):                         # [S, length, H, d]
        return pages[self.table.long()].transpose(2, 3).flatten(1, 2)[:, :self.length]

    def check(self, got, visible=None, joined=None, scale=None, there=None):
        out, lse = got
        k, v = self.rows(self.k_pages), self.rows(self.v_pages)
        for s in range(self.S):
            vis = torch.full((self.n,), self.length, device="cuda") if visible is None else visible[s].long().clamp(0, self.length)
            want = plain64.attend(self.q[s], k[s], v[s], vis, scale or self.q.shape[-1] ** -0.5,
                                  None if joined is None else (joined[0][s], joined[1][s]), None if there is None else there[s])
            plain64.check_out(out[s], want[0], want[2])
            plain64.check_lse(lse[s], want[1], want[3])


SHAPES = [  # tables, tokens, query and KV heads, page, length
    (1, 1, 1, 1, 16, 1), (1, 1, 7, 1, 16, 15), (2, 1, 28, 4, 16, 17), (1, 5, 8, 8, 24, 64), (1, 3, 14, 2, 16, 1003),
    (1, 32, 28, 4, 64, 500), (3, 33, 8, 2, 48, 257), (1, 20, 32, 1, 128, 333), (2, 10, 64, 1, 1, 70), (1, 1, 8, 8, 32, 9001),
    (1, 150, 7, 1, 500, 700), (1, 600, 4, 2, 4096, 130), (2, 63, 5, 1, 17, 40), (1, 1, 28, 4, 256, 40000), (1, 257, 2, 2, 64, 129),
    # many rows: wide blocks, with splits of the entries and without
    (1, 600, 7, 1, 24, 130), (1, 600, 7, 1, 16, 700), (1, 900, 2, 1, 100, 1100), (1, 4500, 4, 1, 48, 130), (1, 9000, 1, 1, 32, 65), (1, 9000, 1, 1, 64, 700)]


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("S,n,Hq,H,page,length", SHAPES)
def test_all_entries(lazyev_lib, dtype, d, S, n, Hq, H, page, length):
    c = Case(lazyev_lib, dtype, d, S, n, Hq, H, page, length)
    got = c.cache.attend(length, c.q)
    c.check(got)
    joined = ((0.3 * c.randn(S, n, Hq, d)).to(c.dt), math.log(length) + 2 * c.randn(S, n, Hq))
    joined[1][:, ::3] = -math.inf                  # nothing there ...
    joined[0][:, ::3] = math.nan                   # ... whatever it says
    if n > 1:
        joined[1][:, 1] = 500.0                    # everything there
    want = joined[0].clone(), joined[1].clone()
    got = c.cache.attend(length, c.q, joined=joined)
    c.check(got, joined=want)
    assert torch.equal(joined[1], want[1])
    same = c.cache.attend(length, c.q, joined=joined, out=joined[0], lse=joined[1])
    assert torch.equal(same[0], got[0]) and torch.equal(same[1], got[1]) and same[0] is joined[0]


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("S,n,Hq,H,page,length", SHAPES)
def test_some_entries(lazyev_lib, dtype, d, S, n, Hq, H, page, length):
    """Any number of entries, none, fewer than none, more than there are."""
    c = Case(lazyev_lib, dtype, d, S, n, Hq, H, page, length, seed=1)
    vis = torch.randint(0, length + 1, (S, n), generator=c.gen, device="cuda").int()
    vis[:, ::5], vis[:, 1::5], vis[:, 2::7] = 0, -3, length + 1000
    c.check(c.cache.attend(length, c.q, visible=vis), visible=vis)
    joined = ((0.3 * c.randn(S, n, Hq, d)).to(c.dt), 3 * c.randn(S, n, Hq))
    joined[1][:, ::10] = -math.inf                 # neither here nor there
    c.check(c.cache.attend(length, c.q, visible=vis, joined=joined), visible=vis, joined=joined)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("S,P,Hq,H,page", [(1, 1, 2, 1, 16), (2, 65, 7, 1, 16), (1, 130, 8, 8, 30), (1, 700, 6, 2, 128), (1, 33, 28, 4, 64)])
def test_a_prompt_over_itself(lazyev_lib, dtype, d, S, P, Hq, H, page):
    c = Case(lazyev_lib, dtype, d, S, P, Hq, H, page, P, seed=2)
    vis = torch.arange(1, P + 1, device="cuda").int().expand(S, P).contiguous()
    c.check(c.cache.attend(P, c.q, visible=vis, scale=0.2), visible=vis, scale=0.2)


def test_nothing_to_read(lazyev_lib):
    c = Case(lazyev_lib, "bf16", 128, 1, 4, 8, 2, 16, 0)
    out, lse = c.cache.attend(0, c.q)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())
    joined = (c.randn(1, 4, 8, 128).bfloat16(), c.randn(1, 4, 8))
    out, lse = c.cache.attend(0, c.q, joined=joined)
    assert torch.equal(out, joined[0]) and torch.equal(lse, joined[1])
    none = c.cache.attend(0, c.q[:, :0])
    assert none[0].shape == (1, 0, 8, 128) and none[1].shape == (1, 0, 8)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("n,length,Hq,H", [(1, 100, 7, 1), (40, 300, 4, 2), (300, 400, 2, 1), (600, 700, 7, 1), (9000, 130, 1, 1)])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_what_a_token_does_not_see_has_no_influence(lazyev_lib, dtype, d, n, length, Hq, H, value):
    """Entries beyond what a token sees hold infinities and NaN, in keys and values; tokens that see such a value have it."""
    c = Case(lazyev_lib, dtype, d, 1, n, Hq, H, 16, length, seed=3)
    vis = torch.randint(1, length + 1, (1, n), generator=c.gen, device="cuda").int()
    vis[0, -1] = length // 2
    clean = c.cache.attend(length, c.q, visible=vis)
    first = length // 2                            # from here on
    dense = torch.arange(first, length, device="cuda")
    page = c.table[0].long()[dense // 16]
    c.v_pages[page[::3], :, dense[::3] % 16, 1::7] = value
    out, lse = c.cache.attend(length, c.q, visible=vis)
    low = vis[0] <= first
    assert bool(low.any())
    assert torch.equal(out[0][low], clean[0][0][low]) and torch.equal(lse, clean[1])
    hit = vis[0] > first
    assert bool((~torch.isfinite(out[0][hit][:, :, 1::7])).all())
    others = torch.ones(d, dtype=torch.bool, device="cuda")
    others[1::7] = False
    plain64_tol = 2.0 ** -6 if dtype == "bf16" else 1e-4     # (another way of summing the same terms, each of at most unit size)
    assert bool(((out[0][..., others].double() - clean[0][0][..., others].double()).abs() <= plain64_tol * 4).all())
    if value == math.inf:
        assert bool((out[0][hit][:, :, 1::7] == math.inf).all())
    c.k_pages[page, :, dense % 16] = value
    out, lse = c.cache.attend(length, c.q, visible=vis)
    assert torch.equal(out[0][low], clean[0][0][low]) and torch.equal(lse[0][low], clean[1][0][low])
    # what lies in pages and places that no entry of the row is, and behind the length
    c = Case(lazyev_lib, dtype, d, 1, n, Hq, H, 16, length, seed=3)
    used = torch.zeros(c.k_pages.shape[:1] + (16,), dtype=torch.bool, device="cuda")
    at = torch.arange(length, device="cuda")
    used[c.table[0].long()[at // 16], at % 16] = True
    for pages in (c.k_pages, c.v_pages):
        pages.transpose(1, 2)[~used] = value
    out, lse = c.cache.attend(length, c.q, visible=vis)
    assert torch.equal(out, clean[0]) and torch.equal(lse, clean[1])
    less = c.cache.attend(length - 3, c.q)
    assert bool(torch.isfinite(less[0]).all())


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("n,length,Hq,page", [(1, 200, 7, 16), (2, 2000, 4, 16), (70, 200, 4, 24), (200, 500, 2, 1), (900, 300, 4, 8), (4500, 130, 2, 16)])
def test_pages_that_are_none(lazyev_lib, dtype, d, n, length, Hq, page):
    """Numbers outside the pages are not followed: their entries are not there for anybody."""
    c = Case(lazyev_lib, dtype, d, 2, n, Hq, 1, page, length, seed=4)
    good = c.table.clone()
    bad = torch.rand(c.table.shape, generator=c.gen, device="cuda") < 0.3
    bad[0, 0] = True
    bad[1] = False
    bad[1, -1] = True
    strange = torch.tensor([-1, c.k_pages.shape[0], 2 ** 31 - 1, -(2 ** 31)], device="cuda").int()
    c.table.copy_(torch.where(bad, strange[torch.arange(bad.shape[1], device="cuda") % 4].expand(bad.shape), good))
    there = (~bad).repeat_interleave(page, 1)[:, :length]
    vis = torch.randint(0, length + 1, (2, n), generator=c.gen, device="cuda").int()
    got = [c.cache.attend(length, c.q), c.cache.attend(length, c.q, visible=vis)]
    c.table.fill_(-7)                              # no page at all
    out, lse = c.cache.attend(length, c.q)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())
    c.table.copy_(good)
    c.check(got[0], there=there)
    c.check(got[1], visible=vis, there=there)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("n,length,Hq", [(1, 3000, 7), (40, 600, 4), (300, 100, 2), (600, 700, 7), (9000, 200, 1)])
def test_large_logits(lazyev_lib, dtype, d, n, length, Hq):
    """Logits that rise and fall by thousands along the entries, so that weights leave the range of 32 bits on the way; all alike; all
    far below zero."""
    c = Case(lazyev_lib, dtype, d, 1, n, Hq, 1, 16, length, seed=5)
    slope = torch.linspace(-1, 1, length, device="cuda")
    for ramp in (slope, -slope, (slope * 9).sin(), slope.abs() - 4):
        c.k_pages.zero_()
        rows = c.randn(length, d) * 0.1
        rows[:, 0] = 40 * ramp
        at = torch.arange(length, device="cuda")
        c.k_pages[c.table[0].long()[at // 16], 0, at % 16] = rows.to(c.dt)
        c.q[..., 0] = 300.0
        c.check(c.cache.attend(length, c.q))
    c.k_pages.zero_()
    c.check(c.cache.attend(length, c.q))


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("n,length", [(1, 1000), (3, 5000), (90, 300)])
def test_places_of_any_element_and_guards(lazyev_lib, dtype, d, n, length):
    """q, out and the joined part start at any element: the same bits, and nothing beside them is written."""
    c = Case(lazyev_lib, dtype, d, 1, n, 6, 2, 16, length, seed=6)
    joined = (c.randn(1, n, 6, d).to(c.dt), 6 + c.randn(1, n, 6))

    def at(x, shift):
        y = torch.full((x.numel() + shift + 64,), 9.0, dtype=x.dtype, device="cuda")
        z = y[shift:shift + x.numel()].view(x.shape)
        z.copy_(x)
        return y, z
    want = c.cache.attend(length, c.q, joined=joined)
    for shifts in ((1, 2, 3), (3, 1, 2), (8, 4, 1)):
        (_, q), (bo, out), (_, jo), (bl, lse) = at(c.q, shifts[0]), at(c.q * 0, shifts[1]), at(joined[0], shifts[2]), at(joined[1] * 0, shifts[1])
        c.cache.attend(length, q, joined=(jo, joined[1]), out=out, lse=lse)
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
        for b, x in ((bo, out), (bl, lse)):
            assert bool((b[:shifts[1]] == 9).all()) and bool((b[shifts[1] + x.numel():] == 9).all())


@pytest.mark.parametrize("dtype,d", TYPES)
def test_more_pages_than_a_block_keeps_the_numbers_of(lazyev_lib, dtype, d):
    """Pages of one entry, more than a thousand of them for every block, some of them none."""
    n, length = 9000, 2500
    c = Case(lazyev_lib, dtype, d, 1, n, 4, 1, 1, length, seed=9)
    vis = torch.randint(0, length + 1, (1, n), generator=c.gen, device="cuda").int()
    vis[:, n // 2:] = length
    c.check(c.cache.attend(length, c.q, visible=vis), visible=vis)
    good = c.table.clone()
    there = torch.ones((1, length), dtype=torch.bool, device="cuda")
    there[0, 1100:2400:7] = False
    c.table[~there] = -1
    got = c.cache.attend(length, c.q)
    c.table.copy_(good)
    c.check(got, there=there)


def test_rows_of_the_table_may_share_pages(lazyev_lib):
    c = Case(lazyev_lib, "bf16", 128, 2, 9, 8, 2, 16, 100, seed=7)
    c.table[1, :4] = c.table[0, :4]
    c.check(c.cache.attend(100, c.q))


@pytest.mark.parametrize("n,length,Hq,H", [(4, 5000, 28, 4), (400, 600, 8, 2)])
def test_repeats_streams_and_replays(lazyev_lib, n, length, Hq, H):
    """The same bits every time: repeated, on two streams at once, and replayed from a graph with inputs written anew."""
    c = Case(lazyev_lib, "bf16", 128, 1, n, Hq, H, 64, length, seed=8)
    qs = [c.q] + [c.randn(*c.q.shape).bfloat16() for _ in range(5)]
    want = [c.cache.attend(length, q) for q in qs]
    for q, w in zip(qs, want):
        assert all(torch.equal(x, y) for x, y in zip(c.cache.attend(length, q), w))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = []
    for i, q in enumerate(qs):
        with torch.cuda.stream(streams[i % 2]):
            got.append(c.cache.attend(length, q))
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for g, w in zip(got, want) for x, y in zip(g, w))
    rope = lazyev_lib.NormRope(128, inv_freq=torch.rand(64, device="cuda"))
    turned = [rope(q, None, start=9)[0] for q in qs]
    both = [c.cache.attend(length, t) for t in turned]
    buf = qs[0].clone()
    out, lse, mid = torch.empty_like(buf), torch.empty(buf.shape[:-1], device="cuda"), torch.empty_like(buf)
    work = torch.empty(max(1, c.cache.workspace_bytes(length, n)), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=streams[0]):
        rope(buf, None, start=9, q_out=mid)
        c.cache.attend(length, mid, out=out, lse=lse, workspace=work)
    for r in range(12):
        buf.copy_(qs[r % 6])
        if r % 3 == 1:
            work.fill_(255)                        # (no initial contents are needed)
            torch.zeros(1 << 20, device="cuda").add_(1)
            torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(mid, turned[r % 6]) and torch.equal(out, both[r % 6][0]) and torch.equal(lse, both[r % 6][1]), r


def test_a_cache_beyond_32_bits_of_elements(lazyev_lib):
    """Pages whose places lie beyond 2^32 elements and bytes."""
    d, H, page = 128, 8, 1024
    n_pages = 4200                                 # 4.4e9 elements, 8.8 GB each
    pools = [torch.zeros((n_pages, H, page, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    table = torch.tensor([[n_pages - 1, 0, n_pages - 2]], device="cuda").int()
    gen = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn((2500, H, d), generator=gen, device="cuda").bfloat16() for _ in range(2))
    cache = lazyev_lib.PagedCache(*pools, table, n_q_heads=8)
    cache.append(0, k, v)
    assert torch.equal(pools[0][n_pages - 1], k[:1024].transpose(0, 1)) and torch.equal(pools[1][n_pages - 2, :, :452], v[2048:].transpose(0, 1))
    q = torch.randn((3, 8, d), generator=gen, device="cuda").bfloat16()
    out, lse = cache.attend(2500, q)
    want = plain64.attend(q, k, v, torch.full((3,), 2500, device="cuda"), d ** -0.5)
    plain64.check_out(out, want[0], want[2])
    plain64.check_lse(lse, want[1], want[3])


def test_numbers_beyond_32_bits_are_refused(lazyev_lib):
    """A table may have room for more entries than have numbers: such a call is refused, not taken for one of fewer."""
    b = lazyev_lib
    page = 1 << 16
    k = torch.zeros((1, 1, page, 64), dtype=torch.bfloat16, device="cuda")
    table = torch.zeros((1, (1 << 16) + 1), dtype=torch.int32, device="cuda")
    cache = b.PagedCache(k, k, table)
    new = torch.ones((1, 1, 64), dtype=torch.bfloat16, device="cuda")
    for entries in ((1 << 32) + 1, (1 << 32), (1 << 31), (1 << 30) + 1, -1):
        with pytest.raises(ValueError):
            cache.attend(entries, new)
        with pytest.raises(ValueError):
            cache.workspace_bytes(entries, 1)
        with pytest.raises(ValueError):
            cache.append(entries, new, new)
    for position in (1 << 31, 1 << 32, -(1 << 31) - 1):
        with pytest.raises(ValueError):
            cache.append(0, new, new, position0=position)
    torch.cuda.synchronize()
    assert int(torch.count_nonzero(k)) == 0


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("n,length,Hq,page", [(1, 300, 7, 16), (50, 1500, 7, 1), (700, 1500, 7, 1), (9000, 1300, 4, 1)])
@pytest.mark.parametrize("value", [math.inf, math.nan])
def test_values_behind_masks_in_long_rows(lazyev_lib, dtype, d, n, length, Hq, page, value):
    """Infinities and NaN at the end of what some tokens see, and in the page whose rows stand in for those of pages that are none: the other
    tokens' bits are the same as without, over more pages than a block keeps the numbers of."""
    c = Case(lazyev_lib, dtype, d, 1, n, Hq, 1, page, length, seed=11)
    entries = torch.arange(length, device="cuda") // page
    c.table[0, ::5] = -1
    c.table[c.table == 0] = c.k_pages.shape[0]
    vis = torch.randint(1, length + 1, (1, n), generator=c.gen, device="cuda").int()
    vis[0, -1] = length - 40
    want = c.cache.attend(length, c.q, visible=vis)
    c.k_pages[0], c.v_pages[0] = value, value
    got = c.cache.attend(length, c.q, visible=vis)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    page_of_last = c.table[0].long()[entries[length - 40:]]
    place = torch.arange(length - 40, length, device="cuda") % page
    on = (page_of_last >= 0) & (page_of_last < c.k_pages.shape[0])
    c.v_pages[page_of_last[on], 0, place[on], ::3] = value
    got = c.cache.attend(length, c.q, visible=vis)
    low = vis[0] <= length - 40
    assert bool(low.any()) and torch.equal(got[1], want[1])
    assert torch.equal(got[0][0][low], want[0][0][low])
    first_on = length - 40 + int(on.nonzero()[0])
    hit = vis[0] > first_on
    assert bool((~torch.isfinite(got[0][0][hit][:, :, ::3])).all())
    assert bool(torch.isfinite(got[0][0][..., 1::3]).all())
