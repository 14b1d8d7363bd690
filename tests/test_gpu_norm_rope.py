"""lazyev_norm_rope and lazyev_pages_append against 64 bits: head and token counts, layouts, partial rotation, strides, places that
no multiple of 16 bytes, far positions, writing in place and into the pages of a cache."""
import pytest
import torch

import plain64

pytestmark = pytest.mark.gpu

TYPES = [("bf16", 128), ("bf16", 64), ("fp32", 128), ("fp32", 64)]
EPS = 1e-6


def _dt(name):
    return torch.float32 if name == "fp32" else torch.bfloat16


def _freq(dims):
    return (10000.0 ** (-torch.arange(0, dims, 2, dtype=torch.float64) / dims)).float().cuda()


def _rope(b, dt, d, dims, layout, norm, gen):
    w = [(1.0 + 0.2 * torch.randn(d, generator=gen, device="cuda")).to(dt) if norm else None for _ in range(2)]
    return b.NormRope(d, dt, q_weight=w[0], k_weight=w[1], eps=EPS, inv_freq=_freq(dims) if dims else None,
                      layout=b.ROPE_HALVES if layout == "halves" else b.ROPE_PAIRS)


def _check(got, x, positions, weight, rope, layout):
    want, bound = plain64.turn(x, positions, weight, EPS, rope.inv_freq, layout)
    plain64.check_out(got, want, bound)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("layout,dims,norm", [("halves", 0, True), ("halves", 1, True), ("pairs", 1, True), ("halves", 1, False),
                                              ("halves", 2, True), ("pairs", 2, False), ("halves", 48, True), ("pairs", 16, True)])
@pytest.mark.parametrize("S,n,Hq,H", [(1, 1, 1, 1), (1, 32, 28, 4), (3, 7, 5, 5), (2, 2250, 3, 1), (2, 900, 20, 3)])
def test_heads_against_64_bits(lazyev_lib, dtype, d, layout, dims, norm, S, n, Hq, H):
    """dims: 0 no rotation, 1 the whole head, 2 half of it.  Of 4500 tokens each lane group has one; 1800 of bf16 rows go four to a block."""
    dt, gen = _dt(dtype), torch.Generator(device="cuda").manual_seed(n + d)
    dims = {0: 0, 1: d, 2: d // 2}.get(dims, dims)
    rope = _rope(lazyev_lib, dt, d, dims, layout, norm, gen)
    q, k = (torch.randn((S, n, h, d), generator=gen, device="cuda").to(dt) for h in (Hq, H))
    pos = torch.randint(-50, 1 << 20, (S, n), generator=gen, device="cuda").int()
    qo, ko = rope(q, k, positions=pos, start=3)
    _check(qo, q, pos + 3, rope.q_weight, rope, layout)
    _check(ko, k, pos + 3, rope.k_weight, rope, layout)
    at = (torch.arange(n, device="cuda") + 11).expand(S, n)
    none, ko = rope(None, k, start=11)             # keys alone, positions in a row
    assert none is None
    _check(ko, k, at, rope.k_weight, rope, layout)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("layout,dims", [("halves", 64), ("pairs", 32)])
@pytest.mark.parametrize("S,n,Hq,H", [(1, 4099, 9, 3), (5, 820, 10, 1), (1, 1100, 40, 8), (1, 700, 3, 30), (3, 171, 70, 1)])
def test_many_tokens_of_many_heads(lazyev_lib, dtype, d, layout, dims, S, n, Hq, H):
    """Four tokens to a block, also where the last block has fewer; one to a block, with results beyond a cache's size and below."""
    dt, gen = _dt(dtype), torch.Generator(device="cuda").manual_seed(n + d)
    rope = _rope(lazyev_lib, dt, d, dims, layout, True, gen)
    qkv = torch.randn((S, n, Hq + 2 * H, d), generator=gen, device="cuda").to(dt)
    q, k = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + H]
    pos = torch.randint(0, 1 << 16, (S, n), generator=gen, device="cuda").int()
    qo, ko = rope(q, k, positions=pos)
    _check(qo, q, pos, rope.q_weight, rope, layout)
    _check(ko, k, pos, rope.k_weight, rope, layout)


@pytest.mark.parametrize("dtype,d", TYPES)
def test_far_positions(lazyev_lib, dtype, d):
    dt, gen = _dt(dtype), torch.Generator(device="cuda").manual_seed(5)
    rope = _rope(lazyev_lib, dt, d, d, "halves", False, gen)
    q = torch.randn((4, 6, d), generator=gen, device="cuda").to(dt)
    pos = torch.tensor([2 ** 31 - 1, 2 ** 24 + 1, -(2 ** 31), 0], device="cuda").int()
    qo, _ = rope(q, None, positions=pos)
    # the angle in binary64: three roundings of up to 2^31 radians on each side
    want, bound = plain64.turn(q, pos, None, EPS, rope.inv_freq, "halves")
    plain64.check_out(qo, want, bound + 2.0 ** 31 * 8 * 2.0 ** -53 * q.double().abs().amax() * 2)
    again, _ = rope(q, None, positions=(pos.long() - 7).clamp(min=-(2 ** 31)).int(), start=7)
    assert torch.equal(again[[0, 1, 3]], qo[[0, 1, 3]])


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("shift", [0, 1, 3])
def test_strides_places_and_writing_in_place(lazyev_lib, dtype, d, shift):
    """Views into a joint projection that start at any element, a broadcast source, results into a transposed cache with other rows
    left as they are; in place."""
    dt, gen = _dt(dtype), torch.Generator(device="cuda").manual_seed(shift)
    S, n, Hq, H = 2, 19, 6, 2
    rope = _rope(lazyev_lib, dt, d, d, "halves", True, gen)
    width = (Hq + 2 * H) * d + shift
    flat = torch.randn(S * n * width + shift, generator=gen, device="cuda").to(dt)
    joint = flat[shift:].view(S, n, width)
    q, k = joint[:, :, :Hq * d].unflatten(2, (Hq, d)), joint[:, :, Hq * d:(Hq + H) * d].unflatten(2, (H, d))
    pos = torch.arange(n, device="cuda").expand(S, n)
    cache = torch.full((S, H, n + 5, d), 7.0, device="cuda", dtype=dt)
    to = cache[:, :, 2:2 + n].transpose(1, 2)
    before = flat.clone()
    qo, ko = rope(q, k, k_out=to)
    assert ko is to and torch.equal(flat, before)
    _check(qo, q, pos, rope.q_weight, rope, "halves")
    _check(to, k, pos, rope.k_weight, rope, "halves")
    assert bool((cache[:, :, :2] == 7).all()) and bool((cache[:, :, 2 + n:] == 7).all())
    src, (old_q, old_k) = flat.clone(), (q.clone(), k.clone())
    rope(q, k, q_out=q, k_out=k)                   # in place
    assert torch.equal(q, qo) and torch.equal(k, to)
    q.copy_(old_q), k.copy_(old_k)
    assert torch.equal(flat, src)                  # nothing else was written
    one = torch.randn((1, 1, Hq, d), generator=gen, device="cuda").to(dt)
    qo, _ = rope(one.expand(S, n, Hq, d), None)
    _check(qo, one.expand(S, n, Hq, d), pos, rope.q_weight, rope, "halves")


@pytest.mark.parametrize("dtype,d", TYPES)
def test_special_values_stay_in_their_pair(lazyev_lib, dtype, d):
    """Without a norm an infinity or NaN reaches its pair's two elements and no other; elements that are not turned go
    through bit by bit; a zero head with a norm stays zero."""
    dt = _dt(dtype)
    gen = torch.Generator(device="cuda").manual_seed(1)
    rope = _rope(lazyev_lib, dt, d, 32, "halves", False, gen)
    x = torch.randn((1, 2, d), generator=gen, device="cuda").to(dt)
    x[0, 0, 3], x[0, 0, 40], x[0, 1, 20] = float("inf"), float("nan"), float("-inf")
    y, _ = rope(x, None, start=5)
    bad = ~torch.isfinite(y[0])
    assert bad[0].nonzero().flatten().tolist() == [3, 19, 40] and bad[1].nonzero().flatten().tolist() == [4, 20]
    assert torch.equal(y[0, :, 32:].view(torch.int32), x[0, :, 32:].view(torch.int32))
    normed = _rope(lazyev_lib, dt, d, d, "pairs", True, gen)
    assert bool((normed(torch.zeros((2, 3, d), dtype=dt, device="cuda"), None)[0] == 0).all())


def test_empty_batches(lazyev_lib):
    rope = lazyev_lib.NormRope(64, torch.float32, inv_freq=_freq(64))
    for shape in ((0, 4, 64), (0, 5, 4, 64), (2, 0, 4, 64)):
        q, _ = rope(torch.empty(shape, device="cuda"), None)
        assert q.shape == shape


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("page,start,n,S", [(16, 0, 1, 1), (16, 9, 40, 2), (24, 77, 601, 2), (1, 3, 5, 1), (4096, 100, 2300, 4), (64, 63, 1, 3)])
def test_append_to_pages(lazyev_lib, dtype, d, page, start, n, S):
    """Keys turned and values bit by bit in their entries, every other entry as it was."""
    dt, gen, H = _dt(dtype), torch.Generator(device="cuda").manual_seed(page + n), 3
    m = (start + n + page - 1) // page + 1
    table = torch.randperm(S * m + 2, generator=gen, device="cuda")[:S * m].view(S, m).int()
    k_pages, v_pages = (torch.randn((S * m + 2, H, page, d), generator=gen, device="cuda").to(dt) for _ in range(2))
    rope = _rope(lazyev_lib, dt, d, d, "halves", True, gen)
    rows = torch.randn((S, n, 2 * H + 1, d), generator=gen, device="cuda").to(dt)
    k, v = rows[:, :, :H], rows[:, :, H:2 * H]
    want_v, old_k = v_pages.clone(), k_pages.clone()
    at = start + torch.arange(n, device="cuda")
    for s in range(S):
        pages = table[s].long()[at // page]
        want_v[pages, :, at % page] = v[s]
    lazyev_lib.PagedCache(k_pages, v_pages, table).append(start, k, v, rope=rope, position0=start + 1000)
    assert torch.equal(v_pages, want_v)
    for s in range(S):
        pages = table[s].long()[at // page]
        _check(k_pages[pages, :, at % page], k[s], at + 1000, rope.k_weight, rope, "halves")
        k_pages[pages, :, at % page] = old_k[pages, :, at % page]
    assert torch.equal(k_pages, old_k)


def test_append_leaves_pages_that_are_none_alone(lazyev_lib):
    gen = torch.Generator(device="cuda").manual_seed(3)
    n, page, H, d = 60, 16, 2, 64
    table = torch.tensor([[2, -1, 5, 0]], device="cuda").int()           # of five pages 0 .. 4: two are none
    k_pages, v_pages = (torch.randn((5, H, page, d), generator=gen, device="cuda") for _ in range(2))
    want_k, want_v = k_pages.clone(), v_pages.clone()
    k, v = (torch.randn((n, H, d), generator=gen, device="cuda") for _ in range(2))
    lazyev_lib.PagedCache(k_pages, v_pages, table).append(0, k, v)       # as they are
    for rows, want, got in ((k, want_k, k_pages), (v, want_v, v_pages)):
        want[2] = rows[:16].transpose(0, 1)
        want[0, :, :12] = rows[48:].transpose(0, 1)
        assert torch.equal(got, want)


def test_append_to_a_contexts_own_cache(lazyev_lib):
    """A layer's cache as pages, one per sequence: prompts that arrive as [sequence, position, head] rows."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    S, H, P, d = 3, 4, 50, 128
    eng = lazyev_lib.LazyEviction(2, S, 28, H, d, 100, 10, P, 0.01)
    k, v = (torch.randn((S, P, H, d), generator=gen, device="cuda").bfloat16() for _ in range(2))
    table = torch.arange(S, device="cuda").int()[:, None]
    lazyev_lib.PagedCache(eng.k_cache[1], eng.v_cache[1], table).append(0, k, v)
    assert torch.equal(eng.k_cache[1, :, :, :P], k.transpose(1, 2)) and torch.equal(eng.v_cache[1, :, :, :P], v.transpose(1, 2))
    assert not eng.k_cache[0].any() and not eng.k_cache[1, :, :, P:].any()
