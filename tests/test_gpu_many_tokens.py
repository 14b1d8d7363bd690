"""Calls of more tokens than one launch has blocks for: a broadcast source, of which the entries of a few pages are kept (the others are no pages)."""
import pytest
import torch

import plain64

pytestmark = pytest.mark.gpu

PAGE = 4096


@pytest.mark.parametrize("dtype,d,H,tokens", [("bf16", 128, 8, 1 << 26),      # four tokens a block: 2^23 blocks are 2^25 tokens
                                              ("fp32", 128, 1, 1 << 27)])      # a token per group of lanes, eight a block: 2^26 tokens
def test_more_tokens_than_a_launch_has(lazyev_lib, dtype, d, H, tokens):
    dt = torch.float32 if dtype == "fp32" else torch.bfloat16
    gen = torch.Generator(device="cuda").manual_seed(H)
    n = tokens + 77
    m = -(-n // PAGE)
    # pages that are kept: the first, both sides of every launch's end, one in between, the last
    step = (1 << 23) * (4 if H == 8 else 8) // PAGE
    kept = sorted({0, step - 1, step, step + 3, 2 * step - 1, m - 1})
    table = torch.full((1, m), -1, dtype=torch.int32, device="cuda")
    table[0, kept] = torch.arange(len(kept), device="cuda").int()
    pools = [torch.full((len(kept), H, PAGE, d), 5.0, dtype=dt, device="cuda") for _ in range(2)]
    freq = torch.logspace(0, -4, 8, device="cuda")
    weight = (1.0 + 0.1 * torch.randn(d, generator=gen, device="cuda")).to(dt)
    rope = lazyev_lib.NormRope(d, dt, k_weight=weight, inv_freq=freq)
    k, v = (torch.randn((1, H, d), generator=gen, device="cuda").to(dt) for _ in range(2))
    lazyev_lib.PagedCache(*pools, table).append(0, k.expand(n, H, d), v.expand(n, H, d), rope=rope)
    for i, page in enumerate(kept):
        at = page * PAGE + torch.arange(PAGE, device="cuda")
        there = at < n
        want, bound = plain64.turn(k.expand(PAGE, H, d), at, weight, 1e-6, freq, "halves")
        # (the angle in binary64: three roundings of up to 2^27 radians on each side)
        bound = bound + 2.0 ** 27 * 8 * 2.0 ** -53 * 2 * want.abs().amax()
        got_k, got_v = (x[i].transpose(0, 1) for x in pools)
        plain64.check_out(got_k[there], want[there], bound[there])
        assert torch.equal(got_v[there], v.expand(PAGE, H, d)[there])
        assert bool((got_k[~there] == 5).all()) and bool((got_v[~there] == 5).all())
