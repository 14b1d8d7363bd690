"""Attention over chosen blocks whose lists are joined for a tile of tokens: numbers that lists have more than once, against the definition in 64 bits."""
import math

import pytest
import torch

from test_gpu_blocks import TYPES, Cache, _attend, _some_blocks

pytestmark = pytest.mark.gpu


# tables, tokens, query and KV heads, page, length, block, numbers of a list: lists shorter and longer than 64 numbers, tiles of 32 tokens and of fewer
@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("S,n,Hq,H,page,length,block,m", [(1, 33, 8, 8, 16, 300, 16, 40), (2, 20, 21, 7, 24, 333, 32, 130), (1, 300, 1, 1, 64, 64, 64, 3),
                                                          (1, 65, 64, 4, 16, 2000, 16, 200)])
def test_numbers_more_than_once(lazyev_lib, dtype, d, S, n, Hq, H, page, length, block, m):
    c = Cache(lazyev_lib, dtype, d, S, H, page, length, seed=30)
    q = c.randn(S, n, Hq, d).to(c.dt)
    n_blocks = -(-length // block)
    any_order = c.randint(-1, n_blocks + 1, S, n, H, m).int()          # -1 and n_blocks: none
    once = _some_blocks(c, n, length, block, m)
    few = once.clone()                                                 # one token of a tile, one number of it
    few[:, n // 2, :, -1] = few[:, n // 2, :, 0]
    alike = any_order.clone()
    alike[:, ::3] = n_blocks // 2                                      # the same number all along
    for blocks in (any_order, few, alike):
        got = _attend(c, length, q, blocks, block)
        again = c.cache.attend_blocks(length, q, blocks, block)
        assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])
    vis = c.randint(0, length + 1, S, n).int()
    vis[:, ::5] = length
    _attend(c, length, q, any_order, block, visible=vis)


@pytest.mark.parametrize("dtype,d", TYPES)
def test_a_number_more_than_once_counts_by_its_times(lazyev_lib, dtype, d):
    """A block listed k times weighs as much as k blocks of its entries: log k more in the log-sum-exp of a list of one block, the output the same."""
    c = Cache(lazyev_lib, dtype, d, 1, 9, 16, 160, seed=31)
    q = c.randn(1, 40, 18, d).to(c.dt)
    one = c.randint(0, 10, 1, 40, 9, 1).int()
    out, lse = c.cache.attend_blocks(160, q, one, 16)
    for times in (2, 63, 64, 65, 700):
        o, l = c.cache.attend_blocks(160, q, one.expand(1, 40, 9, times).contiguous(), 16)
        # a sum of 16 k weights in 32 bits (k additions to one number at most, 16 more) and a logarithm of both sides; the same weights of both outputs
        step = (times + 40) * 2.0 ** -24
        assert bool(((l - lse).double() - torch.tensor(float(times)).double().log().item()).abs().max() <= 2 * step + 4 * 2.0 ** -24 * l.abs().max())
        rounding = 2.0 ** -24 if dtype == "fp32" else 2.0 ** -8
        most = c.rows(c.v_pages).abs().max().double()
        assert bool((o.double() - out.double()).abs().max() <= (2 * rounding + 4 * step) * most)


@pytest.mark.parametrize("dtype,d", TYPES)
def test_lists_of_other_tokens_of_a_tile(lazyev_lib, dtype, d):
    """What the other tokens of a tile list leaves a token's result what it is, in other roundings: their blocks put its own into other stages and splits."""
    n, H, length = 60, 5, 2000
    c = Cache(lazyev_lib, dtype, d, 1, H, 32, length, seed=32)
    q = c.randn(1, n, 7 * H, d).to(c.dt)
    blocks = _some_blocks(c, n, length, 32, 12)
    vis = c.randint(1500, length + 1, 1, n).int()
    vis[:, ::4] = length
    theirs = torch.arange(n, device="cuda") % 3 != 1
    n_blocks = -(-length // 32)
    lists = {"others": _some_blocks(c, n, length, 32, 12), "none": torch.full_like(blocks, -1), "another order": blocks.flip(-1),
             "no blocks": blocks + 10 ** 6, "one of them": blocks[..., :1].expand_as(blocks), "several times": c.randint(0, n_blocks, 1, n, H, 12).int(),
             "the first ones": torch.arange(12, device="cuda").int().expand_as(blocks)}
    mine, my_lse = c.cache.attend_blocks(length, q, blocks, 32, visible=vis)
    # error of a weight, as in plain64.attend: of the logits, which are no larger than `size`, of the exponentials and of a sum of 12 x 32 entries
    size = (q.double().norm(dim=-1).max() * c.rows(c.k_pages).double().norm(dim=-1).max() * d ** -0.5).item()
    e = (2 * (d + 3) * size + 6 * size + 12 * 32 + 16) * 2.0 ** -24
    most = c.rows(c.v_pages).abs().max().double().item()
    for what, other in lists.items():
        mixed = blocks.clone()
        mixed[:, theirs] = other[:, theirs]
        out, lse = _attend(c, length, q, mixed, 32, visible=vis)       # (every token against 64 bits)
        # two results, each off by its weights' error and (bf16) half a step of the weights and of itself
        half = 2.0 ** -24 if dtype == "fp32" else 2 * 2.0 ** -8
        assert (out - mine)[:, ~theirs].abs().double().max() <= 2 * (e + half) * most, what
        assert (lse - my_lse)[:, ~theirs].abs().max() <= 2 * (e + 4 * 2.0 ** -24 * (size + 6)), what


# tables of as many blocks as the joined lists are for (8192), one fewer and one more, where every token is on its own
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("fp32", 64)])
@pytest.mark.parametrize("n_blocks", [8191, 8192, 8193])
def test_very_many_blocks(lazyev_lib, dtype, d, n_blocks):
    n, H, length = 33, 8, 16 * n_blocks - 5
    c = Cache(lazyev_lib, dtype, d, 1, H, 64, length, seed=33)
    q = c.randn(1, n, 2 * H, d).to(c.dt)
    blocks = _some_blocks(c, n, length, 16, 12)
    blocks[:, ::2, :, -1] = n_blocks - 1           # seen in part
    blocks[:, 1::4, :, 0] = 0
    blocks[:, 2, :, 3:6] = torch.tensor([n_blocks - 1, n_blocks, n_blocks + 1], device="cuda").int()     # (twice, and no blocks)
    vis = c.randint(length - 40, length + 1, 1, n).int()
    vis[:, ::4] = length
    _attend(c, length, q, blocks, 16)
    _attend(c, length, q, blocks, 16, visible=vis)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_infinities_and_nan_in_splits_of_a_tile(lazyev_lib, dtype, d, value):
    """Tiles of 18 tokens (9 of fp32 rows of 128) whose lists of up to 64 blocks go in several splits: a value that some tokens see is theirs alone."""
    n, H, length, block = 130, 2, 20000, 64
    c = Cache(lazyev_lib, dtype, d, 1, H, 24, length, seed=34)
    q = c.randn(1, n, 7 * H, d).to(c.dt)
    n_blocks = -(-length // block)
    blocks = (1 + _some_blocks(c, n, length - 5 * block, block, 64)).clamp(max=n_blocks - 4)
    # (the first block nobody's, the last three of tokens 0 mod 3 and 1 mod 3; a block that has been listed twice counts twice for both calls)
    one, other = n_blocks - 3, n_blocks - 2
    blocks[:, ::3, :, 5] = one
    blocks[:, 1::3, :, 9] = other
    vis = torch.full((1, n), length, device="cuda").int()
    vis[:, ::2] = other * block + 7                # of the second one they see seven entries
    parts = lazyev_lib.lib.lazyev_blocks_attend_workspace(c.cache.pages, length, block, 64, n, 7 * H)
    assert parts > n * H * 64 * 8 + 8 * H * 64 * d * 4                  # (pairs of every token, and more than one split's parts)
    clean = c.cache.attend_blocks(length, q, blocks, block, visible=vis)
    assert bool(torch.isfinite(clean[0]).all())
    at = torch.arange(length, device="cuda")
    nobody = at[(at < block) | (at >= (other + 1) * block)]
    c.k_pages[c.table[0, nobody // 24].long(), :, nobody % 24] = value
    c.v_pages[c.table[0, nobody // 24].long(), :, nobody % 24] = value
    hidden = other * block + 7                     # every second token of those that list its block does not see it
    c.v_pages[c.table[0, (one * block + 3) // 24].long(), :, (one * block + 3) % 24, 5] = value
    c.v_pages[c.table[0, hidden // 24].long(), :, hidden % 24, d - 2] = value
    got = c.cache.attend_blocks(length, q, blocks, block, visible=vis)
    token = torch.arange(n, device="cuda")
    hit = torch.zeros((n, d), dtype=torch.bool, device="cuda")
    hit[token % 3 == 0, 5] = True
    hit[(token % 3 == 1) & (token % 2 == 1), d - 2] = True
    hit = hit[:, None].expand(n, 7 * H, d)
    assert torch.equal(got[1], clean[1])
    assert torch.equal(got[0][0][~hit], clean[0][0][~hit])
    odd = got[0][0][hit]
    assert bool((torch.isnan(odd) if math.isnan(value) else odd == value).all())
    again = c.cache.attend_blocks(length, q, blocks, block, visible=vis)
    assert torch.equal(again[0].nan_to_num(nan=7.0), got[0].nan_to_num(nan=7.0)) and torch.equal(again[1], got[1])
