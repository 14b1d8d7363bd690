"""Attention over chosen blocks whose lists are joined for a tile of tokens: numbers that lists have more than once, against the definition in 64 bits."""
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
