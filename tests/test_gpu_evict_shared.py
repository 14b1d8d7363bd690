"""Evictions of table rows that share pages, in the ways that leave every row its own entries (what is shared stays in its place, or was copied before); and those with
the most moves that there can be."""
import numpy as np
import pytest
import torch

import long64
from test_gpu_blocks import TYPES, Cache

pytestmark = pytest.mark.gpu


def _check(c, before, weights, length, keep, recent, first):
    """Every row's first `keep` entries are those that its sources say, as they were."""
    sources, _, _ = c.cache.evict(length, weights, keep, recent=recent, first=first)
    after = c.rows(c.k_pages), c.rows(c.v_pages)
    for s in range(c.S):
        for h in range(c.H):
            want = long64.evict(weights[s, h].cpu().numpy(), None, length, keep, recent, first)
            assert np.array_equal(sources[s, h].cpu().numpy(), want)
            at = torch.tensor(want, device="cuda")
            for x, y in zip(after, before):
                assert torch.equal(x[s, :keep, h], y[s, at, h])
    return sources


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("page,length,keep", [(16, 400, 300), (24, 2000, 700), (64, 40000, 5000)])
def test_a_shared_prefix_that_stays(lazyev_lib, dtype, d, page, length, keep):
    """Three rows with the same pages for their first entries, which are among the `first` ones: nothing moves into a shared page."""
    S, H = 3, 2
    c = Cache(lazyev_lib, dtype, d, S, H, page, length, seed=50)
    shared = 5                                     # pages
    c.table[:, :shared] = c.table[0, :shared]
    before = c.rows(c.k_pages).clone(), c.rows(c.v_pages).clone()
    prefix = [x[c.table[0, :shared].long()].clone() for x in (c.k_pages, c.v_pages)]
    sources = _check(c, before, c.randn(S, H, length).exp(), length, keep, 8, shared * page)
    assert bool((sources[:, :, keep // 2:] >= keep).any())              # (entries moved)
    for x, y in zip((c.k_pages, c.v_pages), prefix):
        assert torch.equal(x[c.table[0, :shared].long()], y)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_shared_prefix_copied_before(lazyev_lib, dtype):
    """Rows with copies of a prefix in pages of their own, of which any entry may go."""
    S, H, page, length, keep = 3, 2, 16, 500, 200
    c = Cache(lazyev_lib, dtype, 128, S, H, page, length, seed=51)
    for s in (1, 2):
        for x in (c.k_pages, c.v_pages):
            x[c.table[s, :6].long()] = x[c.table[0, :6].long()]
    before = c.rows(c.k_pages).clone(), c.rows(c.v_pages).clone()
    _check(c, before, c.randn(S, H, length).exp(), length, keep, 16, 4)


@pytest.mark.parametrize("length,keep", [(65536, 32768), (65535, 32768), (65536, 65535), (65536, 1)])
def test_as_many_moves_as_there_can_be(lazyev_lib, length, keep):
    """All that stay are the last entries, so that every place (or every entry that goes) is one to move to: the largest numbers that the places' sums hold."""
    c = Cache(lazyev_lib, "bf16", 64, 1, 2, 256, length, seed=52)
    before = c.rows(c.k_pages).clone(), c.rows(c.v_pages).clone()
    weights = torch.arange(length, device="cuda").float().expand(1, 2, length).contiguous()
    _check(c, before, weights, length, keep, 0, 0)
