"""Weights relative to a log-sum-exp over chosen blocks alone: what the header says of them."""
import pytest
import torch

import long64
from plain64 import U
from test_gpu_blocks import TYPES, Cache, _some_blocks

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("n", [1, 40])
def test_weights_beside_chosen_blocks(lazyev_lib, dtype, d, n):
    """Entries that a token read have weights that add up to one; those that it did not read have what their logits make beside them, more than one for a
    logit above the log-sum-exp.  Beside all entries no weight is above one."""
    S, H, G, length, block = 1, 2, 7, 900, 32
    c = Cache(lazyev_lib, dtype, d, S, H, 24, length, seed=60)
    q = (1.3 * c.randn(S, n, H * G, d)).to(c.dt)
    blocks = _some_blocks(c, 1, length, block, 6).expand(S, n, H, 6).contiguous()     # (the same of all tokens)
    blocks[:, :, 1] = blocks[:, :, 0]
    lse = c.cache.attend_blocks(length, q, blocks, block)[1]
    got = c.cache.weigh(length, q, lse)
    want, bound = long64.weigh(q[0], lse[0], c.rows(c.k_pages)[0, :length], torch.full((n,), length, device="cuda"), d ** -0.5)
    assert bool(((got[0].double() - want).abs() <= bound + U * want.abs() + 1e-30).all())
    at = torch.arange(length, device="cuda")
    read = (at[:, None] // block == blocks[0, 0, 0]).any(1)
    # each row's sum is off by what its log-sum-exp is, which `bound` counts for that of the weights, and twice at most
    assert bool(((got[0][:, read].double().sum(1) - n * G).abs() <= 2 * bound[:, read].sum(1) + n * G * (6 * block + 16) * U).all())
    assert bool((got[0][:, ~read].double().sum(1) > n * G).all())                     # (most of the entries)
    all_lse = c.cache.attend(length, q)[1]
    assert bool((c.cache.weigh(length, q, all_lse) <= n * G * (1 + 2.0 ** -10)).all())
    # a logit far beyond those of the blocks read
    far = int(at[~read][5])
    c.k_pages[c.table[0, far // 24].long(), :, far % 24] = 30 * q[0, 0].view(H, G, d)[:, 0]
    assert bool((c.cache.weigh(length, q, lse)[0, :, far] > 1e30).all())
    assert torch.equal(c.cache.attend_blocks(length, q, blocks, block)[1], lse)
