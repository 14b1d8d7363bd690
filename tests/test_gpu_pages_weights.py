"""lazyev_pages_attend: what the weights keep in the product with V.  64 x bf16 rows take them as two bf16 terms, as exact beside the output's one
rounding as fp32; an infinity that a token sees still comes out as one."""
import math

import pytest
import torch

import plain64
from test_gpu_pages import TYPES, Case

pytestmark = pytest.mark.gpu

# every shape of blocks, with splits of the entries and without
SHAPES = [(1, 1, 7, 1, 16, 200), (2, 1, 28, 4, 16, 700), (1, 32, 28, 4, 64, 500), (1, 20, 32, 1, 128, 333), (1, 257, 2, 2, 64, 129),
          (1, 600, 7, 1, 16, 700), (1, 4500, 4, 1, 48, 130)]


@pytest.mark.parametrize("S,n,Hq,H,page,length", SHAPES)
@pytest.mark.parametrize("some", [False, True])
def test_weights_of_short_rows_beside_one_rounding(lazyev_lib, S, n, Hq, H, page, length, some):
    """The bound of arithmetic in 32 bits, of the same numbers as fp32 rows, and what two bf16 terms leave of a weight: 2^-8 of 2^-8."""
    c = Case(lazyev_lib, "bf16", 64, S, n, Hq, H, page, length, seed=21)
    vis = torch.full((S, n), length, device="cuda").int()
    if some:
        vis = torch.randint(0, length + 1, (S, n), generator=c.gen, device="cuda").int()
    out, lse = c.cache.attend(length, c.q, visible=vis if some else None)
    k, v = c.rows(c.k_pages).float(), c.rows(c.v_pages).float()
    for s in range(S):
        want, want_lse, bound, bound_lse = plain64.attend(c.q[s].float(), k[s], v[s], vis[s].long(), 64 ** -0.5)
        size = plain64.attend(c.q[s].float(), k[s], v[s].abs(), vis[s].long(), 64 ** -0.5)[0]
        plain64.check_out(out[s], want, bound + 2.0 ** -16 * size)
        plain64.check_lse(lse[s], want_lse, bound_lse)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("S,n,Hq,H,page,length", SHAPES)
def test_infinities_that_every_token_sees(lazyev_lib, dtype, d, S, n, Hq, H, page, length):
    """Columns of V with infinities of one sign, of both, with a NaN: those, and every other column's bits as without; no token's weight
    of any entry is zero."""
    c = Case(lazyev_lib, dtype, d, S, n, Hq, H, page, length, seed=22)
    c.q.mul_(0.25)                                 # (weights far from the end of the range)
    clean = c.cache.attend(length, c.q)
    at = torch.tensor([0, length // 3, length - 1], device="cuda")
    pages, places = c.table.long()[:, at // page], (at % page).expand(S, 3)
    for column, values in ((3, (math.inf,) * 3), (17, (-math.inf,) * 3), (40, (math.inf, -math.inf, math.inf)), (41, (1.0, math.nan, 1.0))):
        c.v_pages[pages, :, places, column] = torch.tensor(values, device="cuda").to(c.dt)[None, :, None].expand(S, 3, H)
    out, lse = c.cache.attend(length, c.q)
    assert torch.equal(lse, clean[1])
    assert bool((out[..., 3] == math.inf).all()) and bool((out[..., 17] == -math.inf).all()) and bool(out[..., 40:42].isnan().all())
    others = torch.ones(d, dtype=torch.bool, device="cuda")
    others[[3, 17, 40, 41]] = False
    assert torch.equal(out[..., others], clean[0][..., others])


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("n,length,Hq,H,page", [(1, 100, 7, 1, 16), (40, 300, 4, 2, 16), (300, 400, 2, 1, 24), (600, 700, 7, 1, 16), (9000, 130, 1, 1, 16)])
@pytest.mark.parametrize("value", [math.inf, math.nan])
def test_other_columns_keep_their_bits(lazyev_lib, dtype, d, n, length, Hq, H, page, value):
    """Infinities or NaN in some columns of entries that some tokens see: the other columns and the log-sum-exps are the same bits for every token,
    those that see the entries among them."""
    c = Case(lazyev_lib, dtype, d, 1, n, Hq, H, page, length, seed=23)
    vis = torch.randint(1, length + 1, (1, n), generator=c.gen, device="cuda").int()
    vis[0, -1], vis[0, 0] = length // 2, length
    clean = c.cache.attend(length, c.q, visible=vis)
    dense = torch.arange(length // 2, length, device="cuda")
    pages = c.table[0].long()[dense // page]
    c.v_pages[pages[::3], :, dense[::3] % page, 1::7] = value
    out, lse = c.cache.attend(length, c.q, visible=vis)
    others = torch.ones(d, dtype=torch.bool, device="cuda")
    others[1::7] = False
    assert torch.equal(lse, clean[1]) and torch.equal(out[..., others], clean[0][..., others])
    low = vis[0] <= length // 2
    assert torch.equal(out[0][low], clean[0][0][low]) and bool((~torch.isfinite(out[0][~low][..., 1::7])).all())
