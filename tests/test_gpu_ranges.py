"""The largest and smallest numbers that include/lazyev.h answers for: values of attention whose weighted sums stay in the range of fp32 on the way, heads whose
squares do."""
import pytest
import torch

import plain64
from test_gpu_pages import TYPES, Case, _dt

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("n,length,Hq", [(1, 1003, 7), (40, 3000, 4), (300, 700, 2), (900, 700, 7), (9000, 260, 1)])
def test_values_of_the_largest_size(lazyev_lib, dtype, d, n, length, Hq):
    """Values around 2^89 behind logits that rise until weights are far above the first reference (by up to 2^12 before it is raised)."""
    c = Case(lazyev_lib, dtype, d, 1, n, Hq, 1, 16, length, seed=31)
    c.v_pages.copy_((torch.rand(c.v_pages.shape, generator=c.gen, device="cuda") - 0.5).to(c.dt) * 2.0 ** 90)
    rows = 0.1 * c.randn(length, d)
    rows[:, 0] = torch.linspace(0, 16.0, length, device="cuda")
    at = torch.arange(length, device="cuda")
    c.k_pages.zero_()
    c.k_pages[c.table[0].long()[at // 16], 0, at % 16] = rows.to(c.dt)
    c.q.zero_()
    c.q[..., 0] = d ** 0.5                         # (logits from 0 to 16)
    c.check(c.cache.attend(length, c.q))
    vis = torch.randint(0, length + 1, (1, n), generator=c.gen, device="cuda").int()
    c.check(c.cache.attend(length, c.q, visible=vis), visible=vis)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("size", [2.0 ** 60, 2.0 ** -60])
def test_heads_of_the_largest_and_smallest_size(lazyev_lib, dtype, d, size):
    """Without an eps to help."""
    dt, gen = _dt(dtype), torch.Generator(device="cuda").manual_seed(d)
    freq = torch.logspace(0, -4, d // 2, device="cuda")
    rope = lazyev_lib.NormRope(d, dt, q_weight=torch.ones(d, device="cuda", dtype=dt), eps=0.0, inv_freq=freq)
    x = ((0.5 + 0.5 * torch.rand((9, 3, d), generator=gen, device="cuda")).to(dt) * size if size > 1 else
         (1.0 + torch.rand((9, 3, d), generator=gen, device="cuda")).to(dt) * size)
    x = x * (2 * torch.randint(0, 2, x.shape, generator=gen, device="cuda") - 1).to(dt)
    got, _ = rope(x, None)
    want, bound = plain64.turn(x, torch.arange(9, device="cuda"), rope.q_weight, 0.0, freq, "halves")
    plain64.check_out(got, want, bound)
