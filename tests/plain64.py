"""The operators around a decode step in 64 bits, from their definitions, with the error that arithmetic in 32 bits and one rounding
to the rows' type can make (helper of the GPU tests, not collected)."""
import math

import torch

HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
U = 2.0 ** -24


def turn(x, positions, weight, eps, inv_freq, layout):
    """(result, bound of its error before the rounding to the rows' type) of heads x [..., H, d] at positions [...].

    The bound, in units of 2^-24 times |a| + |b| of the turned pair: the norm's sum of squares of d <= 128 terms (a chain of 8
    and five more additions: 13, halved by the root), root, quotient, two products (4): 10.5; sine and cosine two units in
    the last place and pi times the rounding of the turn: 5.2; product and sum: 2.  Taken: 20."""
    x = x.double()
    if weight is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * weight.double()
    size = x.abs()
    if inv_freq is not None:
        n = inv_freq.numel()
        angle = (positions.double()[..., None] * inv_freq.double())[..., None, :]
        c, s = torch.cos(angle), torch.sin(angle)
        ia = torch.arange(n, device=x.device) * (1 if layout == "halves" else 2)
        ib = ia + (n if layout == "halves" else 1)
        a, b = x[..., ia], x[..., ib]
        x, size = x.clone(), size.clone()
        x[..., ia], x[..., ib] = a * c - b * s, b * c + a * s
        size[..., ia] = size[..., ib] = a.abs() + b.abs()
    elif weight is None:
        return x, torch.zeros_like(x)
    return x, 20 * U * size


def attend(q, k, v, visible, scale, joined=None, there=None):
    """(out, lse, bound of out's error before its rounding, bound of lse's error) of q [n, Hq, d] over rows k, v
    [len, Hkv, d]; token i sees the entries below visible[i] of those that are `there` [len].

    A logit is a sum of d products in 32 bits, scaled: off by at most (d + 3) 2^-24 sum |q k| scale = e.  A weight is off by e and
    the exponential's error (of its argument's rounding, 2^-24 times the argument, among them), of itself, and so is their
    sum, whose additions bring (len + 16) 2^-24; bf16 weights are rounded to half a step for the product with V."""
    n, Hq, d = q.shape
    length, H, _ = k.shape
    bf16 = q.dtype == torch.bfloat16
    out = torch.zeros((n, Hq, d), dtype=torch.float64, device=q.device)
    lse = torch.full((n, Hq), -math.inf, dtype=torch.float64, device=q.device)
    e_out, e_lse = torch.zeros_like(out), torch.zeros_like(lse)
    sees = torch.arange(length, device=q.device)[None] < visible[:, None]
    if there is not None:
        sees = sees & there[None]
    for h in range(Hq if length else 0):
        kh, vh = k[:, h // (Hq // H)].double(), v[:, h // (Hq // H)].double()
        qh = q[:, h].double()
        s = (qh @ kh.T.contiguous() * scale).masked_fill(~sees, -math.inf)
        top = s.amax(1)
        some = top > -math.inf
        w = torch.exp(s - torch.where(some, top, torch.zeros_like(top))[:, None])
        w[~sees] = 0.0
        z = w.sum(1)
        lse[:, h] = torch.where(some, top + torch.log(z), top)
        p = w / torch.where(some, z, torch.ones_like(z))[:, None]
        vh = torch.where(sees.any(0)[:, None], vh, torch.zeros_like(vh))     # (nobody sees them)
        out[:, h] = p @ vh
        e = (d + 3) * U * ((qh.abs() @ kh.abs().T.contiguous()) * scale).masked_fill(~sees, 0.0).amax(1)
        away = torch.where(sees, top[:, None] - s, torch.zeros_like(s)).clamp(max=100.0).amax(1) + top.abs().clamp(max=1e6)
        e = 2 * e + (2 * away + length + 16) * U
        e = torch.where(some, e, torch.zeros_like(e))
        e_lse[:, h] = e + 4 * U * lse[:, h].abs().nan_to_num(posinf=0.0)
        e_out[:, h] = (p @ vh.abs()) * (e + (HALF_STEP[q.dtype] if bf16 else 0.0))[:, None]
    if joined is not None:
        jo, jl = joined[0].double(), joined[1].double()
        both = torch.logaddexp(lse, jl)
        ref = both.nan_to_num(neginf=0.0)
        a, b = torch.exp(lse - ref), torch.exp(jl - ref)
        jo = torch.where(b[..., None] > 0, jo, torch.zeros_like(jo))
        # both shares are off by what lse is, and the three exponentials and logarithms by a few units of their arguments
        e = e_lse + (16 + 4 * (jl.nan_to_num(neginf=0.0).abs() + lse.nan_to_num(neginf=0.0).abs())) * U
        e_out = a[..., None] * (e_out + e[..., None] * out.abs()) + b[..., None] * e[..., None] * jo.abs() + 2 * U * jo.abs()
        out = a[..., None] * out + b[..., None] * jo
        e_lse = e + 4 * U * ref.abs()
        lse = both
    return out, lse, e_out, e_lse


def check_out(got, want, bound):
    """One rounding to the type of `got` on top of the bound."""
    off = (got.double() - want).abs()
    most = bound + HALF_STEP[got.dtype] * (want.abs() + bound) + 1e-30
    assert bool((off <= most).all()), "off by %.3g of what it may be" % float((off / most).max())


def check_lse(got, want, bound):
    none = want == -math.inf
    assert torch.equal(got == -math.inf, none)
    off, most = (got.double() - want).abs()[~none], (bound + U * want.abs())[~none]
    assert bool((off <= most).all()), "off by %.3g of what it may be" % float((off / most).max())
