"""The operators around a long cache in pages, from their definitions in 64 bits or, where they only pick and move, one after the
other on the host (helper of the tests, not collected)."""
import math

import numpy as np
import torch

from plain64 import U


def scores(q, bounds):
    """q [n, Hq, d], bounds [H, blocks, 2, d] -> [n, H, blocks] in 64 bits; a sum that is no number: +inf."""
    n, Hq, d = q.shape
    H = bounds.shape[0]
    x, lo, hi = q.double().view(n, H, 1, Hq // H, d), bounds[:, :, 0].double()[:, :, None], bounds[:, :, 1].double()[:, :, None]
    out = []
    for i in range(n):
        terms = torch.where(x[i] > 0, x[i] * hi, torch.where(x[i] == 0, torch.zeros_like(lo), x[i] * lo))
        s = terms.sum(-1)
        out.append(torch.where(torch.isnan(s), math.inf, s).amax(-1))
    return torch.stack(out)


def choose(score, seen, block, first, last, chosen):
    """score [n, H, blocks], seen: numbers of entries -> int32 [n, H, chosen]."""
    n, H, _ = score.shape
    score = score.cpu().numpy()
    out = np.full((n, H, chosen), -1, np.int32)
    for i in range(n):
        nb = -(-int(seen[i]) // block)
        for h in range(H):
            if nb <= chosen:
                mine = np.arange(nb)
            else:
                between = np.arange(first, nb - last)
                best = between[np.lexsort((between, -score[i, h, first:nb - last]))][:chosen - first - last]
                mine = np.sort(np.concatenate((np.arange(first), best, np.arange(nb - last, nb))))
            out[i, h, :len(mine)] = mine
    return torch.tensor(out)


def weigh(q, lse, k, visible, scale, there=None):
    """(weights, bound of their error) [H, len] of q [n, Hq, d], lse [n, Hq] over keys k [len, H, d].

    A logit is a sum of d products in 32 bits, scaled: off by at most e = (d + 3) 2^-24 scale sum |q k|.  The exponent's argument x = s - lse is off
    by e, by the roundings of lse in units of log 2, of the factor of s (two) and its own, and the exponential by two of itself: in
    all e + (|lse| + 3 |s| + |x| + 4) 2^-24.  The sum of n G weights, in any order, brings n G 2^-24 of it."""
    n, Hq, d = q.shape
    length, H, _ = k.shape
    G = Hq // H
    weights = torch.zeros((H, length), dtype=torch.float64, device=q.device)
    bound = torch.zeros_like(weights)
    sees = torch.arange(length, device=q.device)[None] < visible[:, None]
    if there is not None:
        sees = sees & there[None]
    for h in range(Hq):
        kh, qh, l = k[:, h // G].double(), q[:, h].double(), lse[:, h].double()[:, None]
        mask = sees & (l > -math.inf)
        s = torch.where(mask, qh @ kh.T.contiguous() * scale, 0.0)
        l = torch.where(l > -math.inf, l, 0.0)
        p = torch.where(mask, torch.exp(s - l), 0.0)
        e = (d + 3) * U * (qh.abs() @ kh.abs().T.contiguous()) * scale
        weights[h // G] += p.sum(0)
        bound[h // G] += (p * (e + (l.abs() + 3 * s.abs() + (s - l).abs() + 4 + n * G) * U)).sum(0)
    return weights, bound


def evict(weights, positions, n, keep, recent, first):
    """One unit: numbers of its first n entries (numpy) -> the entry that each of `keep` places holds, -1 where none."""
    source = np.full(keep, -1, np.int64)
    if n <= keep:
        source[:n] = np.arange(n)
        return source
    positions = np.arange(n) if positions is None else positions[:n].astype(np.int64)
    newest = positions.max()

    def rank(i):
        if positions[i] > newest - recent or positions[i] < first:
            return 0, 0.0, i
        return (1, 0.0, i) if math.isnan(weights[i]) else (2, -float(weights[i]), i)
    stays = np.zeros(n, bool)
    stays[sorted(range(n), key=rank)[:keep]] = True
    source[stays[:keep]] = np.flatnonzero(stays[:keep])
    source[~stays[:keep]] = keep + np.flatnonzero(stays[keep:])
    return source
