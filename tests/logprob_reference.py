"""Class log probabilities, entropy and the gradient of the logits in 64 bits, each with a bound of what fp32 may be off.

With u = 2^-24, d = x - m and e = exp(d) of the hardware's exponential (2 ulp: 4 u) on a rounded argument (x - m, its product with a rounded
log2 e: 2.5 u |d|): an e is off by r = (2.5 |d| + 4) u of itself; sums of D terms in a row by D u more.  D: a thread adds up at most C / 32 + 200 terms one
behind the other, or all C of a short row.
"""
import math

import torch

U32 = 2.0 ** -24


def reference(logits, labels, g=None, h=None):
    x = logits.double()
    n, C = x.shape
    D = min(C, C // 32 + 200) + 2
    m = x.max(1).values
    none = torch.isinf(m) & (m < 0)
    d = x - torch.where(none, 0.0, m)[:, None]
    e = torch.exp(d)
    dz = torch.where(torch.isinf(d), 0.0, d)
    others = e.scatter(1, x.max(1).indices[:, None], 0.0).sum(1)            # without the largest term, which is 1: in 64 bits too it would eat small ones
    total = 1 + others
    l = torch.log1p(others)
    p = e / total[:, None]
    lp = dz - l[:, None]
    H = l - (p * dz).sum(1)                                                 # dz <= 0: both parts are positive
    r = (2.5 * dz.abs() + 4) * U32
    el = (p * r).sum(1) + (D + 2) * U32 * others / total + 4 * U32 * l
    q = (p * dz.abs()).sum(1)
    eH = el + (p * dz.abs() * (r + U32)).sum(1) + (D + 4) * U32 * q + q * el + 4 * U32 * H
    given = labels >= 0
    at = labels.clamp(min=0)[:, None]
    dl = dz.gather(1, at)[:, 0]
    logprob = torch.where(given, torch.where(torch.isinf(d.gather(1, at)[:, 0]) | none, -math.inf, dl - l), 0.0)
    elp = el + 2 * U32 * (dl.abs() + l)
    out = dict(m=m, l=torch.where(none, 0.0, l), el=el, H=torch.where(none, 0.0, H), eH=eH, logprob=logprob, elp=elp, lp=torch.where(torch.isinf(d) | none[:, None], -math.inf, lp))
    if g is None and h is None:
        return out
    g = torch.zeros(n, dtype=torch.float64, device=x.device) if g is None else torch.where(given, g.double(), 0.0)
    h = torch.zeros(n, dtype=torch.float64, device=x.device) if h is None else h.double()
    one = torch.zeros_like(x).scatter_(1, at, given.double()[:, None])
    first = torch.where(one > 0, -torch.expm1(lp), -p)                       # delta - p
    dx = g[:, None] * first - h[:, None] * p * (lp + H[:, None])
    ep = (2.5 * lp.abs() + 6) * U32 + el[:, None] + U32 * dz.abs()           # of p, relative
    size = g.abs()[:, None] + h.abs()[:, None] * (lp.abs() + H[:, None])
    err = p * size * (ep + 6 * U32) + p * h.abs()[:, None] * (el + eH)[:, None] + (one * g.abs()[:, None]) * (first.abs() * 4 * U32)
    masked = torch.isinf(d) | none[:, None]
    out.update(dx=torch.where(masked, 0.0, dx), edx=torch.where(masked, 0.0, err))
    return out


def top_of(logits, k):
    """Classes of the k largest logits, -1 where there are no more; of equal ones the lowest first."""
    x = logits.float()
    x = torch.where(torch.isnan(x), -math.inf, x)
    values, order = torch.sort(x, dim=1, descending=True, stable=True)
    order = torch.where(values == -math.inf, -1, order)
    return torch.nn.functional.pad(order, (0, max(0, k - order.shape[1])), value=-1)[:, :k]


def near(out, ref, err):
    """fp32 results: equal where the reference is infinite, else within err and half a step."""
    out = out.double()
    assert torch.equal(torch.isinf(ref), torch.isinf(out)) and torch.equal(out[torch.isinf(ref)], ref[torch.isinf(ref)])
    f = torch.isfinite(ref)
    off = (out - ref).abs()[f] - (err[f] + U32 * ref.abs()[f] + 2.0 ** -149)
    assert not (off > 0).any() and not torch.isnan(off).any(), "off by %.3e more than allowed" % float(off.max())
