"""The residual norm and its gradients in 64 bits, each with a bound of what fp32 may be off.

u = 2^-24.  A row's sums are chains of at most K = 24 steps (8 elements of a thread, five exchanges in a warp, four warps, and the division): off by K u of the sum of
magnitudes.  From there errors go through each formula to first order; every product, sum and square root adds its own rounding (the hardware's reciprocal
square root: 2 ulp).  Sums over rows: chains of the rows of a team, the teams of a block and the parts that one thread joins.
"""
import torch

U32 = 2.0 ** -24
K = 24


def _norm(x, ex, eps, layer):
    """h, its error, rstd, its relative error."""
    mean = x.mean(1, keepdim=True) if layer else torch.zeros_like(x[:, :1])
    em = ex.mean(1, keepdim=True) + K * U32 * x.abs().mean(1, keepdim=True) + U32 * mean.abs() if layer else 0.0
    d = x - mean
    ed = ex + em + U32 * d.abs()
    q = (d * d).mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(q + eps)
    er = ((d.abs() * ed).mean(1, keepdim=True) + 0.5 * (ed * ed).mean(1, keepdim=True) + K * U32 * q) * rstd ** 2 + 5 * U32
    h = d * rstd
    return h, ed * rstd + h.abs() * (er + 2 * U32), rstd, er, mean


def _back(d, ed, h, eh, rstd, er, layer):
    """rstd (d - mean(d) - h mean(d h)) and its error."""
    m1 = d.mean(1, keepdim=True) if layer else torch.zeros_like(rstd)
    e1 = ed.mean(1, keepdim=True) + K * U32 * d.abs().mean(1, keepdim=True) if layer else 0.0
    m2 = (d * h).mean(1, keepdim=True)
    e2 = (ed * h.abs() + d.abs() * eh).mean(1, keepdim=True) + K * U32 * (d * h).abs().mean(1, keepdim=True)
    t = d - m1 - h * m2
    et = ed + e1 + h.abs() * e2 + eh * m2.abs() + 3 * U32 * (d.abs() + m1.abs() + (h * m2).abs())
    return rstd * t, rstd * (et + t.abs() * (er + 2 * U32))


def _sum(x, ex, group, groups, steps):
    if group is None:
        return x.sum(0), ex.sum(0) + steps * U32 * x.abs().sum(0)
    z = torch.zeros(groups, x.shape[1], dtype=torch.float64, device=x.device)
    return z.index_add(0, group, x), z.index_add(0, group, ex) + steps * U32 * z.index_add(0, group, x.abs())


def reference(res, block, layer, post, post_gamma, group, groups, gate, alpha, gamma, beta, eps, dres=None, dy=None):
    """Rows of groups only; group: their numbers, None without a gate.  alpha is the fp32 value.  Returns {name: (value, error)}."""
    n, C = res.shape
    one = torch.ones(C, dtype=torch.float64, device=res.device)
    ga, pg, be = (one if gamma is None else gamma.double()), (one if post_gamma is None else post_gamma.double()), (one * 0 if beta is None else beta.double())
    r = res.double()
    zero = torch.zeros_like(r)
    out = {}
    new, enew = r, zero
    if block is not None:
        b = block.double()
        ag = (gate.double()[group] if gate is not None else torch.ones_like(r)) * alpha
        h1, eh1, rstd1, er1, mean1 = _norm(b, zero, eps, layer) if post else (b, zero, torch.ones_like(b[:, :1]), 0.0, 0.0)
        u, eu = (h1 * pg, eh1 * pg.abs() + U32 * (h1 * pg).abs()) if post else (b, zero)
        new = r + ag * u
        enew = ag.abs() * eu + U32 * (ag * u).abs() + U32 * new.abs()
        out["res"] = new, enew
    h2, eh2, rstd2, er2, _ = _norm(new, enew, eps, layer)
    y = h2 * ga + be
    out["out"] = y, eh2 * ga.abs() + U32 * (2 * (h2 * ga).abs() + y.abs())
    if dres is None and dy is None:
        return out
    shift = 0
    while (8 << shift) < C:
        shift += 1
    a_block = 256 >> shift
    teams = 296 * a_block
    steps = n // teams + 2 + min(n, teams) / 32 + a_block + 64
    D, eD = (zero, zero) if dres is None else (dres.double(), zero)
    if dy is not None:
        g = dy.double()
        out["gamma"] = _sum(g * h2, g.abs() * eh2 + U32 * (g * h2).abs(), None, 0, steps)
        out["beta"] = _sum(g, zero, None, 0, steps)
        t, et = _back(g * ga, U32 * (g * ga).abs(), h2, eh2, rstd2, er2, layer)
        D, eD = D + t, et + U32 * (D + t).abs()
    out["dres"] = D, eD
    if block is not None:
        du, edu = D * ag, eD * ag.abs() + 2 * U32 * (D * ag).abs()
        if gate is not None:
            out["gate"] = _sum(alpha * D * u, abs(alpha) * (eD * u.abs() + D.abs() * eu + 3 * U32 * (D * u).abs()), group, groups, steps)
        if post:
            out["post_gamma"] = _sum(du * h1, edu * h1.abs() + du.abs() * eh1 + U32 * (du * h1).abs(), None, 0, steps)
            out["dblock"] = _back(du * pg, edu * pg.abs() + U32 * (du * pg).abs(), h1, eh1, rstd1, er1, layer)
        else:
            out["dblock"] = du, edu
    return out
