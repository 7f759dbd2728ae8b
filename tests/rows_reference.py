"""Plain fp64 forms of the operators on typed rows, with the sums of magnitudes that their tolerances are made of.

Tolerances.  Rounding to the output's type is off by at most finfo(t).eps / 2 of the value.  A sum of m terms in fp32, in any
order, is off by at most m 2^-24 of the sum of the terms' magnitudes; where a sum may be formed with rounding toward zero
(tensor cores), by 2^-23 a step.
"""
import torch

U32 = 2.0 ** -24


def half_step(t):
    return torch.finfo(t).eps / 2


def smallest(t):
    return torch.finfo(t).smallest_normal * half_step(t) * 2      # the step of subnormal values


def close(out, ref, err):
    """|out - ref| <= half a step of the output's type + err, elementwise."""
    out64 = out.double()
    tol = err * (1 + half_step(out.dtype)) + half_step(out.dtype) * ref.abs() + smallest(out.dtype)
    bad = ~((out64 - ref).abs() <= tol)
    assert not bad.any(), "%d of %d elements off, worst %.3e with tolerance %.3e" % (
        int(bad.sum()), bad.numel(), float(torch.where(bad, (out64 - ref).abs(), torch.zeros_like(ref)).max()), float(tol[bad].max()))


def embed(ids, table, scale):
    rows = torch.where((ids >= 0)[:, None], table.double()[ids.clamp(min=0)], torch.zeros(1, dtype=torch.float64, device=table.device))
    return rows * scale


def embed_grad(ids, grad, table_rows, scale):
    """(gradient, sum of magnitudes, ids a row)."""
    keep = ids >= 0
    g, i = grad.double()[keep], ids[keep]
    z = torch.zeros(table_rows, grad.shape[1], dtype=torch.float64, device=grad.device)
    return z.index_add(0, i, g) * scale, z.index_add(0, i, g.abs()) * abs(scale), torch.bincount(i, minlength=table_rows)[:, None]


def typed(offsets, x, W, bias):
    """(product, sum of magnitudes); offsets: list."""
    out = torch.zeros(x.shape[0], W.shape[2], dtype=torch.float64, device=x.device)
    mag = torch.zeros_like(out)
    for g in range(W.shape[0]):
        b, e = offsets[g], offsets[g + 1]
        out[b:e] = x[b:e].double() @ W[g].double()
        mag[b:e] = x[b:e].double().abs() @ W[g].double().abs()
        if bias is not None:
            out[b:e] += bias[g].double()
            mag[b:e] += bias[g].double().abs()
    return out, mag


def typed_grad(offsets, x, W, dy):
    """((grad_x, magnitudes), (grad_W, ...), (grad_bias, ...))."""
    x, W, dy = x.double(), W.double(), dy.double()
    res = []
    for f in (lambda t: t, torch.abs):
        dx, dW, db = torch.zeros_like(x), torch.zeros_like(W), torch.zeros(W.shape[0], W.shape[2], dtype=torch.float64, device=x.device)
        for g in range(W.shape[0]):
            b, e = offsets[g], offsets[g + 1]
            dx[b:e] = f(dy[b:e]) @ f(W[g]).T
            dW[g] = f(x[b:e]).T @ f(dy[b:e])
            db[g] = f(dy[b:e]).sum(0)
        res.append((dx, dW, db))
    return tuple(zip(*res))


def act(name, z):
    return torch.relu(z) if name == 1 else z * torch.sigmoid(z) if name == 2 else z


def norm(offsets, x, groups, gamma, beta, eps, a, dy=None):
    """y and, with dy, the gradients (dx, dgamma, dbeta) by autograd, all in fp64; mean and rstd by graph and group."""
    n, C = x.shape
    x64 = x.double().requires_grad_(dy is not None)
    ga = (torch.ones(C, device=x.device) if gamma is None else gamma).double().requires_grad_(dy is not None)
    be = (torch.zeros(C, device=x.device) if beta is None else beta).double().requires_grad_(dy is not None)
    parts, means, rstds = [], [], []
    for b, e in zip(offsets, offsets[1:]):
        if e <= b:
            means.append(torch.zeros(groups, dtype=torch.float64, device=x.device)); rstds.append(means[-1])
            continue
        p = x64[b:e].reshape(e - b, groups, C // groups)
        m = p.mean((0, 2), keepdim=True)
        r = 1 / torch.sqrt(((p - m) ** 2).mean((0, 2), keepdim=True) + eps)
        parts.append(act(a, ((p - m) * r).reshape(e - b, C) * ga + be))
        means.append(m.detach().flatten()); rstds.append(r.detach().flatten())
    y = torch.cat(parts) if parts else x64[:0]
    if dy is None:
        return y, torch.stack(means), torch.stack(rstds)
    grads = torch.autograd.grad(y, (x64, ga, be), dy.double()[offsets[0]:offsets[-1]])
    return y.detach(), torch.stack(means), torch.stack(rstds), grads
