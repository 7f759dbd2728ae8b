"""Group norm with an activation over batches of graphs, and its gradients, against fp64."""
import pytest
import torch

import paper_2607_17374_b200 as tb
from rows_reference import U32, act, close, half_step, norm

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
EPS = 1e-5


def strided(n, width, ld, dtype, shift=0):
    store = torch.full((shift + max(n, 1) * ld + 8,), 7.0, dtype=dtype, device="cuda")
    return torch.as_strided(store, (n, width), (ld, 1), shift), store


def workspace(size):
    return torch.full((size,), 255, dtype=torch.uint8, device="cuda") if size else None


def batch(sizes):
    """Offsets of graphs of these sizes; negative ones in front and behind are rows of no graph."""
    off = [-sizes[0] if sizes[0] < 0 else 0]
    for s in sizes:
        if s >= 0:
            off.append(off[-1] + s)
    return off, off[-1] + (-sizes[-1] if len(sizes) > 1 and sizes[-1] < 0 else 0)


def run(off, n, x, groups, gamma, beta, a, out, dy=None, dx=None, status=None):
    C, G = x.shape[1], len(off) - 1
    o = torch.tensor(off, device="cuda")
    mean, rstd = torch.full((G, groups), 5.0, device="cuda"), torch.full((G, groups), 5.0, device="cuda")
    tb.norm_rows(n, G, o, x, x.stride(0), C, groups, gamma, beta, EPS, a, out, out.stride(0), mean, rstd, workspace(tb.norm_rows_workspace(n, G, C, groups)), status)
    if dy is None:
        return mean, rstd
    dga, dbe = torch.full((C,), 5.0, device="cuda"), torch.full((C,), 5.0, device="cuda")
    tb.norm_rows_grad(n, G, o, x, x.stride(0), C, groups, gamma, beta, a, mean, rstd, dy, dy.stride(0), dx, dx.stride(0), dga, dbe,
                      workspace(tb.norm_rows_grad_workspace(n, G, C, groups)), status)
    return mean, rstd, dga, dbe


SHAPES = [
    # sizes, width, groups
    ([1], 1, 1), ([1], 8, 2), ([2, 1, 0, 3], 64, 8), ([-3, 20, 0, 7, -2], 47, 47), ([26] * 40, 64, 8), ([5, 300, 1, 0, 77], 100, 25), ([1000], 96, 1), ([9, 2500, 30], 256, 16),
    ([5000, 3, 4000], 33, 3), ([40_000], 16, 4), ([-100, 30_000, 1, 25_000, -7], 24, 24), ([3000, 3000], 1024, 32), ([700], 1023, 11), ([100, 60], 514, 257), ([50_001], 7, 1),
    ([1] * 500, 40, 5), ([20_000] + [3] * 200 + [20_000], 32, 2),
]


def bounds(off, x, groups, gamma, beta, mean, rstd):
    """Error of z = gamma (x - mean) rstd + beta.  Sums over a graph's m elements are of x - pivot, |x - pivot| <= span, in chains of at most
    `chain` steps: the mean is off by chain 2^-24 span + 2^-24 |mean|, the variance by 4 chain 2^-24 span^2 at most, rstd by half of that
    relative to var + eps.  (span: the graph's range of the group.)"""
    n, C = x.shape
    ez = torch.zeros(n, C, dtype=torch.float64, device="cuda")
    xh = torch.zeros_like(ez)
    er = torch.zeros(len(off) - 1, groups, dtype=torch.float64, device="cuda")
    for s, (b, e) in enumerate(zip(off, off[1:])):
        if e <= b:
            continue
        p = x[b:e].double().reshape(e - b, groups, -1)
        span = (p.amax((0, 2)) - p.amin((0, 2)))
        chain = min(e - b, 64 + (e - b) // 8) + 40
        em = chain * U32 * span + 4 * U32 * mean[s].abs()
        er[s] = 4 * chain * U32 * span ** 2 * rstd[s] ** 2 + (em * rstd[s]) ** 2 + 8 * U32
        h = ((p - mean[s][None, :, None]) * rstd[s][None, :, None])
        ex = em * rstd[s] + 2 * U32 * rstd[s] * mean[s].abs()
        e_xh = ex[None, :, None] + h.abs() * (er[s][None, :, None] + 4 * U32)
        xh[b:e], ez[b:e] = h.reshape(e - b, C), e_xh.reshape(e - b, C)
    g = 1.0 if gamma is None else gamma.double().abs()
    ezz = ez * g + 4 * U32 * (xh.abs() * g + (0 if beta is None else beta.double().abs()))
    return xh, ez, ezz, er


@pytest.mark.parametrize("t", [F32, BF16, F16])
@pytest.mark.parametrize("a", [tb.ACT_NONE, tb.ACT_RELU, tb.ACT_SILU])
@pytest.mark.parametrize("sizes,C,groups", SHAPES)
@pytest.mark.parametrize("pad,shift,affine", [(0, 0, True), (8, 0, False), (3, 1, True)])
def test_norm_and_gradients(t, a, sizes, C, groups, pad, shift, affine):
    off, n = batch(sizes)
    g = torch.Generator("cuda").manual_seed(C + n)
    x, _ = strided(n, C, C + pad, t, shift)
    x.copy_(torch.randn(n, C, generator=g, device="cuda") * 1.5 + torch.randn(C, generator=g, device="cuda"))
    dy, _ = strided(n, C, C + pad, t, shift)
    dy.copy_(torch.randn(n, C, generator=g, device="cuda"))
    gamma = 1 + 0.3 * torch.randn(C, generator=g, device="cuda") if affine else None
    beta = 0.3 * torch.randn(C, generator=g, device="cuda") if affine else None
    if a == tb.ACT_RELU:                                 # away from the border, where the slope jumps
        _, m, r = norm(off, x, groups, gamma, beta, EPS, tb.ACT_NONE)
        z = torch.zeros(n, C, dtype=torch.float64, device="cuda")
        z[off[0]:off[-1]] = norm(off, x, groups, gamma, beta, EPS, tb.ACT_NONE)[0]
        dy[z.abs() < 0.05] = 0
    out, store = strided(n, C, C + pad, t, shift)
    dx, dstore = strided(n, C, C + pad, t, shift)
    before, dbefore = store.clone(), dstore.clone()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    mean, rstd, dga, dbe = run(off, n, x, groups, gamma, beta, a, out, dy, dx, status)
    y, rm, rr, (rx, rga, rbe) = norm(off, x, groups, gamma, beta, EPS, a, dy)
    lo, hi = off[0], off[-1]
    xh, ex, ez, er = bounds(off, x, groups, gamma, beta, rm, rr)
    assert int(status) == 0
    assert ((rstd.double() - rr).abs() <= er * rr + 8 * U32 * rr).all()
    # |act'| <= 1.1, and expf and the division are right to 4 ulp
    close(out[lo:hi], y, (ez * 1.1 + 8 * U32 * 1.1)[lo:hi] + 8 * U32 * y.abs())
    # slope of silu: |act''| <= 0.5; sums over a graph's elements in chains of at most `chain` steps
    gm = torch.ones(C, dtype=torch.float64, device="cuda") if gamma is None else gamma.double()
    z = xh * gm + (0 if beta is None else beta.double())
    slope = torch.ones_like(z) if a == 0 else (z > 0).double() if a == 1 else torch.sigmoid(z) * (1 + z * (1 - torch.sigmoid(z)))
    dz = dy.double() * slope
    edz = dy.double().abs() * ((0.5 * ez if a == 2 else 0) + 12 * U32 * 1.1)
    tol = torch.zeros(n, C, dtype=torch.float64, device="cuda")
    tga, tbe = torch.zeros(C, dtype=torch.float64, device="cuda"), torch.zeros(C, dtype=torch.float64, device="cuda")
    for s, (b, e) in enumerate(zip(off, off[1:])):
        if e <= b:
            continue
        chain = (min(e - b, 64 + (e - b) // 8) + 40) * U32
        q, eq, h, eh = (dz[b:e] * gm), edz[b:e] * gm.abs(), xh[b:e], ex[b:e]
        v = lambda w: w.reshape(e - b, groups, -1)
        m2, em2 = v(q).mean((0, 2)).abs(), v(eq + chain * q.abs()).mean((0, 2))
        m1, em1 = v(q * h).mean((0, 2)).abs(), v(eq * h.abs() + q.abs() * eh + chain * (q * h).abs()).mean((0, 2))
        total = v(eq + 4 * U32 * q.abs()) + (em2 + 4 * U32 * m2)[None, :, None] + v(h.abs()) * (em1 + 4 * U32 * m1)[None, :, None] + v(eh) * m1[None, :, None]
        size = v(q.abs()) + m2[None, :, None] + v(h.abs()) * m1[None, :, None]
        tol[b:e] = (rr[s][None, :, None] * (total + size * (er[s][None, :, None] + 8 * U32))).reshape(e - b, C)
        tga += (edz[b:e] * h.abs() + dz[b:e].abs() * eh + chain * (dz[b:e] * h).abs()).sum(0)
        tbe += (edz[b:e] + chain * dz[b:e].abs()).sum(0)
    close(dx[lo:hi], rx[lo:hi], tol[lo:hi] * 1.05)       # (1.05: products of two errors)
    close(dga, rga, tga * 1.05 + 64 * U32 * (dz * xh).abs().sum(0))
    close(dbe, rbe, tbe * 1.05 + 64 * U32 * dz.abs().sum(0))
    torch.as_strided(before, (n, C), (C + pad, 1), shift)[lo:hi] = out[lo:hi]
    torch.as_strided(dbefore, (n, C), (C + pad, 1), shift)[lo:hi] = dx[lo:hi]
    assert torch.equal(before, store) and torch.equal(dbefore, dstore)      # rows of no graph, and what lies between the rows
    again = [out.clone(), dx.clone(), dga, dbe]
    _, _, dga2, dbe2 = run(off, n, x, groups, gamma, beta, a, out, dy, dx)
    assert all(torch.equal(p, q) for p, q in zip(again, (out, dx, dga2, dbe2)))


def test_one_graph_without_offsets_and_in_place():
    for n in (1, 50, 9000):
        x = torch.randn(n, 64, device="cuda") * 3 + 1
        dy = torch.randn(n, 64, device="cuda")
        a, b = torch.empty_like(x), torch.empty_like(x)
        mean, rstd = run([0, n], n, x, 4, None, None, tb.ACT_SILU, a)
        ws = workspace(tb.norm_rows_workspace(n, 1, 64, 4))
        tb.norm_rows(n, 1, None, x, 64, 64, 4, None, None, EPS, tb.ACT_SILU, b, 64, None, None, ws)
        assert torch.equal(a, b)
        g = [torch.empty_like(x) for _ in range(2)]
        gw = workspace(tb.norm_rows_grad_workspace(n, 1, 64, 4))
        tb.norm_rows_grad(n, 1, None, x, 64, 64, 4, None, None, tb.ACT_SILU, mean, rstd, dy, 64, g[0], 64, None, None, gw)
        same = dy.clone()
        tb.norm_rows_grad(n, 1, None, x, 64, 64, 4, None, None, tb.ACT_SILU, mean, rstd, same, 64, same, 64, None, None, gw)
        assert torch.equal(g[0], same)
        same = x.clone()
        tb.norm_rows_grad(n, 1, None, same, 64, 64, 4, None, None, tb.ACT_SILU, mean, rstd, dy, 64, same, 64, None, None, gw)
        assert torch.equal(g[0], same)
        tb.norm_rows(n, 1, None, x, 64, 64, 4, None, None, EPS, tb.ACT_SILU, x, 64, None, None, ws)
        assert torch.equal(a, x)


def test_offset_and_outlier_do_not_eat_the_variance():
    """A large common offset, and one element 1e6 times as large as the others, leave fp32's own error only."""
    n, C, groups = 6000, 32, 4
    g = torch.Generator("cuda").manual_seed(1)
    noise = torch.randn(n, C, generator=g, device="cuda")
    for where in (None, 0, 3333):
        x = noise + 1e4
        if where is not None:
            x = noise.clone()
            x[where, 3] = 1e6
        out = torch.empty_like(x)
        run([0, n], n, x, groups, None, None, 0, out)
        y, m, r = norm([0, n], x, groups, None, None, EPS, 0)
        # (x - mean): mean is off by half an ulp of it and the chain's rounding of deviations
        err = (out.double() - y).abs()
        scale = (x.double().abs().amax() * r.max() * 4 * U32) if where is None else 0
        assert (err <= scale + 200 * U32 * (y.abs() + 1)).all()


def test_not_a_number_stays_in_its_graph():
    off, n = [0, 40, 20_040, 20_100], 20_100
    x = torch.randn(n, 32, device="cuda")
    clean, foul = torch.empty_like(x), torch.empty_like(x)
    run(off, n, x, 4, None, None, tb.ACT_RELU, clean)
    x[50, 3], x[20_050, 9] = float("nan"), float("inf")
    run(off, n, x, 4, None, None, tb.ACT_RELU, foul)
    assert torch.equal(clean[:40], foul[:40])
    assert torch.equal(clean[40:20_040, 8:], foul[40:20_040, 8:]) and foul[40:20_040, :8].isnan().all()
    assert torch.equal(clean[20_040:, 16:], foul[20_040:, 16:]) and torch.equal(clean[20_040:, :8], foul[20_040:, :8])


@pytest.mark.parametrize("bad", [[0, 500, 400, 30_000], [-5, 50, 90, 30_000], [0, 50, 90, 30_001], [30_000, 20_000, 100, 0], [0, 1 << 40, 90, 30_000]])
def test_bad_offsets_give_a_status(bad):
    n, C = 30_000, 16
    x = torch.ones(n, C, device="cuda")
    out, store = strided(n, C, C, F32)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    mean, rstd = run(bad, n, x, 2, None, None, 1, out, status=status)
    assert int(status) == tb.ERROR_CODES["INVALID_ARG"] and (store[n * C:] == 7).all()
    status.zero_()
    tb.norm_rows_grad(n, 3, torch.tensor(bad, device="cuda"), x, C, C, 2, None, None, 1, mean, rstd, x, C, out, C, None, None, workspace(tb.norm_rows_grad_workspace(n, 3, C, 2)), status)
    assert int(status) == tb.ERROR_CODES["INVALID_ARG"] and (store[n * C:] == 7).all()


def test_without_rows():
    off = torch.zeros(4, dtype=torch.int64, device="cuda")
    mean, rstd = torch.ones(3, 2, device="cuda"), torch.ones(3, 2, device="cuda")
    tb.norm_rows(0, 3, off, None, 8, 8, 2, None, None, EPS, 0, None, 8, mean, rstd, type=tb.F32)
    assert (mean == 0).all() and (rstd == 0).all()
    dga, dbe = torch.ones(8, device="cuda"), torch.ones(8, device="cuda")
    tb.norm_rows_grad(0, 3, off, None, 8, 8, 2, None, None, 0, mean, rstd, None, 8, None, 8, dga, dbe, type=tb.F32)
    assert (dga == 0).all() and (dbe == 0).all()


def test_gradient_against_differences():
    """<r, y> along a direction d, central differences with step h in fp64 of the fp32 outputs: h^2 / 6 of the third derivative and 2^-24 / h of the
    outputs' rounding stay below 2e-3 of |r| |d| here (h = 1/64, derivatives of order one, rows of unit variance)."""
    off, n, C, groups = [0, 60, 61, 400], 400, 48, 6
    g = torch.Generator("cuda").manual_seed(4)
    x, d, r = (torch.randn(n, C, generator=g, device="cuda") for _ in range(3))
    gamma, beta = 1 + 0.2 * torch.randn(C, generator=g, device="cuda"), 0.2 * torch.randn(C, generator=g, device="cuda")
    out, dx = torch.empty_like(x), torch.empty_like(x)
    h = 2.0 ** -6
    _, _, dga, dbe = run(off, n, x, groups, gamma, beta, tb.ACT_SILU, out, r, dx)

    def loss(x, gamma, beta):
        run(off, n, x, groups, gamma, beta, tb.ACT_SILU, out)
        return float((out.double() * r.double()).sum())
    dg = torch.randn(C, generator=g, device="cuda")
    for grad, dirn, plus, minus in ((dx, d, (x + h * d, gamma, beta), (x - h * d, gamma, beta)), (dga, dg, (x, gamma + h * dg, beta), (x, gamma - h * dg, beta)),
                                    (dbe, dg, (x, gamma, beta + h * dg), (x, gamma, beta - h * dg))):
        num = (loss(*plus) - loss(*minus)) / (2 * h)
        assert abs(num - float((grad.double() * dirn.double()).sum())) <= 2e-3 * float(r.double().norm() * d.double().norm())


def test_refused_on_a_device():
    x, out = torch.zeros(4, 8, device="cuda"), torch.zeros(4, 8, device="cuda")
    off = torch.tensor([0, 4], device="cuda")
    for bad in (dict(x=x.cpu()), dict(off=off.cpu()), dict(out=out.cpu()), dict(gamma=torch.zeros(8)), dict(mean=torch.zeros(2)), dict(out=torch.as_strided(x, (2, 8), (16, 1)), n=2)):
        a = dict(x=x, off=off, out=out, gamma=None, mean=None, n=4)
        a.update(bad)
        with pytest.raises(tb.TaurusError) as e:
            tb.norm_rows(a["n"], 1, a["off"], a["x"], 8, 8, 2, a["gamma"], None, EPS, 1, a["out"], a["out"].stride(0), a["mean"], None)
        assert e.value.code == tb.ERROR_CODES["INVALID_ARG"]
    big = torch.zeros(9000, 64, device="cuda")
    need = tb.norm_rows_workspace(9000, 1, 64, 4)
    assert need > 0
    for ws in (None, torch.empty(need - 1, dtype=torch.uint8, device="cuda"), big.view(torch.uint8)):
        with pytest.raises(tb.TaurusError) as e:
            tb.norm_rows(9000, 1, None, big, 64, 64, 4, None, None, EPS, 1, torch.empty_like(big), 64, None, None, ws)
        assert e.value.code == tb.ERROR_CODES["INVALID_ARG"]


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("width", [1, 6, 24])
@pytest.mark.parametrize("action", [tb.ACT_NONE, tb.ACT_SILU])
def test_an_element_alone_in_its_group_has_no_gradient(t, width, action):
    """Its output does not depend on it: exactly zero, not what rounding leaves of it times 1 / sqrt(eps)."""
    g = torch.Generator("cuda").manual_seed(width)
    n = 50
    x, dy = (torch.randn(n, width, generator=g, device="cuda").to(t) for _ in range(2))
    gamma, beta = torch.randn(width, generator=g, device="cuda"), torch.randn(width, generator=g, device="cuda")
    off = torch.arange(n + 1, device="cuda")
    mean, rstd = torch.empty(n, width, device="cuda"), torch.empty(n, width, device="cuda")
    y, dx = torch.empty_like(x), torch.full_like(x, 3.0)
    ws = torch.empty(max(tb.norm_rows_grad_workspace(n, n, width, width), 256), dtype=torch.uint8, device="cuda")
    tb.norm_rows(n, n, off, x, width, width, width, gamma, beta, 1e-5, action, y, width, mean, rstd, ws)
    tb.norm_rows_grad(n, n, off, x, width, width, width, gamma, beta, action, mean, rstd, dy, width, dx, width, None, None, ws)
    assert torch.equal(mean, x.float()) and (dx == 0).all()


def many(graphs, seed=1):
    """Sizes of a large batch: graphs of 0 to 12 rows, and two beyond the length that one block takes."""
    g = torch.Generator().manual_seed(seed)
    sizes = (torch.rand(graphs, generator=g) ** 2 * 13).long().tolist()
    sizes[graphs // 3], sizes[-7] = 2000, 5000
    return sizes


@pytest.mark.parametrize("t,a,C,groups,pad,shift", [(F32, tb.ACT_SILU, 64, 8, 0, 0), (BF16, tb.ACT_SILU, 64, 8, 0, 0), (F16, tb.ACT_NONE, 33, 3, 0, 0), (F32, tb.ACT_RELU, 40, 20, 3, 1),
                                                    (BF16, tb.ACT_SILU, 96, 1, 8, 0)])
def test_many_graphs(t, a, C, groups, pad, shift):
    """More graphs than the gradient's kernel has blocks, so that each block has several, some empty, and a few long ones among them."""
    test_norm_and_gradients(t, a, many(6000), C, groups, pad, shift, True)


@pytest.mark.parametrize("t", [F32, BF16, F16])
@pytest.mark.parametrize("C,groups", [(8, 2), (6, 3)])
def test_more_graphs_than_blocks(t, C, groups):
    """More than 2^20 graphs: each block of the forward call has several.  The bits are those of calls over a part of the batch, of the same average size (which the block's threads
    depend on), and gradients of gamma and beta those of the parts' sums."""
    G, parts = (1 << 20) + 4096, 16
    sizes = torch.tensor([1, 2, 0, 3, 2, 0, 1, 7] * (G // 8), device="cuda")
    off = torch.cat([sizes.new_zeros(1), sizes.cumsum(0)])
    n, per = int(off[-1]), G // parts
    g = torch.Generator("cuda").manual_seed(8)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")
    x, dy, gamma, beta = r(n, C).to(t), r(n, C).to(t), 1 + 0.1 * r(C), 0.1 * r(C)

    def call(off, x, dy):
        n, G = x.shape[0], off.numel() - 1
        out, dx, mean, rstd, dga, dbe = (torch.full(s, 5.0, dtype=d, device="cuda") for s, d in (((n, C), t), ((n, C), t), ((G, groups), F32), ((G, groups), F32), ((C,), F32), ((C,), F32)))
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        tb.norm_rows(n, G, off, x, C, C, groups, gamma, beta, EPS, tb.ACT_SILU, out, C, mean, rstd, workspace(tb.norm_rows_workspace(n, G, C, groups)), status)
        tb.norm_rows_grad(n, G, off, x, C, C, groups, gamma, beta, tb.ACT_SILU, mean, rstd, dy, C, dx, C, dga, dbe, workspace(tb.norm_rows_grad_workspace(n, G, C, groups)), status)
        assert int(status) == 0
        return out, dx, mean, rstd, dga.double(), dbe.double()
    whole = call(off, x, dy)
    pieces = []
    for p in range(parts):
        o = off[p * per:(p + 1) * per + 1]
        b, e = int(o[0]), int(o[-1])
        pieces.append(call((o - b).contiguous(), x[b:e], dy[b:e]))
    for i, got in enumerate(whole[:4]):
        assert torch.equal(got, torch.cat([p[i] for p in pieces]))
    # terms of order one (|dz| <= 1.1 |dy|, |xh| <= sqrt of the group's elements), at most 2^12 of them to a thread's sum on either side
    y, _, _, (_, rga, rbe) = norm(off[:per + 1].tolist()[:2001], x[:int(off[2000])], groups, gamma, beta, EPS, tb.ACT_SILU, dy[:int(off[2000])])
    small = call(off[:2001].contiguous(), x[:int(off[2000])], dy[:int(off[2000])])
    size = dy.double().abs().sum(0) * 1.1
    span = (7 * C / groups) ** 0.5
    for i, ref, scale in ((4, rga, span), (5, rbe, 1.0)):
        assert ((small[i] - ref).abs() <= 4096 * U32 * size * scale).all()
        assert ((whole[i] - sum(p[i] for p in pieces)).abs() <= 2 * 4096 * U32 * size * scale).all()
