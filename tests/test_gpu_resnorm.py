"""The residual norm and its gradients against fp64: types, widths, pitches, groups that are empty, long, many or none, in place, captured."""
import pytest
import torch

import paper_2607_17374_b200 as tb
from resnorm_reference import reference
from rows_reference import close

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
EPS = 1e-5
LAYER, RMS = tb.NORM_LAYER, tb.NORM_RMS


def strided(n, width, ld, dtype, shift=0):
    store = torch.full((shift + max(n, 1) * ld + 8,), 7.0, dtype=dtype, device="cuda")
    return torch.as_strided(store, (n, width), (ld, 1), shift), store


def untouched(store, n, width, ld, shift, rows=None):
    inside = torch.zeros_like(store, dtype=torch.bool)
    v = torch.as_strided(inside, (n, width), (ld, 1), shift)
    (v if rows is None else v[rows[0]:rows[1]]).fill_(True)
    assert (store[~inside] == 7).all()


def batch(sizes):
    """Offsets of groups of these sizes; negative ones in front and behind are rows of no group."""
    off = [-sizes[0] if sizes[0] < 0 else 0]
    for s in sizes:
        if s >= 0:
            off.append(off[-1] + s)
    return off, off[-1] + (-sizes[-1] if len(sizes) > 1 and sizes[-1] < 0 else 0)


class Case:
    def __init__(self, sizes, C, t, r, kind=LAYER, post=True, gate=True, pad=0, shift=0, affine=True, seed=0):
        self.off, self.n = batch(sizes)
        n = self.n
        g = torch.Generator("cuda").manual_seed(seed + C + n)
        self.C, self.t, self.r, self.kind, self.post, self.ld, self.shift = C, t, r, kind, post, C + pad, shift

        def rows(dtype, scale, offset=0.0):
            x, _ = strided(n, C, self.ld, dtype, shift)
            x.copy_(torch.randn(n, C, generator=g, device="cuda") * scale + offset * torch.randn(C, generator=g, device="cuda"))
            return x

        self.res, self.block = rows(r, 1.5, 0.5), rows(t, 0.7, 0.3)
        self.dres, self.dy = rows(r, 1.0), rows(t, 1.0)

        def vector(base, scale, *shape):
            return base + scale * torch.randn(*shape, generator=g, device="cuda")

        self.gamma, self.beta = (vector(1, 0.2, C), vector(0, 0.2, C)) if affine else (None, None)
        self.post_gamma = vector(1, 0.2, C) if post and affine else None
        self.groups = len(self.off) - 1 if gate else 0
        self.gate, self.offsets = (vector(0.5, 0.4, self.groups, C), torch.tensor(self.off, device="cuda")) if gate else (None, None)
        self.lo, self.hi = (self.off[0], self.off[-1]) if gate else (0, n)
        self.alpha = 0.75
        self.group = torch.repeat_interleave(torch.arange(self.groups, device="cuda"), self.offsets.diff()) if gate else None
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def forward(self, out_res, out, stats=None, res=None, block=None, stream=None):
        res, block = self.res if res is None else res, self.block if block is None else block
        tb.residual_norm(self.n, self.C, res, self.ld, block, self.ld, self.kind, self.post, self.post_gamma, self.groups, self.offsets, self.gate, self.alpha, self.gamma, self.beta, EPS,
                         out_res, out_res.stride(0), out, out.stride(0), stats, self.status, stream)

    def space(self):
        size = tb.residual_norm_grad_workspace(self.n, self.C, self.groups)
        return torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda") if size else None

    def sums(self):
        full = lambda *s: torch.full(s, 55.0, device="cuda")  # noqa: E731
        return dict(grad_post_gamma=full(self.C) if self.post else None, grad_gate=full(self.groups, self.C) if self.groups else None, grad_gamma=full(self.C), grad_beta=full(self.C))

    def backward(self, stats, d_res, d_block, sums, dres="own", dy="own", res=None, block=None, stream=None, workspace="own"):
        dres, dy = self.dres if isinstance(dres, str) else dres, self.dy if isinstance(dy, str) else dy
        tb.residual_norm_grad(self.n, self.C, self.res if res is None else res, self.ld, self.block if block is None else block, self.ld, self.kind, self.post, self.post_gamma, self.groups,
                              self.offsets, self.gate, self.alpha, self.gamma, stats, dres, self.ld, dy, self.ld, d_res, self.ld, d_block, self.ld,
                              workspace=self.space() if isinstance(workspace, str) else workspace, status=self.status, stream=stream, **sums)

    def reference(self, dres="own", dy="own"):
        s = slice(self.lo, self.hi)
        dres, dy = self.dres if isinstance(dres, str) else dres, self.dy if isinstance(dy, str) else dy
        return reference(self.res[s], self.block[s], self.kind == LAYER, self.post, self.post_gamma, self.group, self.groups, self.gate, self.alpha, self.gamma, self.beta, EPS,
                         None if dres is None else dres[s], None if dy is None else dy[s])


SHAPES = [([1], 4), ([1], 8), ([2, 1, 0, 3], 64), ([-3, 20, 0, 7, -2], 47), ([26] * 40, 64), ([5, 300, 1, 0, 77], 100), ([1000], 96), ([9, 2500, 30], 256), ([5000, 3, 4000], 33),
          ([-100, 3000, 1, 2500, -7], 24), ([300, 0, 0, 0, 0, 0, 0, 300], 1024), ([700], 1023), ([100, 60], 514), ([0] * 70 + [41] + [0] * 9, 40), ([1] * 900, 320), ([30_000, 5], 8), ([1] * 3000, 6),
          ([2000], 12), ([1500, 700], 260), ([3, 4000, 2, 2], 512)]
TYPES = [(F32, F32), (BF16, BF16), (BF16, F32), (F16, F16), (F16, F32)]


@pytest.mark.parametrize("t,r", TYPES)
@pytest.mark.parametrize("sizes,C", SHAPES)
@pytest.mark.parametrize("kind,post,gate,pad,shift,affine", [(LAYER, True, True, 0, 0, True), (RMS, True, True, 8, 0, True), (LAYER, False, True, 3, 1, False), (RMS, False, False, 0, 0, True),
                                                              (LAYER, True, False, 4, 4, True)])
def test_forward_and_gradients(t, r, sizes, C, kind, post, gate, pad, shift, affine):
    c = Case(sizes, C, t, r, kind, post, gate, pad, shift, affine)
    n, ld = c.n, c.ld
    (out_res, s1), (out, s2), (d_res, s3), (d_block, s4) = (strided(n, C, ld, x, shift) for x in (r, t, r, t))
    stats, sums = torch.empty(n, 4, device="cuda"), c.sums()
    c.forward(out_res, out, stats)
    c.backward(stats, d_res, d_block, sums)
    ref = c.reference()
    rows = slice(c.lo, c.hi)
    for got, name in ((out_res[rows], "res"), (out[rows], "out"), (d_res[rows], "dres"), (d_block[rows], "dblock"), (sums["grad_gamma"], "gamma"), (sums["grad_beta"], "beta"),
                      (sums["grad_post_gamma"], "post_gamma"), (sums["grad_gate"], "gate")):
        if got is not None:
            close(got, *ref[name])
    for s in (s1, s2, s3, s4):
        untouched(s, n, C, ld, shift, (c.lo, c.hi))
    assert int(c.status) == 0


@pytest.mark.parametrize("t,r", [(F32, F32), (BF16, F32)])
@pytest.mark.parametrize("which", ["dres", "dy"])
@pytest.mark.parametrize("post", [True, False])
def test_one_gradient_alone(t, r, which, post):
    c = Case([50, 0, 333], 130, t, r, post=post)
    stats = torch.empty(c.n, 4, device="cuda")
    c.forward(torch.empty_like(c.res), torch.empty_like(c.block), stats)
    given = dict(dres=c.dres if which == "dres" else None, dy=c.dy if which == "dy" else None)
    ref = c.reference(**given)
    d_res, d_block, sums = torch.empty_like(c.res), torch.empty_like(c.block), c.sums()
    c.backward(stats, d_res, d_block, sums, **given)
    close(d_res, *ref["dres"])
    close(d_block, *ref["dblock"])
    close(sums["grad_gate"], *ref["gate"])
    if which == "dy":
        close(sums["grad_gamma"], *ref["gamma"])
    else:
        assert (sums["grad_gamma"] == 0).all() and (sums["grad_beta"] == 0).all()
    # fewer outputs, the same values
    e_res = torch.empty_like(c.res)
    c.backward(stats, e_res, None, {}, workspace=None, **given)
    assert torch.equal(d_res, e_res)
    for name in [k for k, v in sums.items() if v is not None]:
        alone = {name: torch.full_like(sums[name], 3.0)}
        c.backward(stats, e_res, None, alone, **given)
        assert torch.equal(alone[name], sums[name]), name


@pytest.mark.parametrize("t", [F32, BF16])
@pytest.mark.parametrize("kind", [LAYER, RMS])
def test_the_norm_alone(t, kind):
    """Without a block: the norm in front of the first one."""
    n, C = 333, 200
    x, dy, dres = (torch.randn(n, C, device="cuda").to(t) for _ in range(3))
    gamma, beta = 1 + 0.1 * torch.randn(C, device="cuda"), torch.randn(C, device="cuda")
    y, stats, dx, dga = torch.empty_like(x), torch.empty(n, 4, device="cuda"), torch.empty_like(x), torch.empty(C, device="cuda")
    tb.residual_norm(n, C, x, C, None, C, kind, 0, None, 0, None, None, 1.0, gamma, beta, EPS, None, C, y, C, stats)
    ref = reference(x, None, kind == LAYER, False, None, None, 0, None, 1.0, gamma, beta, EPS, dres, dy)
    close(y, *ref["out"])
    ws = torch.empty(tb.residual_norm_grad_workspace(n, C, 0), dtype=torch.uint8, device="cuda")
    tb.residual_norm_grad(n, C, x, C, None, C, kind, 0, None, 0, None, None, 1.0, gamma, stats, dres, C, dy, C, dx, C, grad_gamma=dga, workspace=ws)
    close(dx, *ref["dres"])
    close(dga, *ref["gamma"])


@pytest.mark.parametrize("t,r", [(F32, F32), (F16, F32)])
@pytest.mark.parametrize("C", [48, 600])
def test_in_place(t, r, C):
    c = Case([40, 500, 3], C, t, r)
    out_res, out, stats = torch.empty_like(c.res), torch.empty_like(c.block), torch.empty(c.n, 4, device="cuda")
    c.forward(out_res, out, stats)
    a, b = c.res.clone(), c.block.clone()
    c.forward(a, b, None, res=a, block=b)
    assert torch.equal(a, out_res) and torch.equal(b, out)
    d_res, d_block, sums = torch.empty_like(c.res), torch.empty_like(c.block), c.sums()
    c.backward(stats, d_res, d_block, sums)
    for over in ("inputs", "gradients"):
        a, b = (c.res.clone(), c.block.clone()) if over == "inputs" else (c.dres.clone(), c.dy.clone())
        again = c.sums()
        c.backward(stats, a, b, again, **(dict(res=a, block=b) if over == "inputs" else dict(dres=a, dy=b)))
        assert torch.equal(a, d_res) and torch.equal(b, d_block) and all(torch.equal(again[k], sums[k]) for k in sums)


def test_rows_of_no_group_may_hold_anything():
    c = Case([-5, 60, 0, 9, -4], 72, F32, F32)
    ref = c.reference()
    for x in (c.res, c.block, c.dres, c.dy):
        x[:5] = float("nan")
        x[-4:] = float("inf")
    stats = torch.full((c.n, 4), float("nan"), device="cuda")
    out_res, out, d_res, d_block, sums = torch.empty_like(c.res), torch.empty_like(c.block), torch.empty_like(c.res), torch.empty_like(c.block), c.sums()
    c.forward(out_res, out, stats)
    c.backward(stats, d_res, d_block, sums)
    for got, name in ((out[5:-4], "out"), (d_res[5:-4], "dres"), (sums["grad_gamma"], "gamma"), (sums["grad_gate"], "gate"), (sums["grad_post_gamma"], "post_gamma")):
        close(got, *ref[name])


def test_a_large_mean_does_not_eat_the_variance():
    n, C = 64, 256
    g = torch.Generator("cuda").manual_seed(1)
    x = 1e4 + torch.randn(n, C, generator=g, device="cuda")
    y = torch.empty_like(x)
    tb.residual_norm(n, C, x, C, None, C, LAYER, 0, None, 0, None, None, 1.0, None, None, EPS, None, C, y, C)
    close(y, *reference(x, None, True, False, None, None, 0, None, 1.0, None, None, EPS)["out"])
    assert abs(float(y.double().std()) - 1) < 1e-2          # the sample's own spread: 1 / sqrt(2 x 16 384) = 0.6 %


@pytest.mark.parametrize("offsets", [[0, 5, 3, 10], [-1, 4, 8, 10], [0, 4, 8, 11], [7, 2, 1, 0], [1 << 40, 1 << 41, 1 << 42, 1 << 43], [-5, -4, -3, -2]])
def test_offsets_that_are_wrong_are_reported(offsets):
    n, C = 10, 40
    x, b = torch.randn(n, C, device="cuda"), torch.randn(n, C, device="cuda")
    gate, off = torch.ones(3, C, device="cuda"), torch.tensor(offsets, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out_res, out, stats = torch.empty_like(x), torch.empty_like(x), torch.zeros(n, 4, device="cuda")
    tb.residual_norm(n, C, x, C, b, C, LAYER, 0, None, 3, off, gate, 1.0, None, None, EPS, out_res, C, out, C, stats, status)
    assert int(status) == tb.ERROR_CODES["INVALID_ARG"]
    status.zero_()
    ws = torch.zeros(tb.residual_norm_grad_workspace(n, C, 3), dtype=torch.uint8, device="cuda")
    tb.residual_norm_grad(n, C, x, C, b, C, LAYER, 0, None, 3, off, gate, 1.0, None, stats, out_res, C, out, C, torch.empty_like(x), C, torch.empty_like(x), C,
                          grad_gate=torch.empty_like(gate), workspace=ws, status=status)
    assert int(status) == tb.ERROR_CODES["INVALID_ARG"]


def test_no_rows():
    gate, ga = torch.full((2, 8), 5.0, device="cuda"), torch.full((8,), 5.0, device="cuda")
    off = torch.zeros(3, dtype=torch.int64, device="cuda")
    e = torch.empty(0, 8, device="cuda")
    tb.residual_norm(0, 8, e, 8, e, 8, LAYER, 1, None, 2, off, gate, 1.0, ga, None, EPS, e, 8, e, 8)
    dgate, dga = torch.full_like(gate, 3.0), torch.full_like(ga, 3.0)
    tb.residual_norm_grad(0, 8, e, 8, e, 8, LAYER, 1, None, 2, off, gate, 1.0, ga, None, e, 8, e, 8, e, 8, e, 8, grad_gate=dgate, grad_gamma=dga)
    assert (dgate == 0).all() and (dga == 0).all()


def test_gradients_against_differences():
    c = Case([2, 3], 16, F32, F32)
    stats, sums = torch.empty(c.n, 4, device="cuda"), c.sums()
    out_res, out, d_res, d_block = torch.empty_like(c.res), torch.empty_like(c.block), torch.empty_like(c.res), torch.empty_like(c.block)
    c.forward(out_res, out, stats)
    c.backward(stats, d_res, d_block, sums)

    def loss():
        c.forward(out_res, out)
        return float((out_res * c.dres).double().sum() + (out * c.dy).double().sum())

    # step 2^-8: the second differences' error is step^2 / 6 times a third derivative (below 100: 2.5e-4), rounding 4e-5 / step = 1e-2 (80 terms of up to 5, off by 2^-22 each)
    for x, dx, at in ((c.res, d_res, (1, 3)), (c.block, d_block, (4, 15)), (c.block, d_block, (0, 0)), (c.gate, sums["grad_gate"], (1, 2)), (c.gate, sums["grad_gate"], (0, 7)),
                      (c.gamma, sums["grad_gamma"], (5,)), (c.beta, sums["grad_beta"], (6,)), (c.post_gamma, sums["grad_post_gamma"], (9,))):
        kept, step = float(x[at]), 2.0 ** -8
        x[at] = kept + step
        up, high = loss(), float(x[at])
        x[at] = kept - step
        down, low = loss(), float(x[at])
        x[at] = kept
        assert abs((up - down) / (high - low) - float(dx[at])) < 2e-2, (at, dx[at])


def test_captured_and_replayed_on_new_rows():
    c = Case([30, 700, 2], 192, BF16, F32)
    stats, sums, ws = torch.empty(c.n, 4, device="cuda"), c.sums(), c.space()
    out_res, out, d_res, d_block = torch.empty_like(c.res), torch.empty_like(c.block), torch.empty_like(c.res), torch.empty_like(c.block)

    def both(stream=None):
        c.forward(out_res, out, stats, stream=stream)
        c.backward(stats, d_res, d_block, sums, stream=stream, workspace=ws)

    both()
    torch.cuda.synchronize()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=stream):
        both(stream)
    for x in (c.res, c.block, c.dres, c.dy):
        x.copy_(torch.randn(c.n, c.C, device="cuda"))
    ws.fill_(0x7F)
    graph.replay()
    torch.cuda.synchronize()
    ref = c.reference()
    for got, name in ((out_res, "res"), (out, "out"), (d_res, "dres"), (d_block, "dblock"), (sums["grad_gate"], "gate"), (sums["grad_gamma"], "gamma"), (sums["grad_post_gamma"], "post_gamma")):
        close(got, *ref[name])
    kept = {k: v.clone() for k, v in sums.items()}
    both()                                              # and once more: the same bits
    assert all(torch.equal(kept[k], sums[k]) for k in sums)


def test_rows_beyond_32_bits():
    n, C, ld = 4, 40, 1 << 30
    stores = [torch.empty(3 * ld + C, dtype=BF16, device="cuda") for _ in range(2)]
    res, block = (torch.as_strided(s, (n, C), (ld, 1)) for s in stores)
    for x in (res, block):
        x.copy_(torch.randn(n, C, device="cuda"))
    want = reference(res, block, True, True, None, None, 0, None, 1.0, None, None, EPS)
    tb.residual_norm(n, C, res, ld, block, ld, LAYER, 1, None, 0, None, None, 1.0, None, None, EPS, res, ld, block, ld)
    close(res, *want["res"])
    close(block, *want["out"])


def test_many_rows_and_groups():
    """More teams than one pass of the grid, groups of every length, a sum over all rows."""
    torch.manual_seed(3)
    sizes = torch.randint(0, 60, (9000,)).tolist() + [100_000, 0, 1]
    c = Case(sizes, 64, F32, F32)
    stats, sums = torch.empty(c.n, 4, device="cuda"), c.sums()
    out_res, out, d_res, d_block = torch.empty_like(c.res), torch.empty_like(c.block), torch.empty_like(c.res), torch.empty_like(c.block)
    c.forward(out_res, out, stats)
    c.backward(stats, d_res, d_block, sums)
    ref = c.reference()
    for got, name in ((out, "out"), (d_res, "dres"), (d_block, "dblock"), (sums["grad_gate"], "gate"), (sums["grad_gamma"], "gamma"), (sums["grad_beta"], "beta"), (sums["grad_post_gamma"], "post_gamma")):
        close(got, *ref[name])
