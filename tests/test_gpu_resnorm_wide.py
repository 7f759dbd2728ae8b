"""The residual norm of rows that a block has to itself, two at a time: groups of one row and of odd numbers of rows, rows of no group, many rows to a block."""
import pytest
import torch

import paper_2607_17374_b200 as tb
from rows_reference import close
from test_gpu_resnorm import LAYER, RMS, TYPES, Case, strided, untouched

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
SHAPES = [([1], 300), ([2], 300), ([3], 1024), ([1] * 1500, 272), ([-3, 1, 2, 3, 0, 5, 4000, 1, 1, 1, 9001, -2], 264), ([-1, 7001, 2, 5000, -1], 301), ([11, 13_000], 516), ([20_001], 1000), ([3] * 2500, 259)]


@pytest.mark.parametrize("t,r", TYPES)
@pytest.mark.parametrize("sizes,C", SHAPES)
@pytest.mark.parametrize("kind,post,gate", [(LAYER, True, True), (RMS, True, True), (LAYER, False, False)])
def test_forward(t, r, sizes, C, kind, post, gate):
    c = Case(sizes, C, t, r, kind, post, gate)
    (out_res, s1), (out, s2) = (strided(c.n, C, c.ld, x) for x in (r, t))
    stats = torch.full((c.n, 4), 7.0, device="cuda")
    c.forward(out_res, out, stats)
    ref = c.reference()
    rows = slice(c.lo, c.hi)
    close(out_res[rows], *ref["res"])
    close(out[rows], *ref["out"])
    for s in (s1, s2):
        untouched(s, c.n, C, c.ld, 0, (c.lo, c.hi))
    assert (stats[:c.lo] == 7).all() and (stats[c.hi:] == 7).all() and int(c.status) == 0
    a, b = c.res.clone(), c.block.clone()        # in place
    c.forward(a, b, None, res=a, block=b)
    assert torch.equal(a[rows], out_res[rows]) and torch.equal(b[rows], out[rows])
    d_res, d_block, sums = torch.empty_like(c.res), torch.empty_like(c.block), c.sums()
    c.backward(stats, d_res, d_block, sums)
    for got, name in ((d_res[rows], "dres"), (d_block[rows], "dblock"), (sums["grad_gamma"], "gamma"), (sums["grad_post_gamma"], "post_gamma"), (sums["grad_gate"], "gate")):
        if got is not None:
            close(got, *ref[name])


@pytest.mark.parametrize("t", [F32, BF16])
def test_without_a_block(t):
    for n in (1, 2, 5, 3001):
        x = torch.randn(n, 640, device="cuda").to(t)
        y = torch.empty_like(x)
        tb.residual_norm(n, 640, x, 640, None, 640, RMS, 0, None, 0, None, None, 1.0, None, None, 1e-5, None, 640, y, 640)
        want = x.double() * torch.rsqrt(x.double().square().mean(1, keepdim=True) + 1e-5)
        assert ((y.double() - want).abs() <= want.abs() * (torch.finfo(t).eps / 2 + 2.0 ** -20)).all()      # the sum of 640 squares in fp32: a few roundings of a thread's 8, 5 + 2 levels; the root


@pytest.mark.parametrize("offsets", [[0, 5, 3, 10], [-1, 4, 8, 10], [0, 4, 8, 11], [7, 2, 1, 0], [1 << 40, 1 << 41, 1 << 42, 1 << 43]])
def test_offsets_that_are_wrong_are_reported(offsets):
    n, C = 10, 400
    x, b = torch.randn(n, C, device="cuda"), torch.randn(n, C, device="cuda")
    gate, off = torch.ones(3, C, device="cuda"), torch.tensor(offsets, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out_res, out = torch.empty_like(x), torch.empty_like(x)
    tb.residual_norm(n, C, x, C, b, C, LAYER, 0, None, 3, off, gate, 1.0, None, None, 1e-5, out_res, C, out, C, None, status)
    assert int(status) == tb.ERROR_CODES["INVALID_ARG"]
