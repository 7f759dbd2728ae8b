"""Class log probabilities of many short rows (tiles of rows, 1 to 16 threads to a row): widths at both sides of each rule, rows without gaps, apart, off the alignment, masked, tied, in place."""
import math

import pytest
import torch

import paper_2607_17374_b200 as tb
from logprob_reference import near, reference, top_of
from rows_reference import close
from test_gpu_logprob import Call, rows, some_labels

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
N = 4100                                               # rows enough for tiles, the last of which is not full
WIDTHS = [1, 2, 3, 8, 16, 31, 47, 64, 65, 100, 127, 128, 129, 172, 255, 256, 257, 300, 384, 385, 511, 512, 513, 640, 768, 769, 1000, 1023, 1024]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("C", WIDTHS)
@pytest.mark.parametrize("pad,shift", [(0, 0), (8, 0), (3, 1), (0, 1), (2, 2)])
def test_forward_and_gradient(dtype, C, pad, shift):
    """pad 8: rows apart, on the alignment where C is; 3, 1: off it; 2, 2: 16-bit rows at even elements, but not at multiples of 16 bytes."""
    x, _ = rows(N, C, C + pad, dtype, shift, seed=C)
    labels = some_labels(N, C)
    Call(x, labels, 0).check(x, labels, 0)
    gen = torch.Generator("cuda").manual_seed(5)
    g, h = torch.randn(N, generator=gen, device="cuda"), torch.randn(N, generator=gen, device="cuda") * 0.3
    ref = reference(x, labels, g, h)
    fwd = Call(x, labels)
    for one_call in (True, False):
        dx, store = rows(N, C, C + pad, dtype, shift)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        if one_call:
            lp, H, st = torch.empty(N, device="cuda"), torch.empty(N, device="cuda"), torch.empty(N, 2, device="cuda")
            tb.class_logprob_train(N, C, x, C + pad, labels, g, h, lp, H, st, dx, C + pad, None, status)
            near(lp, ref["logprob"], ref["elp"])
            near(H, ref["H"], ref["eH"])
        else:
            tb.class_logprob_grad(N, C, x, C + pad, labels, fwd.stats, fwd.entropy, g, h, dx, C + pad, status)
        close(dx, ref["dx"], ref["edx"])
        inside = torch.zeros_like(store, dtype=torch.bool)
        torch.as_strided(inside, (N, C), (C + pad, 1), shift).fill_(True)
        assert (store[~inside] == 7).all() and int(status) == 0


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("C", WIDTHS)
@pytest.mark.parametrize("k", [1, 4, 5, 8, 9, 16])
def test_top(dtype, C, k):
    x, _ = rows(N, C, C, dtype, 0, seed=C + k)
    labels = some_labels(N, C)
    Call(x, labels, k).check(x, labels, k)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("C", [5, 47, 128, 200, 300, 600, 1000])
@pytest.mark.parametrize("kind", ["masks", "constant", "rising", "falling", "few values", "zeros of both signs", "lowest"])
def test_masks_orders_and_ties(dtype, C, kind):
    j = torch.arange(C, device="cuda", dtype=torch.float32)
    labels = some_labels(N, C)
    if kind == "masks":
        x, _ = rows(N, C, C, dtype, seed=9)
        gen = torch.Generator("cuda").manual_seed(4)
        hide = torch.rand(N, C, generator=gen, device="cuda") < 0.5
        x[0::4] = torch.where(hide[0::4], -math.inf, x[0::4])
        x[1::4] = torch.where(hide[1::4], torch.finfo(dtype).min, x[1::4])
        x[2::4, 1:] = -math.inf
        x[3::4] = -math.inf
        g, h = torch.randn(N, device="cuda"), torch.randn(N, device="cuda")
        ref = reference(x, labels, g, h)
        y = x.clone()                                  # in place
        tb.class_logprob_train(N, C, y, C, labels, g, h, None, None, None, y, C)
        close(y, ref["dx"], ref["edx"])
        assert (y[3::4] == 0).all() and (y[x == -math.inf] == 0).all()
    else:
        row = {"constant": torch.full_like(j, 1.5), "rising": j / 64, "falling": -j / 64, "few values": (j * 7919) % 5, "zeros of both signs": torch.where(j % 3 == 1, -0.0, 0.0),
               "lowest": torch.full_like(j, torch.finfo(dtype).min)}[kind]
        x = row.to(dtype).expand(N, C).contiguous()
    for k in (1, 6, 16):
        Call(x, labels, k).check(x, labels, k)


@pytest.mark.parametrize("C", [20, 150, 300, 1000])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_rows_that_hold_no_numbers(C, dtype, value):
    x, _ = rows(N, C, C, dtype)
    bad = torch.tensor([0, 1, 31, 32, 130, N - 1], device="cuda")
    for i, r in enumerate(bad.tolist()):
        x[r, (i * 7919) % C] = value
    labels = torch.zeros(N, dtype=torch.int64, device="cuda")
    c = Call(x, labels, 5)
    good = torch.ones(N, dtype=torch.bool, device="cuda")
    good[bad] = False
    assert torch.isnan(c.logprob[bad]).all() and torch.isnan(c.entropy[bad]).all() and torch.isnan(c.stats[bad]).all() and torch.isnan(c.top_logprob[bad]).all()
    assert torch.equal(c.top_class, top_of(x, 5))
    ref = reference(x[good], labels[good])
    near(c.logprob[good], ref["logprob"], ref["elp"])
    near(c.entropy[good], ref["H"], ref["eH"])


def test_labels_outside_the_classes_are_reported():
    for C in (30, 400):
        x, _ = rows(N, C, C, F32)
        labels = torch.full((N,), C, device="cuda")
        labels[::2] = C - 1
        status, lp = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.full((N,), 5.0, device="cuda")
        tb.class_logprob(N, C, x, C, labels, lp, status=status)
        assert int(status) == tb.ERROR_CODES["INVALID_ARG"] and (lp[1::2] == 0).all() and (lp[::2] < 0).all()
