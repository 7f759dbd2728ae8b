"""Class log probabilities of rows of few classes in tiles, which take two million elements (as many as a top of less): every width of one and two threads to a row, its order, masks and ties."""
import math

import pytest
import torch

import paper_2607_17374_b200 as tb
from logprob_reference import near, reference, top_of
from rows_reference import close
from test_gpu_logprob import Call, rows, some_labels

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
WIDTHS = [1, 2, 3, 5, 7, 8, 9, 16, 31, 32, 33, 47, 64, 65, 80, 81, 96, 100, 127, 128, 129, 160, 161, 172, 191, 192, 193, 255, 256, 257, 300, 384, 385, 511, 512]


def rows_of(C):
    return max(4100, (1 << 21) // C + 37)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("C", WIDTHS)
@pytest.mark.parametrize("pad,shift", [(0, 0), (8, 0), (3, 1), (2, 2)])
def test_forward_and_gradient(dtype, C, pad, shift):
    N = rows_of(C)
    x, _ = rows(N, C, C + pad, dtype, shift, seed=C)
    labels = some_labels(N, C)
    Call(x, labels, 0).check(x, labels, 0)
    gen = torch.Generator("cuda").manual_seed(5)
    g, h = torch.randn(N, generator=gen, device="cuda"), torch.randn(N, generator=gen, device="cuda") * 0.3
    ref = reference(x, labels, g, h)
    fwd = Call(x, labels)
    for one_call in (True, False):
        dx, store = rows(N, C, C + pad, dtype, shift)
        if one_call:
            lp, H, st = torch.empty(N, device="cuda"), torch.empty(N, device="cuda"), torch.empty(N, 2, device="cuda")
            tb.class_logprob_train(N, C, x, C + pad, labels, g, h, lp, H, st, dx, C + pad)
            near(lp, ref["logprob"], ref["elp"])
            near(H, ref["H"], ref["eH"])
        else:
            tb.class_logprob_grad(N, C, x, C + pad, labels, fwd.stats, fwd.entropy, g, h, dx, C + pad)
        close(dx, ref["dx"], ref["edx"])
        inside = torch.zeros_like(store, dtype=torch.bool)
        torch.as_strided(inside, (N, C), (C + pad, 1), shift).fill_(True)
        assert (store[~inside] == 7).all()


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("C", WIDTHS)
@pytest.mark.parametrize("k", [1, 3, 4, 5, 8, 9, 13, 16])
def test_top(dtype, C, k):
    N = rows_of(C)
    x, _ = rows(N, C, C, dtype, 0, seed=C + k)
    labels = some_labels(N, C)
    Call(x, labels, k).check(x, labels, k)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("C", [2, 3, 20, 47, 90, 171, 172, 301, 512])
@pytest.mark.parametrize("k", [2, 6, 16])
@pytest.mark.parametrize("pad,shift", [(0, 1), (3, 1), (8, 0)])
def test_top_of_rows_off_the_alignment(dtype, C, k, pad, shift):
    N = rows_of(C)
    x, _ = rows(N, C, C + pad, dtype, shift, seed=C + k)
    x[::3] = (x[::3] * 2).round() / 2                  # some rows with ties, the first and the last class among them
    x[::3, 0] = x[::3, -1] = 3
    labels = some_labels(N, C)
    Call(x, labels, k).check(x, labels, k)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("C", [5, 47, 90, 128, 150, 172, 300, 500])
@pytest.mark.parametrize("kind", ["masks", "few are left", "constant", "falling", "few values", "lowest"])
def test_masks_orders_and_ties(dtype, C, kind):
    N = rows_of(C)
    j = torch.arange(C, device="cuda", dtype=torch.float32)
    labels = some_labels(N, C)
    gen = torch.Generator("cuda").manual_seed(4)
    if kind == "masks":
        x, _ = rows(N, C, C, dtype, seed=9)
        hide = torch.rand(N, C, generator=gen, device="cuda") < 0.5
        x[0::4] = torch.where(hide[0::4], -math.inf, x[0::4])
        x[1::4] = torch.where(hide[1::4], torch.finfo(dtype).min, x[1::4])
        x[2::4, 1:] = -math.inf
        x[3::4] = -math.inf
        g, h = torch.randn(N, generator=gen, device="cuda"), torch.randn(N, generator=gen, device="cuda")
        ref = reference(x, labels, g, h)
        y = x.clone()                                  # in place
        tb.class_logprob_train(N, C, y, C, labels, g, h, None, None, None, y, C)
        close(y, ref["dx"], ref["edx"])
        assert (y[3::4] == 0).all() and (y[x == -math.inf] == 0).all()
    elif kind == "few are left":                       # fewer than the top asks for, and all of them one thread's
        x, _ = rows(N, C, C, dtype, seed=9)
        x[:, torch.arange(C, device="cuda") % 16 != 3] = -math.inf
    else:
        row = {"constant": torch.full_like(j, 1.5), "falling": -j / 64, "few values": (j * 7919) % 5, "lowest": torch.full_like(j, torch.finfo(dtype).min)}[kind]
        x = row.to(dtype).expand(N, C).contiguous()
    for k in (1, 4, 6, 16):
        Call(x, labels, k).check(x, labels, k)


@pytest.mark.parametrize("C", [20, 150, 300])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("value", [math.nan, math.inf])
@pytest.mark.parametrize("k", [3, 8, 16])
def test_rows_that_hold_no_numbers(C, dtype, value, k):
    N = rows_of(C)
    x, _ = rows(N, C, C, dtype)
    bad = torch.tensor([0, 1, 31, 32, 130, N - 1], device="cuda")
    for i, r in enumerate(bad.tolist()):
        x[r, (i * 7919) % C] = value
    labels = torch.zeros(N, dtype=torch.int64, device="cuda")
    c = Call(x, labels, k)
    good = torch.ones(N, dtype=torch.bool, device="cuda")
    good[bad] = False
    assert torch.isnan(c.logprob[bad]).all() and torch.isnan(c.entropy[bad]).all() and torch.isnan(c.stats[bad]).all()
    assert torch.equal(c.top_class, top_of(x, k))
    ref = reference(x[good], labels[good])
    near(c.logprob[good], ref["logprob"], ref["elp"])
    near(c.entropy[good], ref["H"], ref["eH"])


def test_labels_outside_the_classes_are_reported():
    for C in (30, 130):
        N = rows_of(C)
        x, _ = rows(N, C, C, F32)
        labels = torch.full((N,), C, device="cuda")
        labels[::2] = C - 1
        status, lp = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.full((N,), 5.0, device="cuda")
        tb.class_logprob(N, C, x, C, labels, lp, status=status)
        assert int(status) == tb.ERROR_CODES["INVALID_ARG"] and (lp[1::2] == 0).all() and (lp[::2] < 0).all()
