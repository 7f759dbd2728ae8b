"""Class log probabilities of 513 to 1 024 classes in tiles (4 to 16 threads to a row), with a top: rows off the alignment, of odd widths, with ties across the threads, masks and values that
are no numbers.  4 100 rows are two million elements there, enough for tiles with a top or without."""
import math

import pytest
import torch

from logprob_reference import near, reference, top_of
from test_gpu_logprob import Call, rows, some_labels

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
N = 4100
WIDTHS = [513, 600, 639, 640, 641, 768, 769, 1000, 1001, 1023, 1024]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("C", WIDTHS)
@pytest.mark.parametrize("k", [2, 6, 16])
@pytest.mark.parametrize("pad,shift", [(0, 0), (0, 1), (3, 1), (8, 0)])
def test_top_of_rows_off_the_alignment(dtype, C, k, pad, shift):
    x, _ = rows(N, C, C + pad, dtype, shift, seed=C + k)
    x[::3] = (x[::3] * 2).round() / 2                  # some rows with ties, the first and the last class among them
    x[::3, 0] = x[::3, -1] = 9
    labels = some_labels(N, C)
    labels[:4] = torch.tensor([0, C - 1, C - 2, 1], device="cuda")
    Call(x, labels, k).check(x, labels, k)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("C", [641, 1001, 1024])
@pytest.mark.parametrize("kind", ["masks", "few are left", "the first and the last are left", "constant", "few values"])
def test_masks_and_ties_off_the_alignment(dtype, C, kind):
    x, _ = rows(N, C, C + 3, dtype, 1, seed=9)
    gen = torch.Generator("cuda").manual_seed(4)
    if kind == "masks":
        hide = torch.rand(N, C, generator=gen, device="cuda") < 0.5
        x[0::4] = torch.where(hide[0::4], -math.inf, x[0::4])
        x[1::4] = torch.where(hide[1::4], torch.finfo(dtype).min, x[1::4])
        x[2::4, 1:] = -math.inf
        x[3::4] = -math.inf
    elif kind == "few are left":                       # fewer than the top asks for, and all of them one thread's
        x[:, torch.arange(C, device="cuda") % 16 != 3] = -math.inf
        x[::2, 40:] = -math.inf
    elif kind == "the first and the last are left":
        x[:, 1:-1] = -math.inf
    elif kind == "constant":
        x[:] = 1.5
    else:
        x[:] = ((torch.arange(C, device="cuda") * 7919) % 5).to(dtype)
    labels = some_labels(N, C)
    for k in (1, 4, 16):
        Call(x, labels, k).check(x, labels, k)


@pytest.mark.parametrize("C", [515, 1001])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_rows_that_hold_no_numbers(C, dtype, value):
    x, _ = rows(N, C, C, dtype, 1)
    bad = torch.tensor([0, 1, 2, 3, 31, 32, 130, N - 1], device="cuda")
    for r, at in zip(bad.tolist(), [0, C - 1, 0, C - 1, 7, 77, 300, 500]):
        x[r, at] = value
    labels = torch.zeros(N, dtype=torch.int64, device="cuda")
    for k in (3, 16):
        c = Call(x, labels, k)
        good = torch.ones(N, dtype=torch.bool, device="cuda")
        good[bad] = False
        assert torch.isnan(c.logprob[bad]).all() and torch.isnan(c.entropy[bad]).all() and torch.isnan(c.stats[bad]).all() and torch.isnan(c.top_logprob[bad]).all()
        assert torch.equal(c.top_class, top_of(x, k))
        ref = reference(x[good], labels[good])
        near(c.logprob[good], ref["logprob"], ref["elp"])
        near(c.entropy[good], ref["H"], ref["eH"])
