"""Class log probabilities, entropy, top alternatives and gradients against fp64: sizes at both sides of each kernel's range, pitches, masks, ties, values that are no numbers."""
import math

import pytest
import torch

import paper_2607_17374_b200 as tb
from logprob_reference import near, reference, top_of
from rows_reference import close

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def rows(n, C, ld, dtype, shift=0, seed=1, scale=2.0):
    """n rows of logits, ld apart, `shift` elements behind an aligned address, and the storage around them (7 in the gaps)."""
    store = torch.full((shift + max(n, 1) * ld + 8,), 7.0, dtype=dtype, device="cuda")
    x = torch.as_strided(store, (n, C), (ld, 1), shift)
    g = torch.Generator("cuda").manual_seed(seed)
    x.copy_(torch.randn(n, C, generator=g, device="cuda") * scale)
    return x, store


def some_labels(n, C, seed=2):
    g = torch.Generator("cuda").manual_seed(seed)
    labels = torch.randint(0, C, (n,), generator=g, device="cuda")
    labels[torch.rand(n, generator=g, device="cuda") < 0.2] = -1
    return labels


class Call:
    """Outputs of one call, with what no call may have left alone in them."""

    def __init__(self, x, labels, k=0, **st):
        n, C = x.shape
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.logprob, self.entropy = (torch.full((n,), 55.0, device="cuda") for _ in range(2))
        self.stats = torch.full((n, 2), 55.0, device="cuda")
        self.top_logprob, self.top_class = torch.full((n, k), 55.0, device="cuda"), torch.full((n, k), 55, dtype=torch.int64, device="cuda")
        size = tb.class_logprob_workspace(n, C, k)
        self.workspace = torch.full((size,), 0xC3, dtype=torch.uint8, device="cuda") if size else None
        tb.class_logprob(n, C, x, x.stride(0), labels, self.logprob if labels is not None else None, self.entropy, self.stats, k, self.top_logprob if k else None,
                         self.top_class if k else None, self.workspace, self.status, **st)

    def check(self, x, labels, k=0):
        ref = reference(x, labels)
        near(self.logprob, ref["logprob"], ref["elp"])
        near(self.entropy, ref["H"], ref["eH"])
        assert torch.equal(self.stats[:, 0].double(), ref["m"])
        near(self.stats[:, 1], ref["l"], ref["el"])
        if k:
            order = top_of(x, k)
            assert torch.equal(self.top_class, order)
            at = order.clamp(min=0)
            near(self.top_logprob, torch.where(order < 0, -math.inf, ref["lp"].gather(1, at)),
                 ref["el"][:, None] + 2 * 2.0 ** -24 * torch.nan_to_num(ref["lp"].gather(1, at), neginf=0.0).abs() + 2 * 2.0 ** -24 * ref["l"][:, None])
        assert int(self.status) == 0


SIZES = [(1, 1, 1, 0), (5, 2, 2, 0), (200, 3, 3, 1), (129, 47, 47, 0), (300, 47, 50, 0), (131, 64, 64, 0), (64, 64, 72, 0), (127, 100, 100, 3), (130, 128, 128, 0), (130, 129, 129, 0), (77, 172, 172, 0),
         (140, 255, 256, 0), (140, 256, 256, 0), (33, 257, 257, 0), (3, 511, 511, 5), (2500, 513, 513, 0), (9, 1000, 1024, 0), (7, 4097, 4097, 1), (2, 16_383, 16_383, 0), (3, 16_385, 16_385, 0),
         (1, 40_001, 40_001, 2), (600, 20_000, 20_000, 0), (2, 250_000, 250_000, 0)]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("n,C,ld,shift", SIZES)
@pytest.mark.parametrize("k", [0, 3, 10, 16])
def test_forward(dtype, n, C, ld, shift, k):
    x, _ = rows(n, C, ld, dtype, shift, seed=C + n)
    labels = some_labels(n, C)
    Call(x, labels, k).check(x, labels, k)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("n,C,ld,shift", SIZES)
def test_gradients_of_one_call_and_of_two(dtype, n, C, ld, shift):
    x, _ = rows(n, C, ld, dtype, shift, seed=C + n)
    labels = some_labels(n, C)
    gen = torch.Generator("cuda").manual_seed(5)
    g, h = torch.randn(n, generator=gen, device="cuda"), torch.randn(n, generator=gen, device="cuda") * 0.3
    fwd = Call(x, labels)
    for gg, hh in ((g, h), (g, None), (None, h)):
        ref = reference(x, labels, gg, hh)
        for one_call in (True, False):
            dx, store = rows(n, C, ld + 3, dtype, shift)
            status = torch.zeros(1, dtype=torch.int32, device="cuda")
            if one_call:
                lp, H, st = torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty(n, 2, device="cuda")
                size = tb.class_logprob_workspace(n, C)
                ws = torch.full((size,), 0xC3, dtype=torch.uint8, device="cuda") if size else None
                tb.class_logprob_train(n, C, x, ld, labels, gg, hh, lp, H, st, dx, ld + 3, ws, status)
                near(lp, ref["logprob"], ref["elp"])
                near(H, ref["H"], ref["eH"])
                near(st[:, 1], ref["l"], ref["el"])
            else:
                tb.class_logprob_grad(n, C, x, ld, labels, fwd.stats, fwd.entropy if hh is not None else None, gg, hh, dx, ld + 3, status)
            close(dx, ref["dx"], ref["edx"])
            inside = torch.zeros_like(store, dtype=torch.bool)
            torch.as_strided(inside, (n, C), (ld + 3, 1), shift).fill_(True)
            assert (store[~inside] == 7).all() and int(status) == 0


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,C", [(200, 47), (50, 300), (3, 20_000), (2400, 600)])
def test_gradient_in_place_and_optional_outputs(dtype, n, C):
    x, _ = rows(n, C, C, dtype)
    labels = some_labels(n, C)
    g = torch.randn(n, device="cuda")
    ref = reference(x, labels, g, None)
    size = tb.class_logprob_workspace(n, C)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda") if size else None
    lp, stats = torch.empty(n, device="cuda"), torch.empty(n, 2, device="cuda")
    y = x.clone()
    tb.class_logprob_train(n, C, y, C, labels, g, None, lp, None, None, y, C, ws)          # nothing but log probabilities beside it
    close(y, ref["dx"], ref["edx"])
    near(lp, ref["logprob"], ref["elp"])
    y = x.clone()
    tb.class_logprob(n, C, y, C, None, None, None, stats, workspace=ws)
    near(stats[:, 1], ref["l"], ref["el"])
    tb.class_logprob_grad(n, C, y, C, labels, stats, None, g, None, y, C)
    close(y, ref["dx"], ref["edx"])
    ids = torch.empty(n, 2, dtype=torch.int64, device="cuda")
    size = tb.class_logprob_workspace(n, C, 2)
    tb.class_logprob(n, C, x, C, k=2, top_class=ids, workspace=torch.empty(size, dtype=torch.uint8, device="cuda") if size else None)
    assert torch.equal(ids, top_of(x, 2))


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("n,C", [(40, 5), (130, 100), (40, 700), (2400, 600), (4, 33_000)])
def test_masks(dtype, n, C):
    """-inf and a type's lowest value in masked places, rows with one class left and with none."""
    x, _ = rows(n, C, C, dtype, seed=9)
    gen = torch.Generator("cuda").manual_seed(4)
    hide = torch.rand(n, C, generator=gen, device="cuda") < 0.5
    x[0::4] = torch.where(hide[0::4], -math.inf, x[0::4])
    x[1::4] = torch.where(hide[1::4], torch.finfo(dtype).min, x[1::4])
    x[2::4, 1:] = -math.inf
    x[3::4] = -math.inf
    labels = some_labels(n, C)
    labels[3] = C - 1
    Call(x, labels, 16).check(x, labels, 16)
    g, h = torch.randn(n, device="cuda"), torch.randn(n, device="cuda")
    ref = reference(x, labels, g, h)
    fwd = Call(x, labels)
    for one_call in (True, False):
        dx = torch.full_like(x, 9.0)
        if one_call:
            size = tb.class_logprob_workspace(n, C)
            tb.class_logprob_train(n, C, x, C, labels, g, h, None, None, None, dx, C, torch.empty(size, dtype=torch.uint8, device="cuda") if size else None)
        else:
            tb.class_logprob_grad(n, C, x, C, labels, fwd.stats, fwd.entropy, g, h, dx, C)
        close(dx, ref["dx"], ref["edx"])
        assert (dx[3::4] == 0).all() and (dx[x == -math.inf] == 0).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,C", [(33, 60), (33, 2000), (2400, 600), (2, 40_000)])
@pytest.mark.parametrize("kind", ["constant", "rising", "falling", "few values", "zeros of both signs", "lowest"])
def test_orders_and_ties(dtype, n, C, kind):
    j = torch.arange(C, device="cuda", dtype=torch.float32)
    row = {"constant": torch.full_like(j, 1.5), "rising": j / 64, "falling": -j / 64, "few values": (j * 7919) % 5, "zeros of both signs": torch.where(j % 3 == 1, -0.0, 0.0),
           "lowest": torch.full_like(j, torch.finfo(dtype).min)}[kind]
    x = row.to(dtype).expand(n, C).contiguous()
    labels = some_labels(n, C)
    for k in (1, 4, 16):
        Call(x, labels, k).check(x, labels, k)


@pytest.mark.parametrize("n,C", [(8, 50), (8, 900), (2400, 600), (8, 20_000)])
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_rows_that_hold_no_numbers(n, C, value):
    x, _ = rows(n, C, C, F32)
    at = [0, C // 2, C - 1, 7]
    for i, c in enumerate(at):
        x[i, c] = value
    x[4] = math.nan
    labels = torch.zeros(n, dtype=torch.int64, device="cuda")
    c = Call(x, labels, 5)
    assert torch.isnan(c.logprob[:5]).all() and torch.isnan(c.entropy[:5]).all() and torch.isnan(c.stats[:5]).all()
    assert torch.equal(c.top_class, top_of(x, 5)) and torch.isnan(c.top_logprob[:4]).all()
    ref = reference(x[5:], labels[5:])
    near(c.logprob[5:], ref["logprob"], ref["elp"])
    dx = torch.zeros_like(x)
    tb.class_logprob_grad(n, C, x, C, labels, c.stats, None, torch.ones(n, device="cuda"), None, dx, C)
    assert torch.isnan(dx[:5]).all() and torch.isfinite(dx[5:]).all()


def test_a_class_that_has_nearly_everything():
    """What is left for the others keeps its digits: entropy, 1 - p and the logarithm of the sum."""
    for C in (10, 300, 20_000):
        x = torch.zeros(4, C, device="cuda")
        x[:, 3] = torch.tensor([8.0, 14.0, 20.0, 40.0], device="cuda") + math.log(C)
        labels = torch.full((4,), 3, device="cuda")
        c = Call(x, labels, 1)
        ref = reference(x, labels, torch.ones(4, device="cuda"), None)
        for out, r in ((c.logprob, ref["logprob"]), (c.entropy, ref["H"]), (c.stats[:, 1], ref["l"])):
            assert ((out.double() - r).abs() <= 1e-4 * r.abs()).all(), (C, out, r)      # argument of up to 50: 2.5 x 50 u = 7.5e-6, sums of 8 200 terms 5e-4 of u
        dx = torch.empty_like(x)
        tb.class_logprob_grad(4, C, x, C, labels, c.stats, None, torch.ones(4, device="cuda"), None, dx, C)
        assert ((dx[:, 3].double() - ref["dx"][:, 3]).abs() <= 1e-4 * ref["dx"][:, 3].abs()).all()


def test_labels_outside_the_classes_are_reported():
    for C in (20, 2000):
        x, _ = rows(6, C, C, F32)
        labels = torch.tensor([0, -1, C, -2, 1 << 40, C - 1], device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        lp = torch.empty(6, device="cuda")
        stats = torch.empty(6, 2, device="cuda")
        tb.class_logprob(6, C, x, C, labels, lp, None, stats, status=status)
        assert int(status) == tb.ERROR_CODES["INVALID_ARG"] and (lp[1:5] == 0).all()
        status.zero_()
        good = torch.where((labels >= 0) & (labels < C), labels, -1)
        dx, want = torch.empty_like(x), torch.empty_like(x)
        g = torch.ones(6, device="cuda")
        tb.class_logprob_grad(6, C, x, C, labels, stats, None, g, None, dx, C, status)
        assert int(status) == tb.ERROR_CODES["INVALID_ARG"]
        tb.class_logprob_grad(6, C, x, C, good, stats, None, g, None, want, C)
        assert torch.equal(dx, want) and (dx[1:5] == 0).all()


def test_gradient_against_differences():
    x = torch.randn(3, 12, device="cuda")
    labels = torch.tensor([4, -1, 0], device="cuda")
    g, h = torch.tensor([1.0, 2.0, -0.5], device="cuda"), torch.tensor([0.3, -0.7, 0.1], device="cuda")

    def loss(x):
        c = Call(x, labels)
        return float((g * c.logprob).double().sum() + (h * c.entropy).double().sum())

    dx = torch.empty_like(x)
    tb.class_logprob_train(3, 12, x, 12, labels, g, h, None, None, None, dx, 12)
    step = 2.0 ** -6
    for i, j in ((0, 4), (0, 5), (1, 0), (2, 0), (2, 11)):
        e = torch.zeros_like(x)
        e[i, j] = step
        # third derivatives are below 2: step^2 / 3; each loss off by less than 1e-6
        assert abs((loss(x + e) - loss(x - e)) / (2 * step) - float(dx[i, j])) < 2 * step * step / 3 + 2e-6 / step


def test_rows_beyond_32_bits():
    n, C, ld = 4, 300, 1 << 30
    store = torch.empty(3 * ld + C, dtype=BF16, device="cuda")
    x = torch.as_strided(store, (n, C), (ld, 1))
    x.copy_(torch.randn(n, C, device="cuda"))
    labels = some_labels(n, C)
    Call(x, labels, 4).check(x, labels, 4)
    y = torch.as_strided(store, (n, 40), (ld, 1))
    Call(y, labels % 40, 4).check(y, labels % 40, 4)
    g = torch.ones(n, device="cuda")
    ref = reference(x, labels, g, None)
    tb.class_logprob_train(n, C, x, ld, labels, g, None, None, None, None, x, ld)
    close(x, ref["dx"], ref["edx"])


@pytest.mark.parametrize("n,C", [(100, 50), (5, 30_000)])
def test_captured_and_replayed_on_new_logits(n, C):
    x, _ = rows(n, C, C, BF16)
    labels = some_labels(n, C)
    g = torch.ones(n, device="cuda")
    out = [torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty(n, 2, device="cuda"), torch.empty_like(x)]
    size = tb.class_logprob_workspace(n, C)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda") if size else None

    def call(stream=None):
        tb.class_logprob_train(n, C, x, C, labels, g, None, *out[:3], out[3], C, ws, stream=stream)

    call()
    torch.cuda.synchronize()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=stream):
        call(stream)
    x.copy_(torch.randn(n, C, device="cuda"))
    for o in out:
        o.fill_(3.0)
    if ws is not None:
        ws.fill_(0xFF)
    graph.replay()
    torch.cuda.synchronize()
    got = [o.clone() for o in out]
    call()
    assert all(torch.equal(a, b) for a, b in zip(got, out))
    ref = reference(x, labels, g, None)
    near(got[0], ref["logprob"], ref["elp"])
    close(got[3], ref["dx"], ref["edx"])


def test_the_same_bits_on_another_stream_and_again():
    for n, C in ((1000, 47), (700, 5000), (2, 60_000)):
        x, _ = rows(n, C, C, F32)
        labels = some_labels(n, C)
        a = Call(x, labels, 7)
        torch.cuda.synchronize()
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            b = Call(x, labels, 7, stream=s)
        s.synchronize()
        for f in ("logprob", "entropy", "stats", "top_logprob", "top_class"):
            assert torch.equal(getattr(a, f), getattr(b, f))
