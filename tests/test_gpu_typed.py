"""Products by vertex type and their gradients against fp64: types, ragged and empty groups, odd widths, pitches, rows outside the groups."""
import pytest
import torch

import paper_2607_17374_b200 as tb
from rows_reference import U32, close, typed, typed_grad

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def strided(n, width, ld, dtype, shift=0):
    store = torch.full((shift + max(n, 1) * ld + 8,), 7.0, dtype=dtype, device="cuda")
    return torch.as_strided(store, (n, width), (ld, 1), shift), store


def workspace(size):
    return torch.full((size,), 255, dtype=torch.uint8, device="cuda") if size else None


def sums(m):
    """Bound on the relative error of a sum of m products: a step of a tensor core's sum may round toward zero, and there are no more
    steps than terms."""
    return (m + 4) * 2 * U32


# sizes of the groups; a list that begins or ends with a negative number leaves that many rows in front or behind
SHAPES = [
    ([1], 1, 1), ([5], 100, 256), ([0, 3, 0], 37, 130), ([-2, 1, 0, 2, 1, -3], 64, 64), ([130, 1, 127, 128, 129], 128, 128), ([300, 0, 41, 7], 33, 47),
    ([1000], 100, 256), ([257, 511], 512, 200), ([64] * 20, 16, 24), ([700, 90], 1000, 72), ([90, 333], 72, 1000), ([-5, 400, 200, -9], 96, 96), ([2] * 300, 40, 40),
    ([2600], 48, 264), ([5000, 3], 24, 16),
    ([300, 50, 0, 1], 46, 58), ([64], 50, 36), ([65], 36, 50), ([1500, 1030, 40], 66, 130),
    ([1, 2, 0] * 70, 260, 24), ([70, 65] * 40, 392, 120), ([9000], 136, 264),
]


def lay_out(sizes):
    front = -sizes[0] if sizes[0] < 0 else 0
    behind = -sizes[-1] if len(sizes) > 1 and sizes[-1] < 0 else 0
    groups = [s for s in sizes if s >= 0]
    off = [front]
    for s in groups:
        off.append(off[-1] + s)
    return off, off[-1] + behind


def make(sizes, K, N, t, seed=0, pad=0, shift=0):
    off, n = lay_out(sizes)
    g = torch.Generator("cuda").manual_seed(seed + K * 7 + N)
    x, xs = strided(n, K, K + pad, t, shift)
    x.copy_(torch.randn(n, K, generator=g, device="cuda"))
    W = torch.randn(len(off) - 1, K, N, generator=g, device="cuda").to(t)
    bias = torch.randn(len(off) - 1, N, generator=g, device="cuda")
    dy, _ = strided(n, N, N + pad, t, shift)
    dy.copy_(torch.randn(n, N, generator=g, device="cuda"))
    return off, n, x, W, bias, dy


def forward(off, n, x, W, bias, out, status=None, **kw):
    G, K, N = W.shape
    ws = workspace(tb.typed_project_workspace(n, G, K, N, x))
    tb.typed_project(n, G, torch.tensor(off, device="cuda"), x, x.stride(0), W, bias, K, N, out, out.stride(0), ws, status, **kw)


def backward(off, n, x, W, dy, dx, dW, db, status=None):
    G, K, N = W.shape
    ws = workspace(tb.typed_project_grad_workspace(n, G, K, N, dy))
    tb.typed_project_grad(n, G, torch.tensor(off, device="cuda"), x, x.stride(0), W, dy, dy.stride(0), K, N, dx, dx.stride(0) if dx is not None else 0, dW, db, ws, status)


@pytest.mark.parametrize("t,ot", [(F32, F32), (BF16, BF16), (BF16, F32), (F16, F16), (F16, F32)])
@pytest.mark.parametrize("sizes,K,N", SHAPES)
@pytest.mark.parametrize("pad,shift", [(0, 0), (8, 0), (3, 1)])
def test_project(t, ot, sizes, K, N, pad, shift):
    off, n, x, W, bias, _ = make(sizes, K, N, t, pad=pad, shift=shift)
    for b in (bias, None):
        out, store = strided(n, N, N + pad, ot, shift)
        before = store.clone()
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        forward(off, n, x, W, b, out, status)
        ref, mag = typed(off, x, W, b)
        lo, hi = off[0], off[-1]
        close(out[lo:hi], ref[lo:hi], mag[lo:hi] * sums(K))
        assert int(status) == 0
        torch.as_strided(before, (n, N), (N + pad, 1), shift)[lo:hi] = out[lo:hi]
        assert torch.equal(before, store)               # nothing else was written


@pytest.mark.parametrize("t,wt", [(F32, F32), (BF16, BF16), (BF16, F32), (F16, F16), (F16, F32)])
@pytest.mark.parametrize("sizes,K,N", SHAPES)
@pytest.mark.parametrize("pad,shift", [(0, 0), (8, 0), (3, 1)])
def test_gradients(t, wt, sizes, K, N, pad, shift):
    off, n, x, W, bias, dy = make(sizes, K, N, t, pad=pad, shift=shift)
    G = W.shape[0]
    dx, store = strided(n, K, K + pad, t, shift)
    before = store.clone()
    dW, db = torch.full((G, K, N), 9.0, dtype=wt, device="cuda"), torch.full((G, N), 9.0, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    backward(off, n, x, W, dy, dx, dW, db, status)
    (rx, mx), (rw, mw), (rb, mb) = typed_grad(off, x, W, dy)
    lo, hi = off[0], off[-1]
    most = max(b - a for a, b in zip(off, off[1:]))
    close(dx[lo:hi], rx[lo:hi], mx[lo:hi] * sums(N))
    close(dW, rw, mw * sums(most))
    close(db, rb, mb * sums(most))
    assert int(status) == 0
    torch.as_strided(before, (n, K), (K + pad, 1), shift)[lo:hi] = dx[lo:hi]
    assert torch.equal(before, store)
    again = [dx.clone(), dW.clone(), db.clone()]
    backward(off, n, x, W, dy, dx, dW, db)
    assert all(torch.equal(a, b) for a, b in zip(again, (dx, dW, db)))
    for which in range(3):                              # one at a time: the same bits
        alone = [torch.full_like(o, 5.0) if i == which else None for i, o in enumerate((dx, dW, db))]
        if which == 0:
            alone[0] = torch.as_strided(torch.zeros_like(store), (n, K), (K + pad, 1), shift)
        backward(off, n, x, W, dy, *alone)
        got, want = alone[which], again[which]
        assert torch.equal(got[lo:hi], want[lo:hi]) if which == 0 else torch.equal(got, want)


@pytest.mark.parametrize("t", [F32, BF16, F16])
def test_rows_outside_the_groups_may_hold_anything(t):
    """NaN and infinity in rows of no group and in the rows of one group reach no other group's results."""
    off, n = [3, 103, 103, 205, 400], 410
    g = torch.Generator("cuda").manual_seed(3)
    x = torch.randn(n, 72, generator=g, device="cuda").to(t)
    dy = torch.randn(n, 56, generator=g, device="cuda").to(t)
    W = torch.randn(4, 72, 56, generator=g, device="cuda").to(t)
    rows = torch.ones(n, dtype=torch.bool, device="cuda")
    rows[:3] = rows[400:] = rows[103:205] = False
    xn, dyn, Wn = x.clone(), dy.clone(), W.clone()
    xn[~rows], dyn[~rows] = float("nan"), float("inf")
    Wn[1], Wn[2] = float("nan"), float("inf")

    def results(x, dy, W):
        out, dx = torch.zeros(n, 56, dtype=t, device="cuda"), torch.zeros(n, 72, dtype=t, device="cuda")
        dW, db = torch.empty(4, 72, 56, device="cuda"), torch.empty(4, 56, device="cuda")
        forward(off, n, x, W, None, out)
        backward(off, n, x, W, dy, dx, dW, db)
        return out, dx, dW, db
    clean, foul = results(x, dy, W), results(xn, dyn, Wn)
    for a, b in zip(clean[:2], foul[:2]):
        assert torch.equal(a[rows], b[rows])
    for a, b in zip(clean[2:], foul[2:]):
        assert torch.equal(a[[0, 1, 3]], b[[0, 1, 3]])


@pytest.mark.parametrize("n", [3, 400])
@pytest.mark.parametrize("t", [F32, BF16])
def test_infinities_stay_infinities(t, n):
    """A row with an infinity gives infinities of the weights' signs, as the formula does.  40 times 1e37 is above fp32's largest value (3.4e38) and
    becomes infinity too; 40 times 8e36 is below it and stays finite."""
    x = torch.ones(n, 40, dtype=t, device="cuda")
    W = torch.ones(1, 40, 24, dtype=t, device="cuda")
    W[0, 7, 3] = -1.0
    x[1, 7] = float("inf")
    x[2] = 1e37
    out = torch.empty(n, 24, device="cuda")
    forward([0, n], n, x, W, None, out)
    want = x.double() @ W[0].double()
    assert torch.equal(out[:3], want[:3].float())
    x[2] = 8e36
    forward([0, n], n, x, W, None, out)
    want = x.double() @ W[0].double()
    assert torch.isfinite(out[2]).all() and ((out[2].double() - want[2]).abs() <= 40 * x[2, 0].double() * sums(40)).all()


@pytest.mark.parametrize("t", [F32, BF16])
@pytest.mark.parametrize("bad", [[0, 50, 40, 300], [-5, 50, 90, 300], [0, 50, 90, 301], [0, 1 << 40, 90, 300], [300, 200, 100, 0], [0, -(1 << 50), 90, 200]])
def test_bad_offsets_give_a_status(bad, t):
    """Offsets that run backwards or leave the rows: an error in the status word, nothing outside the arrays is touched."""
    n, K, N = 300, 40, 48
    x, dy, W = (torch.ones(s, dtype=t, device="cuda") for s in ((n, K), (n, N), (3, K, N)))
    out, os = strided(n, N, N, t)
    dx, xs = strided(n, K, K, t)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    forward(bad, n, x, W, None, out, status)
    assert int(status) == tb.ERROR_CODES["INVALID_ARG"]
    status.zero_()
    backward(bad, n, x, W, dy, dx, torch.empty(3, K, N, device="cuda"), torch.empty(3, N, device="cuda"), status)
    assert int(status) == tb.ERROR_CODES["INVALID_ARG"]
    assert (os[n * N:] == 7).all() and (xs[n * K:] == 7).all()


def test_gradients_against_differences():
    """The product is linear in x and in W: central differences of <r, out> against the gradients, up to the rounding of the sums."""
    sizes, K, N = [150, 0, 333], 60, 52
    off, n, x, W, bias, r = make(sizes, K, N, F32)
    g = torch.Generator("cuda").manual_seed(9)
    dX, dWd = torch.randn(n, K, generator=g, device="cuda"), torch.randn(3, K, N, generator=g, device="cuda")
    dx, dW, db = torch.empty(n, K, device="cuda"), torch.empty(3, K, N, device="cuda"), torch.empty(3, N, device="cuda")
    backward(off, n, x, W, r, dx, dW, db)

    def loss(x, W):
        out = torch.empty(n, N, device="cuda")
        forward(off, n, x, W, bias, out)
        return float((out.double() * r.double()).sum()), float((typed(off, x, W, bias)[1] * r.double().abs()).sum())
    for grad, d, plus, minus in ((dx, dX, (x + dX, W), (x - dX, W)), (dW, dWd, (x, W + dWd), (x, W - dWd))):
        (a, ma), (b, mb) = loss(*plus), loss(*minus)
        i = 0 if grad is dx else 1
        step = plus[i].double() - minus[i].double()
        assert abs((a - b) - float((grad.double() * step).sum())) <= (ma + mb) * (sums(K) + sums(N if grad is dx else 333))


@pytest.mark.parametrize("t", [F32, BF16, F16])
@pytest.mark.parametrize("K,N", [(40, 24), (33, 47)])
def test_weights_at_any_element(t, K, N):
    """Weights that begin at an odd element of their storage."""
    off, n, x, W, bias, dy = make([70, 0, 130], K, N, t)
    V = torch.empty(W.numel() + 1, dtype=t, device="cuda")[1:].view(W.shape)
    V.copy_(W)
    out, dx = torch.empty(n, N, device="cuda"), torch.empty(n, K, dtype=t, device="cuda")
    forward(off, n, x, V, bias, out)
    backward(off, n, x, V, dy, dx, None, None)
    ref, mag = typed(off, x, W, bias)
    close(out, ref, mag * sums(K))
    (rx, mx), _, _ = typed_grad(off, x, W, dy)
    close(dx, rx, mx * sums(N))


@pytest.mark.parametrize("n", [30, 300])
def test_what_is_not_asked_for_needs_no_arguments(n):
    """grad_bias alone: no x, no W, no pitches of either, no type of grad_W."""
    off, dy = torch.tensor([0, 10, n], device="cuda"), torch.randn(n, 24, device="cuda")
    db = torch.empty(2, 24, device="cuda")
    ws = workspace(tb.typed_project_grad_workspace(n, 2, 16, 24, dy))
    rc = tb.load_library().taurus_typed_project_grad(n, 2, off.data_ptr(), None, 0, tb.F32, None, dy.data_ptr(), 24, 16, 24, None, 0, None, -1, db.data_ptr(),
                                                     ws.data_ptr() if ws is not None else None, ws.numel() if ws is not None else 0, None, None)
    assert rc == 0
    ref, mag = torch.stack([dy[:10].double().sum(0), dy[10:].double().sum(0)]), torch.stack([dy[:10].double().abs().sum(0), dy[10:].double().abs().sum(0)])
    close(db, ref, mag * sums(n))


def test_without_rows():
    W = torch.ones(2, 8, 16, device="cuda")
    off = torch.zeros(3, dtype=torch.int64, device="cuda")
    dW, db = torch.ones(2, 8, 16, device="cuda"), torch.ones(2, 16, device="cuda")
    ws = workspace(tb.typed_project_grad_workspace(0, 2, 8, 16, torch.float32))
    tb.typed_project_grad(0, 2, off, None, 8, W, None, 16, 8, 16, None, 0, dW, db, ws, type=tb.F32)
    assert (dW == 0).all() and (db == 0).all()


def test_most_types_and_wide_rows():
    """1 024 types, most without rows; rows of 1 024 columns."""
    n = 500
    g = torch.Generator("cuda").manual_seed(1)
    ends = torch.sort(torch.randint(0, n + 1, (1023,), generator=g, device="cuda")).values
    off = [0] + ends.tolist() + [n]
    x = torch.randn(n, 40, generator=g, device="cuda").bfloat16()
    W = torch.randn(1024, 40, 24, generator=g, device="cuda").bfloat16()
    out = torch.empty(n, 24, device="cuda")
    forward(off, n, x, W, None, out)
    ref, mag = typed(off, x, W, None)
    close(out, ref, mag * sums(40))
    for t in (F32, BF16):
        off, n, x, W, bias, dy = make([400, 30], 1024, 1024, t)
        out, dx = torch.empty(n, 1024, device="cuda"), torch.empty(n, 1024, dtype=t, device="cuda")
        dW, db = torch.empty(2, 1024, 1024, device="cuda"), torch.empty(2, 1024, device="cuda")
        forward(off, n, x, W, bias, out)
        backward(off, n, x, W, dy, dx, dW, db)
        ref, mag = typed(off, x, W, bias)
        close(out, ref, mag * sums(1024))
        (rx, mx), (rw, mw), (rb, mb) = typed_grad(off, x, W, dy)
        close(dx, rx, mx * sums(1024)); close(dW, rw, mw * sums(400)); close(db, rb, mb * sums(400))


def test_fp32_products_keep_their_bits():
    """fp32 operands whose products cancel to their last bits: the error stays at fp32's own, also beside elements 1e6 times as large."""
    n, K, N = 2000, 256, 128
    g = torch.Generator("cuda").manual_seed(2)
    x = torch.randn(n, K, generator=g, device="cuda")
    x[:, 5] *= 1e6
    W = torch.randn(1, K, N, generator=g, device="cuda")
    W[0, 5] = 0
    out = torch.empty(n, N, device="cuda")
    forward([0, n], n, x, W, None, out)
    ref, mag = typed([0, n], x, W, None)
    assert float(((out.double() - ref).abs() / mag).max()) <= sums(K)
    assert float(((out.double() - ref) / mag).pow(2).mean().sqrt()) <= 16 * U32      # as a mean: nowhere near the bound of the sum


def test_refused_on_a_device():
    x, W, out = torch.zeros(4, 8, device="cuda"), torch.zeros(2, 8, 8, device="cuda"), torch.zeros(4, 8, device="cuda")
    off = torch.tensor([0, 2, 4], device="cuda")
    for bad in (dict(x=x.cpu()), dict(W=W.cpu()), dict(off=off.cpu()), dict(out=x), dict(out=W[0, :4]), dict(bias=torch.zeros(16))):
        a = dict(x=x, W=W, off=off, out=out, bias=None)
        a.update(bad)
        with pytest.raises(tb.TaurusError) as e:
            tb.typed_project(4, 2, a["off"], a["x"], 8, a["W"], a["bias"], 8, 8, a["out"], 8, workspace(1 << 20))
        assert e.value.code == tb.ERROR_CODES["INVALID_ARG"]
    dW, db = torch.zeros_like(W), torch.zeros(2, 8, device="cuda")
    for bad in (dict(dx=out), dict(dx=x), dict(dW=W), dict(db=out[:2]), dict(dW=dW.cpu())):
        a = dict(dx=torch.zeros(4, 8, device="cuda"), dW=dW, db=db)
        a.update(bad)
        with pytest.raises(tb.TaurusError) as e:
            tb.typed_project_grad(4, 2, off, x, 8, W, out, 8, 8, 8, a["dx"], 8, a["dW"], a["db"], workspace(1 << 20))
        assert e.value.code == tb.ERROR_CODES["INVALID_ARG"]


@pytest.mark.parametrize("t", [F32, BF16, F16])
@pytest.mark.parametrize("sizes,K,N", [([5000, 0, 65, 3], 136, 264), ([30, 10], 40, 24), ([2100] * 40, 37, 130)])
def test_each_gradient_alone_is_what_it_is_beside_the_others(t, sizes, K, N):
    off, n, x, W, bias, dy = make(sizes, K, N, t)
    new = lambda: (torch.full((n, K), 3.0, dtype=t, device="cuda"), torch.full((len(sizes), K, N), 3.0, device="cuda"), torch.full((len(sizes), N), 3.0, device="cuda"))
    together, alone = new(), new()
    backward(off, n, x, W, dy, *together)
    for i in range(3):
        backward(off, n, x, W, dy, *(a if i == j else None for j, a in enumerate(alone)))
    for a, b in zip(together, alone):
        assert torch.equal(a, b)


@pytest.mark.parametrize("t", [F32, BF16, F16])
@pytest.mark.parametrize("sizes,K,N", [([300, 0, 41, 7], 100, 36), ([1500, 1030, 40], 68, 132), ([70, 65] * 40, 392, 120)])
@pytest.mark.parametrize("pad,shift", [(0, 0), (4, 4)])
def test_offsets_at_any_element(t, sizes, K, N, pad, shift):
    """Offsets that begin at the second element of their storage, 8 bytes off 16: the bits that offsets of their own give, also where a stage of the rows is only partly there."""
    off, n, x, W, bias, dy = make(sizes, K, N, t, pad=pad, shift=shift)
    own = torch.tensor(off, device="cuda")
    slid = torch.tensor([-1] + off, device="cuda")[1:]
    assert own.data_ptr() % 16 == 0 and slid.data_ptr() % 16 == 8
    G, results = len(sizes), []
    for o in (own, slid):
        out, dx = torch.empty(n, N, dtype=t, device="cuda"), torch.empty(n, K, dtype=t, device="cuda")
        dW, db, alone = torch.empty(G, K, N, device="cuda"), torch.empty(G, N, device="cuda"), torch.empty(G, N, device="cuda")
        ws = workspace(tb.typed_project_grad_workspace(n, G, K, N, t))
        tb.typed_project(n, G, o, x, x.stride(0), W, bias, K, N, out, N, ws)
        tb.typed_project_grad(n, G, o, x, x.stride(0), W, dy, dy.stride(0), K, N, dx, K, dW, db, ws)
        tb.typed_project_grad(n, G, o, x, x.stride(0), W, dy, dy.stride(0), K, N, grad_bias=alone, workspace=ws)
        assert torch.equal(db, alone)
        results.append((out, dx, dW, db))
    assert all(torch.equal(a, b) for a, b in zip(*results))
    ref, mag = typed(off, x, W, bias)
    close(results[1][0], ref, mag * sums(K))


def test_a_single_product_is_as_exact_as_fp32():
    """Sums of one term.  What the split of the operands leaves out is below 2^-24 of a product; the five smaller products, together at most 2^-7 + 2^-16 of it, are added in steps
    that lose 2^-23 of their sum each (below 2^-26 in all), and the last addition rounds by 2^-24: 2.25 2^-24.  Operands in [1, 2), and such whose middle and last parts are largest."""
    n, N = 4096, 1024
    g = torch.Generator("cuda").manual_seed(12)
    bits = torch.randint(0, 1 << 23, (n + N,), generator=g, device="cuda", dtype=torch.int32)
    bits[n // 2:n + N // 2] &= 0xFFFF
    bits[:64] = bits[n:n + 64] = torch.arange(0xFFC0 - 64, 0xFFC0, device="cuda", dtype=torch.int32) | 0x7F0000
    bits[64:128] = bits[n + 64:n + 128] = torch.arange(0x7FC0, 0x8000, device="cuda", dtype=torch.int32)
    bits[128] = bits[n + 128] = 0xFF80
    v = (bits | 0x3F800000).view(F32)
    x, W = v[:n].view(n, 1).contiguous(), v[n:].view(1, 1, N).contiguous()
    out = torch.empty(n, N, device="cuda")
    forward([0, n], n, x, W, None, out)
    ref = x.double() * W[0].double()
    assert float(((out.double() - ref).abs() / ref).max()) <= 2.25 * U32
    dx, dy = torch.empty(n, 1, device="cuda"), torch.zeros(n, N, device="cuda")
    c = torch.arange(n, device="cuda") % N
    dy[torch.arange(n, device="cuda"), c] = x[:, 0]
    backward([0, n], n, x, W, dy, dx, None, None)
    ref = x.double() * W[0, 0, c].double()[:, None]
    assert float(((dx.double() - ref).abs() / ref).max()) <= 2.25 * U32
    dW, one = torch.empty(n // 128, 1, N, device="cuda"), torch.zeros(n, N, device="cuda")      # a row that is not zero to each type
    one[::128] = W[0, 0]
    backward(list(range(0, n + 1, 128)), n, x, torch.zeros(n // 128, 1, N, device="cuda"), one, None, dW, None)
    ref = x[::128, None].double() * W.double()
    assert float(((dW.double() - ref).abs() / ref).max()) <= 2.25 * U32


def test_largest_values_stay_finite():
    """fp32's largest value times one, and sums of products up to (1 - 2^-7) times it."""
    most = torch.finfo(F32).max
    x = torch.tensor([most, -most, most * 0.999, 1.0], device="cuda").repeat(200)[:, None].contiguous()
    W = torch.tensor([1.0, 0.5, -1.0, 2.0 ** -30], device="cuda").view(1, 1, 4)
    out = torch.empty(800, 4, device="cuda")
    forward([0, 800], 800, x, W, None, out)
    assert torch.equal(out.double(), x.double() * W[0].double())
    x = torch.full((300, 16), most / 16, device="cuda")
    W = torch.full((1, 16, 8), 1 - 2.0 ** -7, device="cuda")
    out = torch.empty(300, 8, device="cuda")
    forward([0, 300], 300, x, W, None, out)
    assert (out.double() - most * (1 - 2.0 ** -7)).abs().max() <= most * sums(16)
