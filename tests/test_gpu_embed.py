"""Embedding lookup and its gradient against fp64: types, widths, pitches, ids that are missing, bad, all alike or none."""
import pytest
import torch

import paper_2607_17374_b200 as tb
from rows_reference import U32, close, embed, embed_grad

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def strided(n, width, ld, dtype, shift=0, value=None):
    """n rows ld elements apart that begin `shift` elements behind an aligned address, and the storage around them."""
    store = torch.full((shift + max(n, 1) * ld + 8,), 7.0 if value is None else value, dtype=dtype, device="cuda")
    return torch.as_strided(store, (n, width), (ld, 1), shift), store


def make_ids(n, rows, kind, seed=1):
    g = torch.Generator("cuda").manual_seed(seed)
    if kind == "same":
        return torch.full((n,), rows // 2, dtype=torch.int64, device="cuda")
    if kind == "none":
        return torch.full((n,), -1, dtype=torch.int64, device="cuda")
    if kind == "skew":
        ids = (torch.rand(n, generator=g, device="cuda", dtype=torch.float64) ** 4 * rows).long().clamp_(max=rows - 1)
    else:
        ids = torch.randint(0, rows, (n,), generator=g, device="cuda")
    if kind == "missing" and n > 2:
        ids[torch.rand(n, generator=g, device="cuda") < 0.3] = -1
    return ids


@pytest.mark.parametrize("tt", [F32, BF16, F16])
@pytest.mark.parametrize("ot", [F32, BF16, F16])
@pytest.mark.parametrize("n,rows,width,ld_t,ld_o,shift", [
    (1, 1, 1, 1, 1, 0), (1, 10, 64, 64, 64, 0), (5, 3, 47, 47, 47, 0), (1000, 77, 100, 100, 104, 0), (333, 50, 128, 136, 128, 0), (2049, 600, 1024, 1024, 1024, 0),
    (70, 9, 96, 97, 96, 0), (65, 20, 32, 32, 32, 1), (4000, 1000, 8, 8, 24, 2), (257, 31, 1023, 1023, 1030, 0)])
def test_lookup(tt, ot, n, rows, width, ld_t, ld_o, shift):
    g = torch.Generator("cuda").manual_seed(n + width)
    table, _ = strided(rows, width, ld_t, tt, shift)
    table.copy_(torch.randn(rows, width, generator=g, device="cuda"))
    out, store = strided(n, width, ld_o, ot, shift)
    ids = make_ids(n, rows, "missing")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    tb.embed_rows(n, ids, table, rows, width, ld_t, out, ld_o, 1.7, status)
    ref = embed(ids, table, torch.tensor(1.7, dtype=F32).double().item())
    close(out, ref, ref.abs() * U32)                    # one product in fp32
    inside = torch.zeros_like(store, dtype=torch.bool)
    torch.as_strided(inside, (n, width), (ld_o, 1), shift).fill_(True)
    assert (store[~inside] == 7).all()                  # what stands between the rows is left alone
    assert int(status) == 0


def test_bad_ids_give_zeros_and_a_status():
    ids = torch.tensor([0, -1, 5, -2, 4, 1 << 40], device="cuda")
    table = torch.randn(5, 12, device="cuda")
    out = torch.full((6, 12), 9.0, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    tb.embed_rows(2, ids, table, 5, 12, 12, out, 12, 1.0, status)
    assert int(status) == 0
    tb.embed_rows(6, ids, table, 5, 12, 12, out, 12, 1.0, status)
    assert int(status) == tb.ERROR_CODES["INVALID_ARG"]
    assert torch.equal(out[[0, 4]], table[[0, 4]]) and (out[[1, 2, 3, 5]] == 0).all()
    grad = torch.ones(6, 12, device="cuda")
    gt = torch.full((5, 12), 9.0, device="cuda")
    ws = torch.empty(tb.embed_grad_workspace(6, 5, 12), dtype=torch.uint8, device="cuda")
    status.zero_()
    tb.embed_grad(6, ids, grad, 12, 12, gt, 5, 12, ws, 1.0, status)
    assert int(status) == tb.ERROR_CODES["INVALID_ARG"]
    assert gt[:, 0].tolist() == [1, 0, 0, 0, 1]


def test_offsets_beyond_32_bits():
    """A table and an output of more than 2^32 bytes and 2^31 elements."""
    rows, width = 1 << 22, 1024
    table = torch.empty(rows, width, dtype=BF16, device="cuda")
    table.copy_((torch.arange(rows, device="cuda") % 251)[:, None].expand(rows, width))
    ids = torch.tensor([rows - 1, 0, rows // 2 + 3], device="cuda")
    out = torch.empty(3, width, device="cuda")
    tb.embed_rows(3, ids, table, rows, width, width, out, width)
    assert torch.equal(out[:, 0], (ids % 251).float()) and torch.equal(out[:, -1], out[:, 0])
    n = 1 << 22
    big = torch.empty(n, width, dtype=BF16, device="cuda")
    tb.embed_rows(n, torch.arange(n, device="cuda").flip(0).contiguous(), table, rows, width, width, big, width)
    assert torch.equal(big[-3:], table[:3].flip(0)) and torch.equal(big[:3], table[-3:].flip(0))


@pytest.mark.parametrize("gt,tt", [(F32, F32), (F32, BF16), (BF16, BF16), (F16, F32), (F16, F16), (BF16, F32)])
@pytest.mark.parametrize("n,rows,width,ld_g,ld_t,shift,kind", [
    (1, 1, 1, 1, 1, 0, "skew"), (1, 9, 64, 64, 64, 0, "skew"), (17, 5, 33, 33, 40, 0, "skew"), (16, 3, 47, 47, 47, 0, "same"), (33, 3, 128, 128, 128, 0, "same"),
    (1000, 77, 100, 104, 100, 0, "missing"), (5000, 4, 16, 16, 16, 0, "skew"), (20_000, 1, 64, 64, 64, 0, "skew"), (3000, 5000, 8, 8, 8, 1, "uniform"),
    (2500, 300, 1024, 1024, 1024, 0, "missing"), (4097, 90, 257, 257, 300, 0, "missing"), (500, 40, 36, 36, 36, 0, "none"), (160_001, 2000, 24, 24, 24, 0, "skew")])
def test_gradient(gt, tt, n, rows, width, ld_g, ld_t, shift, kind):
    g = torch.Generator("cuda").manual_seed(n + width)
    ids = make_ids(n, rows, kind)
    grad, _ = strided(n, width, ld_g, gt, shift)
    grad.copy_(torch.randn(n, width, generator=g, device="cuda"))
    table, store = strided(rows, width, ld_t, tt, shift)
    ws = torch.full((tb.embed_grad_workspace(n, rows, width),), 255, dtype=torch.uint8, device="cuda")     # NaN wherever it is read before it is written
    tb.embed_grad(n, ids, grad, ld_g, width, table, rows, ld_t, ws, 0.5)
    ref, mag, count = embed_grad(ids, grad, rows, 0.5)
    close(table, ref, mag * count * U32)
    inside = torch.zeros_like(store, dtype=torch.bool)
    torch.as_strided(inside, (rows, width), (ld_t, 1), shift).fill_(True)
    assert (store[~inside] == 7).all()
    again = table.clone()
    tb.embed_grad(n, ids, grad, ld_g, width, table, rows, ld_t, ws, 0.5)
    assert torch.equal(again, table)                    # the same bits every time


def test_gradient_without_rows():
    table = torch.full((9, 20), 3.0, device="cuda")
    tb.embed_grad(0, None, None, 20, 20, table, 9, 20, None, 1.0, grad_type=tb.F32)
    assert (table == 0).all()


def test_gradient_ignores_what_missing_rows_hold():
    """Rows whose id is -1 may hold anything."""
    ids = torch.tensor([2, -1, 2, -1, 0], device="cuda")
    grad = torch.ones(5, 64, device="cuda")
    grad[1], grad[3] = float("nan"), float("inf")
    table = torch.empty(3, 64, device="cuda")
    ws = torch.empty(tb.embed_grad_workspace(5, 3, 64), dtype=torch.uint8, device="cuda")
    tb.embed_grad(5, ids, grad, 64, 64, table, 3, 64, ws)
    assert table[:, 0].tolist() == [1, 0, 2] and torch.equal(table, table[:, :1].expand(3, 64))


def test_gradient_against_differences():
    """The lookup is linear: (L(t + d) - L(t - d)) / 2 = <gradient, d> for L = <r, lookup>, up to the rounding of the lookups."""
    n, rows, width = 700, 60, 40
    g = torch.Generator("cuda").manual_seed(5)
    table, d = (torch.randn(rows, width, generator=g, device="cuda") for _ in range(2))
    r = torch.randn(n, width, generator=g, device="cuda")
    ids = make_ids(n, rows, "missing")
    loss = []
    for t in (table + d, table - d):
        out = torch.empty(n, width, device="cuda")
        tb.embed_rows(n, ids, t, rows, width, width, out, width, 3.0)
        loss.append(float((out.double() * r.double()).sum()))
    grad = torch.empty(rows, width, device="cuda")
    ws = torch.empty(tb.embed_grad_workspace(n, rows, width), dtype=torch.uint8, device="cuda")
    tb.embed_grad(n, ids, r, width, width, grad, rows, width, ws, 3.0)
    inner = float((grad.double() * ((table + d).double() - (table - d).double())).sum()) / 2
    size = float((r.double().abs() * embed(ids, table.abs() + d.abs(), 3.0)).sum())
    count = int(torch.bincount(ids[ids >= 0]).max())
    assert abs((loss[0] - loss[1]) / 2 - inner) <= size * (count + 4) * U32


def test_refused_on_a_device():
    ids, table, out = torch.zeros(4, dtype=torch.int64, device="cuda"), torch.zeros(10, 8, device="cuda"), torch.zeros(4, 8, device="cuda")
    for bad in (dict(ids=ids.cpu()), dict(table=table.cpu()), dict(out=out.cpu()), dict(out=table), dict(status=torch.zeros(1, dtype=torch.int32))):
        a = dict(ids=ids, table=table, out=out, status=None)
        a.update(bad)
        with pytest.raises(tb.TaurusError) as e:
            tb.embed_rows(4, a["ids"], a["table"], 10, 8, 8, a["out"], 8, 1.0, a["status"])
        assert e.value.code == tb.ERROR_CODES["INVALID_ARG"]
    need = tb.embed_grad_workspace(4, 10, 8)
    ws = torch.empty(need + 512, dtype=torch.uint8, device="cuda")
    for w, g, t in ((ws[:need - 1], out, table), (ws[64:], out, table), (ws, table[:4], table), (ws, out.cpu(), table), (table.view(torch.uint8), out, table)):
        with pytest.raises(tb.TaurusError) as e:
            tb.embed_grad(4, ids, g, 8, 8, t, 10, 8, w)
        assert e.value.code == tb.ERROR_CODES["INVALID_ARG"]


@pytest.mark.parametrize("gt", [F32, BF16])
@pytest.mark.parametrize("n,rows,width,kind", [
    (20_000, 1, 64, "skew"), (2048, 3, 5, "skew"), (2049, 3, 5, "missing"), (160_001, 2000, 24, "same"), (310_000, 50, 12, "skew"), (310_000, 300_000, 8, "uniform"),
    (606_207, 700, 4, "skew"), (606_208, 700, 4, "skew"), (700_001, 2, 3, "missing"), (1_300_000, 90_000, 16, "skew"), (2_500_000, 40, 2, "missing"), (5_000_000, 7, 1, "skew"),
    (700_001, (1 << 22) + 7, 2, "skew"), (5000, (1 << 22) + 7, 3, "uniform"), (900_000, 1 << 22, 1, "missing"), (3000, (1 << 24) + 1, 1, "same")])
def test_whole_numbers_add_up_exactly(gt, n, rows, width, kind):
    """Small whole numbers, whose sums fp32 holds in any order: a row that is lost, doubled or added to another id's sum shows, however many an id has.  Calls with longer pieces,
    sort blocks of several tiles, digits of three passes, and ids over many pieces."""
    g = torch.Generator("cuda").manual_seed(n + rows)
    ids = make_ids(n, rows, kind)
    grad = torch.randint(-3, 4, (n, width), generator=g, device="cuda", dtype=torch.int8).to(gt)
    table = torch.full((rows, width), 9.0, device="cuda")
    ws = torch.full((tb.embed_grad_workspace(n, rows, width),), 255, dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    tb.embed_grad(n, ids, grad, width, width, table, rows, width, ws, 1.0, status)
    assert 3 * n < 1 << 24 and int(status) == 0
    want = torch.zeros(rows, width, dtype=torch.int64, device="cuda")
    keep = ids >= 0
    want.index_add_(0, ids[keep], grad[keep].long())
    assert torch.equal(table, want.float())
