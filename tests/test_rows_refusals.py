"""What the operators on typed rows refuse before they touch the device (no GPU needed): sizes, types, pitches, null and misaligned pointers."""
import pytest
import torch

import paper_2607_17374_b200 as tb

INVALID, UNSUPPORTED = tb.ERROR_CODES["INVALID_ARG"], tb.ERROR_CODES["UNSUPPORTED"]
P = 1 << 20                 # an address that is never used


@pytest.fixture(scope="module")
def lib():
    from paper_2607_17374_b200 import build
    build.build()
    return tb.load_library()


def call(f, good, **change):
    return f(*dict(good, **change).values())


EMBED = dict(n=4, ids=P, table=P, table_type=0, table_rows=10, width=8, ld_table=8, scale=1.0, out=P, out_type=0, ld_out=8, status=None, stream=None)
GRAD = dict(n=4, ids=P, grad=P, grad_type=0, ld_grad=8, width=8, scale=1.0, table=P, table_type=0, table_rows=10, ld_table=8, ws=P, ws_bytes=1 << 30, status=None, stream=None)
TYPED = dict(n=4, types=2, offsets=P, x=P, ld_x=8, type=1, W=P, bias=None, d_in=8, d_out=8, out=P, out_type=1, ld_out=8, ws=None, ws_bytes=0, status=None, stream=None)
TGRAD = dict(n=4, types=2, offsets=P, x=P, ld_x=8, type=1, W=P, dy=P, ld_dy=8, d_in=8, d_out=8, dx=P, ld_dx=8, dW=P, dW_type=1, db=P, ws=None, ws_bytes=0, status=None, stream=None)
NORM = dict(n=4, graphs=1, offsets=P, x=P, ld_x=8, type=1, width=8, groups=2, gamma=P, beta=P, eps=1e-5, act=1, out=P, ld_out=8, mean=None, rstd=None, ws=None, ws_bytes=0,
            status=None, stream=None)
NGRAD = dict(n=4, graphs=1, offsets=P, x=P, ld_x=8, type=1, width=8, groups=2, gamma=P, beta=P, act=1, mean=P, rstd=P, dy=P, ld_dy=8, dx=P, ld_dx=8, dgamma=P, dbeta=P,
             ws=P, ws_bytes=1 << 30, status=None, stream=None)
BIG = 1 << 31


@pytest.mark.parametrize("name,good,bad", [
    ("taurus_embed_rows", EMBED, [dict(n=-1), dict(n=BIG), dict(ids=None), dict(table=None), dict(out=None), dict(table_type=3), dict(out_type=-1), dict(table_rows=0),
                                  dict(table_rows=BIG), dict(width=0), dict(ld_table=7), dict(ld_out=7), dict(ids=P + 4), dict(table=P + 2), dict(out=P + 1), dict(status=P + 2),
                                  dict(ld_out=1 << 62)]),
    ("taurus_embed_grad", GRAD, [dict(n=-1), dict(n=BIG), dict(ids=None), dict(grad=None), dict(table=None), dict(ws=None), dict(ws=P + 128), dict(grad_type=7), dict(table_type=-1),
                                 dict(table_rows=0), dict(ld_grad=7), dict(ld_table=7), dict(table=P + 2), dict(grad=P + 2), dict(ids=P + 4)]),
    ("taurus_typed_project", TYPED, [dict(n=-1), dict(n=BIG), dict(types=0), dict(offsets=None), dict(x=None), dict(W=None), dict(out=None), dict(type=5), dict(out_type=2), dict(d_in=0),
                                     dict(d_out=-3), dict(ld_x=7), dict(ld_out=7), dict(x=P + 1), dict(W=P + 1), dict(offsets=P + 4), dict(bias=P + 2)]),
    ("taurus_typed_project_grad", TGRAD, [dict(n=-1), dict(types=0), dict(offsets=None), dict(x=None), dict(W=None), dict(dy=None), dict(type=5), dict(dW_type=2), dict(ld_x=7), dict(ld_dy=7),
                                          dict(ld_dx=7), dict(dx=P + 1), dict(dW=P + 1), dict(db=P + 2)]),
    ("taurus_norm_rows", NORM, [dict(n=-1), dict(n=BIG), dict(graphs=0), dict(groups=0), dict(groups=3), dict(width=0), dict(x=None), dict(out=None), dict(type=9), dict(act=3), dict(act=-1),
                                dict(eps=-1.0), dict(eps=float("nan")), dict(ld_x=7), dict(ld_out=7), dict(x=P + 1), dict(gamma=P + 2), dict(offsets=None, graphs=2)]),
    ("taurus_norm_rows_grad", NGRAD, [dict(n=-1), dict(graphs=0), dict(groups=3), dict(x=None), dict(dy=None), dict(dx=None), dict(mean=None), dict(rstd=None), dict(act=4), dict(ld_dx=7),
                                      dict(ld_dy=7), dict(dgamma=P + 2), dict(offsets=None, graphs=2)]),
])
def test_arguments_that_are_refused(lib, name, good, bad):
    f = getattr(lib, name)
    for change in bad:
        assert call(f, good, **change) == INVALID, change


@pytest.mark.parametrize("name,good,wide", [
    ("taurus_embed_rows", EMBED, dict(width=1025, ld_table=2000, ld_out=2000)),
    ("taurus_embed_grad", GRAD, dict(width=1025, ld_table=2000, ld_grad=2000)),
    ("taurus_typed_project", TYPED, dict(d_in=1025, ld_x=2000)),
    ("taurus_typed_project", TYPED, dict(d_out=1025, ld_out=2000)),
    ("taurus_typed_project", TYPED, dict(types=1025)),
    ("taurus_typed_project_grad", TGRAD, dict(d_in=1025, ld_x=2000, ld_dx=2000)),
    ("taurus_norm_rows", NORM, dict(width=1026, ld_x=2000, ld_out=2000)),
    ("taurus_norm_rows_grad", NGRAD, dict(width=1026, ld_x=2000, ld_dy=2000, ld_dx=2000)),
])
def test_sizes_that_are_not_supported(lib, name, good, wide):
    assert call(getattr(lib, name), good, **wide) == UNSUPPORTED


def test_calls_with_nothing_to_do_need_no_device(lib):
    assert call(lib.taurus_embed_rows, EMBED, n=0, ids=None, out=None) == 0
    assert call(lib.taurus_typed_project, TYPED, n=0, x=None, out=None) == 0
    assert call(lib.taurus_typed_project_grad, TGRAD, dx=None, dW=None, db=None) == 0


def test_workspace_sizes_that_are_refused(lib):
    assert lib.taurus_embed_grad_workspace(4, 10, 0) == INVALID
    assert lib.taurus_embed_grad_workspace(4, 10, 1025) == UNSUPPORTED
    assert lib.taurus_typed_project_workspace(4, 0, 8, 8, 0) == INVALID
    assert lib.taurus_typed_project_workspace(4, 1025, 8, 8, 0) == UNSUPPORTED
    assert lib.taurus_typed_project_grad_workspace(4, 1, 8, 8, 5) == INVALID
    assert lib.taurus_norm_rows_workspace(4, 1, 8, 3) == INVALID
    assert lib.taurus_norm_rows_grad_workspace(4, 1, 2048, 1) == UNSUPPORTED


def test_tensors_that_do_not_fit_the_call():
    """The binding's own checks: sizes, strides and dtypes of the tensors it is given."""
    ids, table, out = torch.zeros(4, dtype=torch.int64), torch.zeros(10, 8), torch.zeros(4, 8)
    with pytest.raises(ValueError):
        tb.embed_rows(5, ids, table, 10, 8, 8, torch.zeros(5, 8), 8)
    with pytest.raises(ValueError):
        tb.embed_rows(4, ids, table, 10, 8, 8, out[:, :7], 8)
    with pytest.raises(ValueError):
        tb.embed_rows(4, ids, table.T.contiguous().T, 10, 8, 8, out, 8)
    with pytest.raises(TypeError):
        tb.embed_rows(4, ids.int(), table, 10, 8, 8, out, 8)
    with pytest.raises(TypeError):
        tb.embed_rows(4, ids, table.double(), 10, 8, 8, out, 8)
    off = torch.tensor([0, 4])
    with pytest.raises(TypeError):
        tb.typed_project(4, 1, off, out, 8, torch.zeros(1, 8, 8, dtype=torch.bfloat16), None, 8, 8, torch.zeros(4, 8), 8)
    with pytest.raises(ValueError):
        tb.typed_project(4, 2, off, out, 8, torch.zeros(2, 8, 8), None, 8, 8, torch.zeros(4, 8), 8)
    with pytest.raises(TypeError):
        tb.norm_rows(4, 1, off, out, 8, 8, 2, None, None, 1e-5, 1, out.half(), 8)


@pytest.mark.skipif(torch.cuda.is_available(), reason="needs a machine without a GPU")
def test_host_memory_and_no_device_are_errors_not_crashes():
    ids, table, out = torch.zeros(4, dtype=torch.int64), torch.zeros(10, 8), torch.zeros(4, 8)
    with pytest.raises(tb.TaurusError) as e:
        tb.embed_rows(4, ids, table, 10, 8, 8, out, 8)
    assert e.value.code in (tb.ERROR_CODES["CUDA"], INVALID)


def test_more_graphs_than_there_may_be(lib):
    for f in (lib.taurus_norm_rows_workspace, lib.taurus_norm_rows_grad_workspace):
        assert f(4, (1 << 30) + 1, 8, 1) == INVALID and f(4, 1 << 30, 8, 1) >= 0
    assert call(lib.taurus_norm_rows, NORM, graphs=(1 << 30) + 1) == INVALID


def test_a_type_that_is_said_and_is_not_the_tensors():
    """Tensors are taken at their own type; an argument that says a wider one would have the call reach past their end."""
    ids, off, v = torch.zeros(4, dtype=torch.int64), torch.tensor([0, 4]), torch.zeros(8)
    x, y, table, W = (torch.zeros(s, dtype=torch.bfloat16) for s in ((4, 8), (4, 8), (10, 8), (1, 8, 8)))
    ws = torch.empty(1 << 16, dtype=torch.uint8)
    one = torch.zeros(1, 2)
    P = x.data_ptr()
    for call in (lambda: tb.embed_rows(4, ids, table, 10, 8, 8, x, 8, table_type=tb.F32),
                 lambda: tb.embed_rows(4, ids, table, 10, 8, 8, x, 8, out_type=torch.float32),
                 lambda: tb.embed_grad(4, ids, x, 8, 8, table, 10, 8, ws, grad_type=tb.F32),
                 lambda: tb.embed_grad(4, ids, x, 8, 8, table, 10, 8, ws, table_type=tb.F16),
                 lambda: tb.typed_project(4, 1, off, x, 8, P, None, 8, 8, P, 8, type=tb.F32, out_type=tb.F32),
                 lambda: tb.typed_project(4, 1, off, x, 8, W, None, 8, 8, y, 8, out_type=tb.F32),
                 lambda: tb.typed_project_grad(4, 1, off, P, 8, P, x, 8, 8, 8, P, 8, type=tb.F32),
                 lambda: tb.typed_project_grad(4, 1, off, x, 8, W, y, 8, 8, 8, grad_W=W, grad_W_type=tb.F32),
                 lambda: tb.norm_rows(4, 1, off, x, 8, 8, 2, v, v, 1e-5, 1, P, 8, type=tb.F32),
                 lambda: tb.norm_rows_grad(4, 1, off, x, 8, 8, 2, v, v, 1, one, one, P, 8, P, 8, workspace=ws, type=tb.F32)):
        with pytest.raises(TypeError):
            call()


def test_a_workspace_for_more_rows_does_for_fewer(lib):
    """A program that asks once, for its largest batch, has enough for the others."""
    import random
    rng = random.Random(4)
    sizes = sorted({1, 64, 65, 606_207, 606_208, 1_212_415, 1_212_416, 2_424_831, 2_424_832, 2_424_833, 308_223, 308_224, 151_552, 151_553, 303_104, 303_105, (1 << 31) - 1}
                   | {int(2 ** rng.uniform(0, 31)) - 1 for _ in range(600)} | {k * 1184 + d for k in (2, 3, 4, 8, 9, 100) for d in (-1, 0, 1)})
    cases = [(lib.taurus_embed_grad_workspace, a) for a in ((1003, 47), (400_000, 128), (1 << 22, 1024), (5, 1))]
    cases += [(f, a) for f in (lib.taurus_typed_project_workspace, lib.taurus_typed_project_grad_workspace) for a in
              ((1, 64, 64, 0), (16, 512, 256, 1), (200, 128, 128, 2), (1000, 1024, 1024, 1), (7, 37, 130, 1), (7, 37, 130, 0), (3, 300, 1000, 2))]
    for f, rest in cases:
        got = [f(n, *rest) for n in sizes]
        assert all(g >= 0 for g in got) and got == sorted(got), (f.__name__, rest)
    for f in (lib.taurus_norm_rows_workspace, lib.taurus_norm_rows_grad_workspace):
        for width, groups in ((64, 8), (1024, 1024), (1, 1), (257, 1), (1024, 32)):
            for graphs in (1, 3, 1183, 1184, 9001, 100_000):
                got = [f(n, graphs, width, groups) for n in sizes]
                assert all(g >= 0 for g in got) and got == sorted(got), (f.__name__, width, groups, graphs)
            for n in (5000, 262_144, 3_000_000):      # and one for more graphs does for fewer
                got = [f(n, graphs, width, groups) for graphs in (1, 2, 100, 1183, 1184, 1185, 2368, 2369, 5000, 100_000, 1 << 30)]
                assert got == sorted(got), (f.__name__, width, groups, n)
