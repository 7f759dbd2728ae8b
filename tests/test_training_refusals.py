"""What class log probabilities, the residual norm and AdamW refuse before they touch the device (no GPU needed): sizes, types, pitches, null and misaligned pointers."""
import ctypes

import pytest
import torch

import paper_2607_17374_b200 as tb
from paper_2607_17374_b200.binding import _AdamWTensor

INVALID, UNSUPPORTED, CUDA = (tb.ERROR_CODES[k] for k in ("INVALID_ARG", "UNSUPPORTED", "CUDA"))
P = 1 << 20                 # an address that is never used
BIG = 1 << 31


@pytest.fixture(scope="module")
def lib():
    from paper_2607_17374_b200 import build
    build.build()
    return tb.load_library()


def call(f, good, **change):
    return f(*dict(good, **change).values())


LOGPROB = dict(n=4, classes=8, x=P, ld=8, type=0, labels=P, logprob=P, entropy=P, stats=P, k=2, top=P, cls=P, ws=None, ws_bytes=0, status=None, stream=None)
TRAIN = dict(n=4, classes=8, x=P, ld=8, type=1, labels=P, g=P, h=P, logprob=P, entropy=P, stats=P, dx=P, ld_dx=8, ws=None, ws_bytes=0, status=None, stream=None)
LGRAD = dict(n=4, classes=8, x=P, ld=8, type=1, labels=P, stats=P, entropy=P, g=P, h=P, dx=P, ld_dx=8, status=None, stream=None)
NORM = dict(n=4, width=8, res=P, ld_res=8, res_type=0, block=P, ld_block=8, type=1, kind=0, post=1, post_gamma=P, groups=2, offsets=P, gate=P, alpha=1.0, gamma=P, beta=P, eps=1e-5,
            out_res=P, ld_out_res=8, out=P, ld_out=8, stats=P, status=None, stream=None)
NGRAD = dict(n=4, width=8, res=P, ld_res=8, res_type=0, block=P, ld_block=8, type=1, kind=0, post=1, post_gamma=P, groups=2, offsets=P, gate=P, alpha=1.0, gamma=P, stats=P, dres=P, ld_dres=8,
             dy=P, ld_dy=8, d_res=P, ld_d_res=8, d_block=P, ld_d_block=8, d_post=P, d_gate=P, d_gamma=P, d_beta=P, ws=P, ws_bytes=1 << 30, status=None, stream=None)
NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("name,good,bad", [
    ("taurus_class_logprob", LOGPROB, [dict(n=-1), dict(n=BIG), dict(classes=0), dict(classes=-5), dict(x=None), dict(x=P + 2), dict(ld=7), dict(ld=1 << 61), dict(type=3), dict(type=-1), dict(labels=None),
                                       dict(labels=P + 4), dict(logprob=P + 2), dict(entropy=P + 1), dict(stats=P + 4), dict(k=-1), dict(top=None, cls=None), dict(top=P + 2), dict(cls=P + 4), dict(status=P + 2)]),
    ("taurus_class_logprob_train", TRAIN, [dict(n=-1), dict(classes=0), dict(x=None), dict(x=P + 1), dict(ld=7), dict(type=4), dict(labels=None), dict(labels=None, logprob=None), dict(g=None, h=None), dict(g=P + 2),
                                           dict(h=P + 2), dict(dx=None), dict(dx=P + 1), dict(ld_dx=7), dict(stats=P + 4)]),
    ("taurus_class_logprob_grad", LGRAD, [dict(n=BIG), dict(classes=0), dict(x=None), dict(ld=7), dict(type=4), dict(labels=None), dict(stats=None), dict(stats=P + 4), dict(entropy=None), dict(g=None, h=None), dict(dx=None),
                                          dict(dx=P + 1), dict(ld_dx=7)]),
    ("taurus_residual_norm", NORM, [dict(n=-1), dict(n=BIG), dict(width=0), dict(res=None), dict(res=P + 2), dict(ld_res=7), dict(res_type=2), dict(res_type=3), dict(type=3), dict(block=P + 1), dict(ld_block=7),
                                    dict(kind=2), dict(kind=-1), dict(post=2), dict(post=0), dict(groups=0), dict(groups=-1), dict(offsets=P + 4), dict(offsets=None), dict(gate=None), dict(gate=P + 2), dict(alpha=NAN),
                                    dict(alpha=INF), dict(gamma=P + 2), dict(beta=P + 2), dict(eps=-1.0), dict(eps=NAN), dict(out_res=None), dict(out_res=P + 2), dict(ld_out_res=7), dict(out=None), dict(out=P + 1),
                                    dict(ld_out=7), dict(stats=P + 8), dict(status=P + 2), dict(block=None), dict(block=None, post=0, post_gamma=None, groups=0, offsets=None, gate=None), dict(groups=(1 << 30) + 1)]),
    ("taurus_residual_norm_grad", NGRAD, [dict(n=-1), dict(width=0), dict(res=None), dict(ld_res=7), dict(res_type=2), dict(type=9), dict(kind=5), dict(post=0), dict(groups=0), dict(stats=None), dict(stats=P + 8),
                                          dict(dres=None, dy=None), dict(dres=P + 2), dict(ld_dres=7), dict(dy=P + 1), dict(ld_dy=7), dict(d_res=None), dict(d_res=P + 2), dict(ld_d_res=7), dict(d_block=P + 1),
                                          dict(ld_d_block=7), dict(d_post=P + 2), dict(d_gate=P + 2), dict(d_gamma=P + 2), dict(d_beta=P + 2), dict(gate=None, groups=0, offsets=None),
                                          dict(block=None, post=0, post_gamma=None, groups=0, offsets=None, gate=None, d_gate=None, d_post=None)]),
])
def test_arguments_that_are_refused(lib, name, good, bad):
    f = getattr(lib, name)
    for change in bad:
        assert call(f, good, **change) == INVALID, change


@pytest.mark.parametrize("name,good,wide", [
    ("taurus_class_logprob", LOGPROB, dict(classes=tb.MAX_CLASSES + 1, ld=1 << 21)),
    ("taurus_class_logprob", LOGPROB, dict(k=tb.MAX_TOP + 1)),
    ("taurus_class_logprob_train", TRAIN, dict(classes=tb.MAX_CLASSES + 1, ld=1 << 21, ld_dx=1 << 21)),
    ("taurus_class_logprob_grad", LGRAD, dict(classes=tb.MAX_CLASSES + 1, ld=1 << 21, ld_dx=1 << 21)),
    ("taurus_residual_norm", NORM, dict(width=1025, ld_res=2000, ld_block=2000, ld_out_res=2000, ld_out=2000)),
    ("taurus_residual_norm_grad", NGRAD, dict(width=1025, ld_res=2000, ld_block=2000, ld_dres=2000, ld_dy=2000, ld_d_res=2000, ld_d_block=2000)),
])
def test_sizes_that_are_not_supported(lib, name, good, wide):
    assert call(getattr(lib, name), good, **wide) == UNSUPPORTED


def test_calls_with_nothing_to_do_need_no_device(lib):
    assert call(lib.taurus_class_logprob, LOGPROB, n=0, x=None, labels=None) == 0
    assert call(lib.taurus_class_logprob_train, TRAIN, n=0, x=None, dx=None) == 0
    assert call(lib.taurus_class_logprob_grad, LGRAD, n=0, x=None, dx=None) == 0
    assert call(lib.taurus_residual_norm, NORM, n=0, res=None, block=None, out_res=None, out=None, post=0, post_gamma=None) == 0


def test_workspaces(lib):
    assert lib.taurus_class_logprob_workspace(4, 0, 0) == INVALID and lib.taurus_class_logprob_workspace(-1, 5, 0) == INVALID and lib.taurus_class_logprob_workspace(4, 5, -1) == INVALID
    assert lib.taurus_class_logprob_workspace(4, tb.MAX_CLASSES + 1, 0) == UNSUPPORTED and lib.taurus_class_logprob_workspace(4, 5, 17) == UNSUPPORTED
    assert lib.taurus_residual_norm_grad_workspace(4, 0, 1) == INVALID and lib.taurus_residual_norm_grad_workspace(4, 8, -1) == INVALID and lib.taurus_residual_norm_grad_workspace(4, 1025, 1) == UNSUPPORTED
    sizes = sorted({1, 2, 3, 9, 10, 63, 64, 65, 295, 296, 297, 591, 592, 593, 2368, 2369, 75_776, 1_000_000, BIG - 1} | {k * 592 + d for k in (2, 3, 8) for d in (-1, 0, 1)})
    for classes in (10, 1024, 16_383, 16_384, 40_000, 1 << 20):
        for k in (0, 1, 16):
            got = [lib.taurus_class_logprob_workspace(n, classes, k) for n in sizes]
            assert all(g >= 0 for g in got) and got == sorted(got)
    for width in (1, 8, 9, 100, 256, 1000, 1024):
        for groups in (0, 1, 5000, 1 << 30):
            got = [lib.taurus_residual_norm_grad_workspace(n, width, groups) for n in sizes]
            assert all(g >= 0 for g in got) and got == sorted(got)


def tensor(**change):
    d = dict(param=P, grad=2 * P, m=3 * P, v=4 * P, m_scale=None, v_scale=None, master=None, count=100, weight_decay=0.1, param_type=0, grad_type=0, state_type=0)
    return _AdamWTensor(*dict(d, **change).values())


def test_adamw_lists_that_are_refused(lib):
    h = ctypes.c_void_p()

    def create(*tensors, count=None):
        table = (_AdamWTensor * max(1, len(tensors)))(*tensors)
        return lib.taurus_adamw_create(ctypes.byref(h), table, len(tensors) if count is None else count)

    for bad in (dict(param=None), dict(m=None), dict(v=None), dict(param=P + 2), dict(grad=2 * P + 1, grad_type=1), dict(m=3 * P + 2), dict(count=-1), dict(count=1 << 41), dict(weight_decay=NAN), dict(weight_decay=INF),
                dict(param_type=3), dict(grad_type=5), dict(state_type=1), dict(state_type=3), dict(master=5 * P), dict(state_type=3, m_scale=5 * P), dict(state_type=3, m_scale=5 * P + 2, v_scale=6 * P),
                dict(param_type=1, master=5 * P + 2), dict(grad=P), dict(v=3 * P + 396), dict(m=P + 396), dict(grad=P + 396), dict(param_type=1, master=3 * P)):
        assert create(tensor(**bad)) == INVALID, bad
    assert create(tensor(), tensor(param=7 * P, m=8 * P, v=9 * P, grad=3 * P)) == INVALID                 # the gradient of one is the state of another
    assert create(tensor(), tensor()) == INVALID                                                          # the same tensor twice
    assert create(tensor(), count=-1) == INVALID and lib.taurus_adamw_create(ctypes.byref(h), None, 1) == INVALID and lib.taurus_adamw_create(None, None, 0) == INVALID
    assert lib.taurus_adamw_step(None, P, P, 0.9, 0.999, 1e-8, None, 0, None, None) == INVALID
    lib.taurus_adamw_destroy(None)
    assert not h.value


@pytest.mark.skipif(torch.cuda.is_available(), reason="needs a machine without a GPU")
def test_no_device_is_an_error_and_not_a_crash(lib):
    h = ctypes.c_void_p()
    assert lib.taurus_adamw_create(ctypes.byref(h), (_AdamWTensor * 1)(tensor()), 1) == CUDA and not h.value
    assert call(lib.taurus_class_logprob, LOGPROB) == CUDA and call(lib.taurus_residual_norm, NORM) == CUDA and call(lib.taurus_residual_norm_grad, NGRAD) == CUDA


def test_tensors_that_do_not_fit_the_call():
    """The binding's own checks: sizes, strides and dtypes of the tensors it is given."""
    x, labels, lp = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int64), torch.zeros(4)
    b = torch.zeros(4, 8, dtype=torch.bfloat16)
    v = torch.zeros(8)
    for error, f in [
            (ValueError, lambda: tb.class_logprob(5, 8, x, 8, labels, lp)), (ValueError, lambda: tb.class_logprob(4, 9, x, 8, labels, lp)), (TypeError, lambda: tb.class_logprob(4, 8, x, 8, labels.int(), lp)),
            (TypeError, lambda: tb.class_logprob(4, 8, x, 8, labels, lp.double())), (ValueError, lambda: tb.class_logprob(4, 8, x, 8, labels, lp, stats=torch.zeros(4))),
            (ValueError, lambda: tb.class_logprob(4, 8, x, 8, k=3, top_class=labels)), (TypeError, lambda: tb.class_logprob(4, 8, x, 8, labels, lp, type=tb.BF16)),
            (TypeError, lambda: tb.class_logprob_train(4, 8, x, 8, labels, lp, None, None, None, None, b, 8)), (TypeError, lambda: tb.class_logprob_grad(4, 8, x, 8, labels, x, None, lp, None, b, 8)),
            (TypeError, lambda: tb.residual_norm(4, 8, x, 8, x, 8, 0, 0, None, 0, None, None, 1.0, v, v, 1e-5, x, 8, b, 8)), (TypeError, lambda: tb.residual_norm(4, 8, x, 8, b, 8, 0, 0, None, 0, None, None, 1.0, v, v, 1e-5, b, 8, b, 8)),
            (ValueError, lambda: tb.residual_norm(4, 8, x, 8, b, 8, 0, 1, torch.zeros(7), 0, None, None, 1.0, v, v, 1e-5, x, 8, b, 8)),
            (ValueError, lambda: tb.residual_norm(4, 8, x, 8, b, 8, 0, 0, None, 2, labels[:3], torch.zeros(1, 8), 1.0, v, v, 1e-5, x, 8, b, 8)),
            (ValueError, lambda: tb.residual_norm(4, 8, x, 8, b, 8, 0, 0, None, 0, None, None, 1.0, v, v, 1e-5, x, 8, b, 8, stats=torch.zeros(4, 3))),
            (TypeError, lambda: tb.residual_norm_grad(4, 8, x, 8, b, 8, 0, 0, None, 0, None, None, 1.0, v, torch.zeros(4, 4), x, 8, x, 8, x, 8, b, 8)),
            (TypeError, lambda: tb.residual_norm_grad(4, 8, x, 8, b, 8, 0, 0, None, 0, None, None, 1.0, v, torch.zeros(4, 4), b, 8, b, 8, x, 8, b, 8)),
            (ValueError, lambda: tb.AdamW([v], [], [v], [v])), (ValueError, lambda: tb.AdamW([v], [torch.zeros(7)], [v], [v])), (TypeError, lambda: tb.AdamW([v], [v], [v], [v.half()])),
            (ValueError, lambda: tb.AdamW([v], [v], [torch.zeros(7)], [v])), (TypeError, lambda: tb.AdamW([v.double()], [v], [v], [v])),
            (ValueError, lambda: tb.AdamW([torch.zeros(600)], [torch.zeros(600)], [torch.zeros(600, dtype=torch.uint8)], [torch.zeros(600, dtype=torch.uint8)], [torch.zeros(2)], [torch.zeros(3)])),
            (ValueError, lambda: tb.AdamW([torch.zeros(8, 8).T[:4]], [torch.zeros(32)], [torch.zeros(32)], [torch.zeros(32)]))]:
        with pytest.raises(error):
            f()
