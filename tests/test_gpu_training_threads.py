"""Calls of several host threads at once, whose tiles take different amounts of shared memory in the same kernel."""
import threading

import pytest
import torch

import paper_2607_17374_b200 as tb

pytestmark = pytest.mark.gpu


def in_threads(jobs, times=300):
    """Every job `times` times in a thread of its own; the exceptions."""
    errors, gate = [], threading.Barrier(len(jobs))

    def work(job):
        stream = torch.cuda.Stream()
        try:
            gate.wait()
            for _ in range(times):
                job(stream)
        except Exception as e:                   # the library's errors come as exceptions
            errors.append(e)
        stream.synchronize()

    threads = [threading.Thread(target=work, args=(job,)) for job in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    return errors


def test_logprob_of_several_widths():
    jobs, outs = [], []
    for C in (90, 105, 128):                     # tiles of one thread to a row: 45 to 64 KB
        x = torch.randn(5000, C, device="cuda")
        top = torch.empty(5000, 3, dtype=torch.int64, device="cuda")
        jobs.append(lambda s, x=x, top=top, C=C: tb.class_logprob(5000, C, x, C, None, None, None, None, 3, None, top, stream=s))
        outs.append((x, top))
    torch.cuda.synchronize()
    assert in_threads(jobs) == []
    for x, top in outs:
        assert torch.equal(top, x.topk(3, dim=1).indices)


def test_residual_norm_of_several_widths():
    jobs, outs = [], []
    for C, dtype in ((256, torch.float32), (200, torch.float32), (255, torch.float32), (250, torch.float32)):      # 16-byte vectors; words of a team
        x, r, y = (torch.randn(300, C, device="cuda", dtype=dtype) for _ in range(3))
        b, dy, dx, db = (torch.randn(300, C, device="cuda", dtype=dtype) for _ in range(4))
        stats = torch.empty(300, 4, device="cuda")

        def job(s, C=C, x=x, b=b, r=r, y=y, dy=dy, dx=dx, db=db, stats=stats):
            tb.residual_norm(300, C, x, C, b, C, tb.NORM_LAYER, False, None, 0, None, None, 1.0, None, None, 1e-5, r, C, y, C, stats, stream=s)
            tb.residual_norm_grad(300, C, x, C, b, C, tb.NORM_LAYER, False, None, 0, None, None, 1.0, None, stats, None, C, dy, C, dx, C, db, C, None, None, None, None, stream=s)

        jobs.append(job)
        outs.append((x, b, y))
    torch.cuda.synchronize()
    assert in_threads(jobs) == []
    for x, b, y in outs:
        assert torch.allclose(y, torch.nn.functional.layer_norm((x + b).double(), x.shape[1:]).float(), rtol=0, atol=2e-5)     # |y| below 17, a row's mean and sums of 256 in fp32: 17 x 2^-20
