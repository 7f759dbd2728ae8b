"""Calls of several host threads at once of one kernel whose shared memory is of another size in each, above what a kernel may have without asking: rows of logits in tiles, and gradients of the
residual norm, each bit for bit what a call alone gives."""
import pytest
import torch

import paper_2607_17374_b200 as tb
from logprob_reference import top_of
from test_gpu_training_threads import in_threads

pytestmark = pytest.mark.gpu
N = 10_000                                       # rows: 900 000 elements and more, so that they come in tiles


def test_logprob_in_tiles_of_several_widths():
    jobs, outs = [], []
    for C in (90, 105, 128):                     # top 16: one thread to a row, 128 rows of 90, 105, 129 words: 45 to 65 KB in rows_kernel<float, top 16, 1 thread>
        x = torch.randn(N, C, device="cuda")
        labels = torch.randint(0, C, (N,), device="cuda")

        def call(s, out, x=x, labels=labels, C=C):
            tb.class_logprob(N, C, x, C, labels, out[0], out[1], out[2], 16, out[3], out[4], stream=s)

        def empty():
            return [torch.empty(N, device="cuda"), torch.empty(N, device="cuda"), torch.empty(N, 2, device="cuda"), torch.empty(N, 16, device="cuda"), torch.empty(N, 16, dtype=torch.int64, device="cuda")]

        alone, out = empty(), empty()
        call(None, alone)
        jobs.append(lambda s, call=call, out=out: call(s, out))
        outs.append((x, alone, out))
    torch.cuda.synchronize()
    assert in_threads(jobs) == []
    for x, alone, out in outs:
        assert all(torch.equal(a, b) for a, b in zip(alone, out)) and torch.equal(out[4], top_of(x, 16))


def test_residual_norm_and_gradients_of_several_widths():
    jobs, outs = [], []
    n = 300
    for C in (256, 200, 255, 250, 7, 3):         # 16-byte vectors; words of a team, up to 96 KB for rows of one thread
        x, b, dy, dr = (torch.randn(n, C, device="cuda") for _ in range(4))
        gamma = torch.randn(C, device="cuda")

        def call(s, out, ws, x=x, b=b, dy=dy, dr=dr, gamma=gamma, C=C):
            y, r, stats, dx, db, dg, dp = out
            tb.residual_norm(n, C, x, C, b, C, tb.NORM_LAYER, True, gamma, 0, None, None, 1.0, gamma, None, 1e-5, r, C, y, C, stats, stream=s)
            tb.residual_norm_grad(n, C, x, C, b, C, tb.NORM_LAYER, True, gamma, 0, None, None, 1.0, gamma, stats, dr, C, dy, C, dx, C, db, C, dp, None, dg, None, ws, stream=s)

        def empty():
            return [torch.empty(n, C, device="cuda"), torch.empty(n, C, device="cuda"), torch.empty(n, 4, device="cuda"), torch.empty(n, C, device="cuda"), torch.empty(n, C, device="cuda"),
                    torch.empty(C, device="cuda"), torch.empty(C, device="cuda")]

        alone, out = empty(), empty()
        ws = [torch.empty(tb.residual_norm_grad_workspace(n, C, 0), dtype=torch.uint8, device="cuda") for _ in range(2)]
        call(None, alone, ws[0])
        jobs.append(lambda s, call=call, out=out, w=ws[1]: call(s, out, w))
        outs.append((alone, out))
    torch.cuda.synchronize()
    assert in_threads(jobs, 200) == []
    for alone, out in outs:
        assert all(torch.equal(a, b) for a, b in zip(alone, out))
