"""AdamW lists whose last reference goes while a stream is being captured, as the garbage collector chooses: the capture goes on, and so does everything else."""
import gc

import pytest
import torch

import paper_2607_17374_b200 as tb

pytestmark = pytest.mark.gpu


def some(n=5000, tensors=1, seed=1):
    g = torch.Generator("cuda").manual_seed(seed)
    p, grad = (torch.randn(n * tensors, generator=g, device="cuda") for _ in range(2))
    m, v = torch.zeros(n * tensors, device="cuda"), torch.zeros(n * tensors, device="cuda")
    return tb.AdamW(*(list(x.split(n)) for x in (p, grad, m, v))), p


def test_a_list_is_collected_during_a_capture():
    step, lr = torch.ones(1, dtype=torch.int64, device="cuda"), torch.full((1,), 1e-2, device="cuda")
    eager, want = some()
    eager.step(step, lr)
    kept, p = some()
    gone = [some(tensors=3)[0] for _ in range(3)]
    gone[0].step(step, lr)
    cycle = [gone.pop()]
    cycle.append(cycle)                                # what only the collector finds
    torch.cuda.synchronize()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=stream):
        gone.clear()
        kept.step(step, lr, stream=stream)
        del cycle
        gc.collect()
    before = p.clone()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(p, want) and not torch.equal(p, before)
    again, q = some()                                  # and no error is left for the next call
    again.step(step, lr)
    assert torch.equal(q, want)


def test_its_memory_is_given_back():
    """30 lists of 20 000 tensors, 2 MB of device memory each, dropped in captures."""
    n = 20_000
    x = torch.zeros(4 * n, device="cuda")
    lists = [list(x[i * n:(i + 1) * n].split(1)) for i in range(4)]
    tb.AdamW(*lists).destroy()
    torch.cuda.synchronize()
    free = torch.cuda.mem_get_info()[0]
    for _ in range(6):
        five = [tb.AdamW(*lists) for _ in range(5)]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            x.add_(1)
            five.clear()
        del graph
    torch.cuda.synchronize()
    assert free - torch.cuda.mem_get_info()[0] < 30 << 20
