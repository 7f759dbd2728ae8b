"""The operators on typed rows as they are used together: rows looked up in a table, projected by vertex type, normed, handed to the layers; their gradients
back to the table; and how they are launched: other streams, captured graphs, workspaces of their own."""
import numpy as np
import pytest
import torch

import paper_2607_17374_b200 as tb
import taurus_gen as tg
from rows_reference import U32, act, norm

pytestmark = pytest.mark.gpu
EPS = 1e-5


class Encoder:
    """Table -> scaled rows -> W of the vertex's type + bias -> group norm + silu, for n vertices grouped by type (one graph)."""

    def __init__(self, n, rows, d, h, types, groups, t, seed=0):
        g = torch.Generator("cuda").manual_seed(seed)
        self.n, self.rows, self.d, self.h, self.groups, self.t, self.types = n, rows, d, h, groups, t, types
        self.table = (torch.randn(rows, d, generator=g, device="cuda") * 0.3).to(t)
        self.ids = torch.randint(-1, rows, (n,), generator=g, device="cuda")
        cut = torch.sort(torch.randint(0, n + 1, (types - 1,), generator=g, device="cuda")).values
        self.offsets = torch.cat([cut.new_zeros(1), cut, cut.new_full((1,), n)])
        self.W = (torch.randn(types, d, h, generator=g, device="cuda") / d ** 0.5).to(t)
        self.b = torch.randn(types, h, generator=g, device="cuda") * 0.1
        self.gamma, self.beta = 1 + 0.1 * torch.randn(h, generator=g, device="cuda"), 0.1 * torch.randn(h, generator=g, device="cuda")
        self.dy = torch.randn(n, h, generator=g, device="cuda").to(t)
        e = lambda *s, dt=t: torch.full(s, 77.0, dtype=dt, device="cuda")
        f = torch.float32
        self.x, self.p, self.y = e(n, d), e(n, h), e(n, h)
        self.mean, self.rstd = e(1, groups, dt=f), e(1, groups, dt=f)
        self.dp, self.dx, self.dtable = e(n, h), e(n, d), e(rows, d)
        self.dW, self.db, self.dgamma, self.dbeta = e(types, d, h, dt=f), e(types, h, dt=f), e(h, dt=f), e(h, dt=f)
        need = [tb.embed_grad_workspace(n, rows, d), tb.typed_project_workspace(n, types, d, h, t), tb.typed_project_grad_workspace(n, types, d, h, t),
                tb.norm_rows_workspace(n, 1, h, groups), tb.norm_rows_grad_workspace(n, 1, h, groups)]
        self.ws = torch.empty(max(need), dtype=torch.uint8, device="cuda")            # calls in order share it
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def run(self, stream):
        k = dict(status=self.status, stream=stream)
        n, d, h = self.n, self.d, self.h
        tb.embed_rows(n, self.ids, self.table, self.rows, d, d, self.x, d, 2.0, **k)
        tb.typed_project(n, self.types, self.offsets, self.x, d, self.W, self.b, d, h, self.p, h, self.ws, **k)
        tb.norm_rows(n, 1, None, self.p, h, h, self.groups, self.gamma, self.beta, EPS, tb.ACT_SILU, self.y, h, self.mean, self.rstd, self.ws, **k)
        tb.norm_rows_grad(n, 1, None, self.p, h, h, self.groups, self.gamma, self.beta, tb.ACT_SILU, self.mean, self.rstd, self.dy, h, self.dp, h, self.dgamma, self.dbeta,
                          self.ws, **k)
        tb.typed_project_grad(n, self.types, self.offsets, self.x, d, self.W, self.dp, h, d, h, self.dx, d, self.dW, self.db, self.ws, **k)
        tb.embed_grad(n, self.ids, self.dx, d, d, self.dtable, self.rows, d, self.ws, 2.0, **k)

    def results(self):
        return [t.clone() for t in (self.x, self.p, self.y, self.mean, self.rstd, self.dp, self.dgamma, self.dbeta, self.dx, self.dW, self.db, self.dtable)]


def exact(e):
    """The same in fp64, gradients by autograd."""
    leaves = [p.double().requires_grad_() for p in (e.table, e.W, e.b, e.gamma, e.beta)]
    table, W, b, gamma, beta = leaves
    x = torch.where((e.ids >= 0)[:, None], table[e.ids.clamp(min=0)], torch.zeros(1, dtype=torch.float64, device="cuda")) * 2
    off = e.offsets.tolist()
    p = torch.cat([x[s:t] @ W[g] + b[g] for g, (s, t) in enumerate(zip(off, off[1:]))])
    v = p.reshape(e.n, e.groups, -1)
    m = v.mean((0, 2), keepdim=True)
    r = 1 / torch.sqrt(((v - m) ** 2).mean((0, 2), keepdim=True) + EPS)
    y = act(2, ((v - m) * r).reshape(e.n, e.h) * gamma + beta)
    return y.detach(), torch.autograd.grad(y, leaves, e.dy.double())


@pytest.mark.parametrize("n,rows,d,h,types,groups", [(50, 20, 40, 48, 3, 6), (3000, 500, 64, 96, 5, 8), (40_000, 3000, 100, 128, 7, 16)])
def test_forward_and_back(n, rows, d, h, types, groups):
    """fp32 end to end: each result within 2^-24 times 4 096 of the largest of its kind in the norm of the whole (rounding errors of sums of up to 40 000 terms
    grow like their square root, 200, through three operators there and back)."""
    e = Encoder(n, rows, d, h, types, groups, torch.float32)
    e.run(None)
    y, grads = exact(e)
    assert int(e.status) == 0
    for got, want in [(e.y, y)] + list(zip((e.dtable, e.dW, e.db, e.dgamma, e.dbeta), grads)):
        assert float((got.double() - want).norm()) <= 4096 * U32 * float(want.norm())


def test_rows_into_a_layer():
    """What the encoder made goes into taurus_push_chunk as a chunk's features, on the same stream, and comes out as the layer's result for those rows."""
    from dataclasses import replace
    w = replace(tg.scaled(tg.WORKLOADS["large"], 3_000, chunk=512, name="encoder"), dims=(96, 64), fanout=(0,), pool_slots=3_000, hub_count=5, mode=tg.SAGE_MEAN)
    g, m = tg.make_graph(w), tg.make_model(w, bias_scale=0.3)
    e = Encoder(g.V, 500, 64, 96, 4, 8, torch.float32)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    ctx = tb.Context(g.V, g.E, g.row_ptr, g.col_idx, g.in_degree, w.mode, w.dims, m.W_neigh, m.W_self, m.bias, m.act, w.chunk, w.pool_slots, w.hub_count, w.fanout, w.seed, 0, g.V)
    out = torch.empty(g.V, 64, device="cuda")
    ctx.layer_begin(0, stream)
    ctx.layer_set_dense_output(out, 64)
    e.run(stream)
    for b in range(0, g.V, w.chunk):
        ctx.push_chunk(b, min(b + w.chunk, g.V), e.y[b:b + w.chunk], stream)
    assert ctx.layer_end()["completed"] == g.V
    x = e.y.double().cpu().numpy()
    agg = np.zeros_like(x)
    for u in range(g.V):
        np.add.at(agg, g.col_idx[g.row_ptr[u]:g.row_ptr[u + 1]], x[u])
    agg /= np.maximum(g.in_degree, 1)[:, None]
    want = agg @ m.W_neigh[0].astype(np.float64) + x @ m.W_self[0].astype(np.float64) + m.bias[0]
    if m.act[0]:
        want = np.maximum(want, 0)
    got = out.double().cpu().numpy()
    assert np.linalg.norm(got - want) <= 1e-5 * np.linalg.norm(want)


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n", [40, 5000, 60_000])
def test_captured_and_replayed(t, n):
    """Captured into a graph and replayed on new inputs: the bits of the eager calls; an eager run between replays changes nothing."""
    e = Encoder(n, 300, 64, 96, 4, 8, t)
    e.run(None)
    first = e.results()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        e.run(torch.cuda.current_stream())
    for _ in range(2):
        for r in (e.x, e.p, e.y, e.dp, e.dx, e.dtable, e.dW, e.db, e.mean, e.rstd):
            r.fill_(55.0)
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(first, e.results()))
    e.table.mul_(0.5)
    e.ids.copy_(e.ids.flip(0))
    e.offsets[1:-1] = e.offsets[1:-1] // 2                # other groups, as the device has them at the replay
    graph.replay()
    replayed = e.results()
    e.run(None)
    assert all(torch.equal(a, b) for a, b in zip(replayed, e.results()))
    assert not torch.equal(first[2], replayed[2])


def test_two_streams_and_two_graphs_with_their_own_workspaces():
    es = [Encoder(20_000 + i, 400, 64, 96, 4, 8, torch.bfloat16, seed=i) for i in range(2)]
    for e in es:
        e.run(None)
    want = [e.results() for e in es]
    streams = [torch.cuda.Stream() for _ in es]
    torch.cuda.synchronize()
    graphs = []
    for e, s in zip(es, streams):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            e.run(torch.cuda.current_stream())
        graphs.append(g)
    for rep in range(4):
        for e in es:
            e.y.fill_(9.0), e.dtable.fill_(9.0), e.dW.fill_(9.0)
        torch.cuda.synchronize()
        for e, s, g in zip(es, streams, graphs):
            with torch.cuda.stream(s):
                e.run(s) if rep % 2 else g.replay()
        torch.cuda.synchronize()
        for e, w in zip(es, want):
            assert all(torch.equal(a, b) for a, b in zip(w, e.results()))


def test_rows_beyond_32_bits():
    """Rows whose elements lie beyond 2^31 elements and 2^32 bytes of their matrix: the last rows come out as they do in a small call."""
    n, d, t = (1 << 21) + 300, 1024, torch.bfloat16
    x = torch.randn(4096, d, device="cuda").to(t).repeat(n // 4096 + 1, 1)[:n].contiguous()
    W = (torch.randn(2, d, 64, device="cuda") / 32).to(t)
    off = torch.tensor([0, n - 500, n], device="cuda")
    out = torch.empty(n, 64, device="cuda")
    tb.typed_project(n, 2, off, x, d, W, None, d, 64, out, 64, None)
    small = torch.empty(500, 64, device="cuda")
    tb.typed_project(500, 1, torch.tensor([0, 500], device="cuda"), x[n - 500:], d, W[1:], None, d, 64, small, 64, None)
    assert torch.equal(out[n - 500:], small)
    dx = torch.empty(n, d, dtype=t, device="cuda")
    dy = torch.randn(n, 64, device="cuda").to(t)
    tb.typed_project_grad(n, 2, off, x, d, W, dy, 64, d, 64, dx, d, workspace=torch.empty(tb.typed_project_grad_workspace(n, 2, d, 64, t), dtype=torch.uint8, device="cuda"))
    sx = torch.empty(500, d, dtype=t, device="cuda")
    tb.typed_project_grad(500, 1, torch.tensor([0, 500], device="cuda"), x[n - 500:], d, W[1:], dy[n - 500:], 64, d, 64, sx, d,
                          workspace=torch.empty(tb.typed_project_grad_workspace(500, 1, d, 64, t), dtype=torch.uint8, device="cuda"))
    assert torch.equal(dx[n - 500:], sx)
    y = dx                                               # (reused)
    off = torch.tensor([0, n - 70_000, n - 300, n], device="cuda")
    tb.norm_rows(n, 3, off, x, d, d, 8, None, None, EPS, 1, y, d, None, None, torch.empty(tb.norm_rows_workspace(n, 3, d, 8), dtype=torch.uint8, device="cuda"))
    ref, _, _ = norm([0, 300], x[n - 300:], 8, None, None, EPS, 1)
    assert ((y[n - 300:].double() - ref).abs() <= 2.0 ** -8 * ref.abs() + 1e-5).all()
    ref, _, _ = norm([0, 69_700], x[n - 70_000:n - 300], 8, None, None, EPS, 1)
    assert ((y[n - 70_000:n - 300].double() - ref).abs() <= 2.0 ** -8 * ref.abs() + 1e-4).all()


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [40, 1000])
def test_columns_of_one_matrix(t, n):
    """Inputs and outputs that are neighbouring columns of one matrix give what matrices of their own give; columns that meet are refused."""
    g = torch.Generator("cuda").manual_seed(n)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")
    d, h, ids = 64, 96, torch.randint(0, 50, (n,), generator=g, device="cuda")
    table, W, off, dy = r(50, d).to(t), r(2, d, h).to(t), torch.tensor([0, n // 3, n], device="cuda"), r(n, h).to(t)
    ws = torch.empty(max(tb.embed_grad_workspace(n, 50, d), tb.typed_project_grad_workspace(n, 2, d, h, t), tb.norm_rows_grad_workspace(n, 2, h, 4)), dtype=torch.uint8, device="cuda")

    def run(x, p, y, dp, dx):
        mean, rstd, dtable = torch.empty(2, 4, device="cuda"), torch.empty(2, 4, device="cuda"), torch.empty_like(table)
        tb.embed_rows(n, ids, table, 50, d, d, x, x.stride(0))
        tb.typed_project(n, 2, off, x, x.stride(0), W, None, d, h, p, p.stride(0), ws)
        tb.norm_rows(n, 2, off, p, p.stride(0), h, 4, None, None, EPS, tb.ACT_SILU, y, y.stride(0), mean, rstd, ws)
        tb.norm_rows_grad(n, 2, off, p, p.stride(0), h, 4, None, None, tb.ACT_SILU, mean, rstd, dy, h, dp, dp.stride(0), None, None, ws)
        tb.typed_project_grad(n, 2, off, x, x.stride(0), W, dp, dp.stride(0), d, h, dx, dx.stride(0), workspace=ws)
        tb.embed_grad(n, ids, dx, dx.stride(0), d, dtable, 50, d, ws)
        return [v.clone() for v in (x, p, y, dp, dx, dtable)]

    own = run(*(torch.empty(n, w, dtype=t, device="cuda") for w in (d, h, h, h, d)))
    big = torch.full((n, 2 * d + 3 * h + 8), 7.0, dtype=t, device="cuda")
    at, cut = 0, []
    for w in (d, h, h, h, d):
        cut.append(big[:, at:at + w])
        at += w
    for a, b in zip(own, run(*cut)):
        assert torch.equal(a, b)
    assert (big[:, at:] == 7.0).all()
    x, p, over, first = cut[0], cut[1], big[:, d - 8:d - 8 + h], big[1:, :h]
    before = big.clone()
    for call in (lambda: tb.typed_project(n, 2, off, x, x.stride(0), W, None, d, h, over, over.stride(0), ws),
                 lambda: tb.embed_rows(n - 1, ids, over[:, :d], 50, d, over.stride(0), first[:, :d], first.stride(0)) if n > 50 else tb.embed_rows(
                     n, ids, over[:, :d], n, d, over.stride(0), x, x.stride(0)),
                 lambda: tb.norm_rows(n, 2, off, p, p.stride(0), h, 4, None, None, EPS, 0, over, over.stride(0), workspace=ws),
                 lambda: tb.norm_rows_grad(n, 2, off, p, p.stride(0), h, 4, None, None, 0, torch.zeros(2, 4, device="cuda"), torch.zeros(2, 4, device="cuda"), dy, h, over,
                                           over.stride(0), workspace=ws)):
        with pytest.raises(tb.TaurusError) as e:
            call()
        assert e.value.code == tb.ERROR_CODES["INVALID_ARG"]
    assert torch.equal(big, before)


def test_most_rows_of_one_type():
    """2^31 - 1 rows of one type: small whole numbers, whose products and sums fp32 holds (a sum of ones to its nearest value)."""
    n = (1 << 31) - 1
    x, out, off = torch.ones(n, 1, device="cuda"), torch.zeros(n, 1, device="cuda"), torch.tensor([0, 0, n], device="cuda")
    x[-1], x[1 << 30] = 5.0, 7.0
    W, b = torch.tensor([[[2.0]], [[3.0]]], device="cuda"), torch.tensor([[9.0], [1.0]], device="cuda")
    ws = torch.empty(tb.typed_project_grad_workspace(n, 2, 1, 1, x), dtype=torch.uint8, device="cuda")
    tb.typed_project(n, 2, off, x, 1, W, b, 1, 1, out, 1, ws)
    assert out[-1] == 16.0 and out[1 << 30] == 22.0 and out[0] == 4.0
    out[-1] = out[1 << 30] = 4.0
    assert (out == 4.0).all()
    x[-1] = x[1 << 30] = 1.0
    out.fill_(1.0)
    dW, db = torch.empty(2, 1, 1, device="cuda"), torch.empty(2, 1, device="cuda")
    dx = torch.empty_like(x)
    tb.typed_project_grad(n, 2, off, x, 1, W, out, 1, 1, 1, dx, 1, dW, db, ws)
    assert (dx == 3.0).all()
    assert dW.flatten().tolist() == [0.0, 2.0 ** 31] and db.flatten().tolist() == [0.0, 2.0 ** 31]


@pytest.mark.parametrize("stream", [None, "own"])
def test_a_norm_between_two_layers(stream):
    """A layer's dense output on the device, normed in place, is what the next layer's chunks are pushed from."""
    from dataclasses import replace
    w = replace(tg.scaled(tg.WORKLOADS["large"], 2_500, chunk=512, name="normed"), dims=(48, 96, 40), fanout=(0, 0), pool_slots=2_500, hub_count=5, mode=tg.SAGE_MEAN)
    g, m = tg.make_graph(w), tg.make_model(w, bias_scale=0.3)
    stream = torch.cuda.Stream() if stream else None
    r = torch.Generator("cuda").manual_seed(6)
    x = torch.randn(g.V, 48, generator=r, device="cuda")
    gamma, beta = 1 + 0.2 * torch.randn(96, generator=r, device="cuda"), 0.2 * torch.randn(96, generator=r, device="cuda")
    h, out = torch.empty(g.V, 96, device="cuda"), torch.empty(g.V, 40, device="cuda")
    off = torch.tensor([0, g.V // 3, g.V], device="cuda")      # (two graphs of a batch, for the norm)
    ws = torch.empty(tb.norm_rows_workspace(g.V, 2, 96, 8), dtype=torch.uint8, device="cuda")
    ctx = tb.Context(g.V, g.E, g.row_ptr, g.col_idx, g.in_degree, w.mode, w.dims, m.W_neigh, m.W_self, m.bias, m.act, w.chunk, w.pool_slots, w.hub_count, w.fanout, w.seed, 0, g.V)
    torch.cuda.synchronize()
    for l, (src, dst) in enumerate(((x, h), (h, out))):
        ctx.layer_begin(l, stream)
        ctx.layer_set_dense_output(dst, dst.shape[1])
        for b in range(0, g.V, w.chunk):
            ctx.push_chunk(b, min(b + w.chunk, g.V), src[b:b + w.chunk], stream)
        assert ctx.layer_end()["completed"] == g.V
        if l == 0:
            tb.norm_rows(g.V, 2, off, h, 96, 96, 8, gamma, beta, EPS, tb.ACT_SILU, h, 96, workspace=ws, stream=stream)
    torch.cuda.synchronize()

    def layer(l, x):
        agg = np.zeros_like(x)
        for u in range(g.V):
            np.add.at(agg, g.col_idx[g.row_ptr[u]:g.row_ptr[u + 1]], x[u])
        agg /= np.maximum(g.in_degree, 1)[:, None]
        y = agg @ m.W_neigh[l].astype(np.float64) + x @ m.W_self[l].astype(np.float64) + m.bias[l]
        return np.maximum(y, 0) if m.act[l] else y
    y, _, _ = norm(off.tolist(), torch.from_numpy(layer(0, x.double().cpu().numpy())).cuda(), 8, gamma, beta, EPS, tb.ACT_SILU)
    assert float((h.double() - y).norm()) <= 1e-4 * float(y.norm())
    want = layer(1, y.cpu().numpy())
    assert np.linalg.norm(out.double().cpu().numpy() - want) <= 1e-4 * np.linalg.norm(want)


@pytest.mark.parametrize("most,n", [(606_300, 606_207), (310_000, 308_223), (300_000, 150_000)])
def test_a_workspace_asked_for_once(most, n):
    """A workspace of the largest batch's size takes a smaller batch, whose pieces, chunks or blocks may be more than the largest one's."""
    ids = torch.randint(-1, 900, (n,), device="cuda")
    grad, table = torch.ones(n, 8, device="cuda"), torch.empty(900, 8, device="cuda")
    tb.embed_grad(n, ids, grad, 8, 8, table, 900, 8, torch.full((tb.embed_grad_workspace(most, 900, 8),), 255, dtype=torch.uint8, device="cuda"))
    assert torch.equal(table[:, 3], torch.bincount(ids[ids >= 0], minlength=900).float())
    x, W = torch.ones(n, 72, dtype=torch.bfloat16, device="cuda"), torch.ones(3, 72, 40, dtype=torch.bfloat16, device="cuda")
    dy, dW, off = torch.ones(n, 40, dtype=torch.bfloat16, device="cuda"), torch.empty(3, 72, 40, device="cuda"), torch.tensor([0, 1000, 1000, n], device="cuda")
    tb.typed_project_grad(n, 3, off, x, 72, W, dy, 40, 72, 40, grad_W=dW,
                          workspace=torch.full((tb.typed_project_grad_workspace(most, 3, 72, 40, x),), 255, dtype=torch.uint8, device="cuda"))
    assert dW[:, 5, 7].tolist() == [1000.0, 0.0, n - 1000.0]
    graphs = n // 3
    off = torch.cat([torch.arange(graphs, device="cuda") * 3, torch.tensor([n], device="cuda")])
    y, g, mean, rstd = torch.randn(n, 16, device="cuda"), torch.empty(n, 16, device="cuda"), torch.empty(graphs, 1, device="cuda"), torch.empty(graphs, 1, device="cuda")
    ws = torch.full((max(tb.norm_rows_workspace(most, graphs, 16, 1), tb.norm_rows_grad_workspace(most, graphs, 16, 1)),), 255, dtype=torch.uint8, device="cuda")
    tb.norm_rows(n, graphs, off, y, 16, 16, 1, None, None, EPS, 0, g, 16, mean, rstd, ws)
    assert float(g[:3].mean().abs()) < 1e-6
    tb.norm_rows_grad(n, graphs, off, y, 16, 16, 1, None, None, 0, mean, rstd, y, 16, g, 16, workspace=ws)
    assert torch.isfinite(g).all()
