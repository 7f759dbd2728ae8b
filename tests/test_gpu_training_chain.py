"""One training step of an encoder with a classifier, through the operators as they would be used together: lookup, products by type, the residual norm, the loss and its gradient,
the gradients back to the table, AdamW.  Its gradients against fp64, and captured as a graph."""
import pytest
import torch

import paper_2607_17374_b200 as tb

pytestmark = pytest.mark.gpu
F32 = torch.float32
B1, B2, ADAM_EPS, EPS = 0.9, 0.999, 1e-8, 1e-5


class Net:
    """rows = table[ids]; x = rows W1; b = x W2 + b2; r = x + alpha gate[type] norm(b) post; y = norm(r) gamma + beta; logits = y W3 + b3."""

    def __init__(self, eight=False, n=3000, types=4, rows=500, d0=32, d=48, classes=20):
        g = torch.Generator("cuda").manual_seed(11)

        def normal(*shape, scale=1.0, base=0.0):
            return base + scale * torch.randn(*shape, generator=g, device="cuda")

        self.n, self.types, self.rows, self.d0, self.d, self.classes, self.alpha = n, types, rows, d0, d, classes, 0.5
        self.p = dict(table=normal(rows, d0), W1=normal(types, d0, d, scale=d0 ** -0.5), W2=normal(types, d, d, scale=d ** -0.5), b2=normal(types, d, scale=0.1), gate=normal(types, d, scale=0.3, base=0.7),
                      post=normal(d, scale=0.1, base=1), gamma=normal(d, scale=0.1, base=1), beta=normal(d, scale=0.1), W3=normal(types, d, classes, scale=d ** -0.5), b3=normal(types, classes, scale=0.1))
        self.ids = torch.randint(0, rows, (n,), generator=g, device="cuda")
        self.ids[torch.rand(n, generator=g, device="cuda") < 0.05] = -1
        self.labels = torch.randint(0, classes, (n,), generator=g, device="cuda")
        self.labels[torch.rand(n, generator=g, device="cuda") < 0.3] = -1
        self.off = [0, 700, 700, 2500, n]
        self.offsets = torch.tensor(self.off, device="cuda")
        self.weight = torch.full((n,), -1.0 / int((self.labels >= 0).sum()), device="cuda")       # the mean of -log p over the rows with a label
        self.grads = {k: torch.zeros_like(v) for k, v in self.p.items()}

        def empty(*shape, dtype=F32):
            return torch.empty(*shape, dtype=dtype, device="cuda")

        self.x0, self.x, self.b, self.r, self.y, self.logits = empty(n, d0), empty(n, d), empty(n, d), empty(n, d), empty(n, d), empty(n, classes)
        self.dlogits, self.dy, self.dx, self.db, self.dxb, self.dx0 = empty(n, classes), empty(n, d), empty(n, d), empty(n, d), empty(n, d), empty(n, d0)
        self.stats, self.logprob, self.entropy, self.lstats = empty(n, 4), empty(n), empty(n), empty(n, 2)
        space = max(tb.typed_project_workspace(n, types, d, d, F32), tb.typed_project_grad_workspace(n, types, d, d, F32), tb.typed_project_grad_workspace(n, types, d, classes, F32),
                    tb.typed_project_grad_workspace(n, types, d0, d, F32), tb.typed_project_workspace(n, types, d0, d, F32), tb.typed_project_workspace(n, types, d, classes, F32),
                    tb.embed_grad_workspace(n, rows, d0), tb.residual_norm_grad_workspace(n, d, types), tb.class_logprob_workspace(n, classes))
        self.ws = empty(space, dtype=torch.uint8)
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        names = list(self.p)
        flat = [self.p[k].view(-1) for k in names]
        kind = torch.float8_e4m3fn if eight else F32
        self.m, self.v = ([torch.zeros(len(x), dtype=kind, device="cuda") for x in flat] for _ in range(2))
        scales = [[torch.zeros(-(-len(x) // tb.STATE_BLOCK), device="cuda") for x in flat] for _ in range(2)] if eight else [None, None]
        self.adamw = tb.AdamW(flat, [self.grads[k].view(-1) for k in names], self.m, self.v, *scales, weight_decay=[0.01 if k[0] in "tW" else 0.0 for k in names])
        self.count, self.lr = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.full((1,), 5e-3, device="cuda")

    def gradients(self, stream=None):
        p, g, n, t, d0, d, c = self.p, self.grads, self.n, self.types, self.d0, self.d, self.classes
        st = dict(status=self.status, stream=stream)
        tb.embed_rows(n, self.ids, p["table"], self.rows, d0, d0, self.x0, d0, **st)
        tb.typed_project(n, t, self.offsets, self.x0, d0, p["W1"], None, d0, d, self.x, d, self.ws, **st)
        tb.typed_project(n, t, self.offsets, self.x, d, p["W2"], p["b2"], d, d, self.b, d, self.ws, **st)
        norm = (n, d, self.x, d, self.b, d, tb.NORM_LAYER, True, p["post"], t, self.offsets, p["gate"], self.alpha, p["gamma"])
        tb.residual_norm(*norm, p["beta"], EPS, self.r, d, self.y, d, self.stats, **st)
        tb.typed_project(n, t, self.offsets, self.y, d, p["W3"], p["b3"], d, c, self.logits, c, self.ws, **st)
        tb.class_logprob_train(n, c, self.logits, c, self.labels, self.weight, None, self.logprob, self.entropy, self.lstats, self.dlogits, c, self.ws, **st)
        tb.typed_project_grad(n, t, self.offsets, self.y, d, p["W3"], self.dlogits, c, d, c, self.dy, d, g["W3"], g["b3"], self.ws, **st)
        tb.residual_norm_grad(*norm, self.stats, None, d, self.dy, d, self.dx, d, self.db, d, g["post"], g["gate"], g["gamma"], g["beta"], self.ws, **st)
        tb.typed_project_grad(n, t, self.offsets, self.x, d, p["W2"], self.db, d, d, d, self.dxb, d, g["W2"], g["b2"], self.ws, **st)
        self.dx += self.dxb
        tb.typed_project_grad(n, t, self.offsets, self.x0, d0, p["W1"], self.dx, d, d0, d, self.dx0, d0, g["W1"], None, self.ws, **st)
        tb.embed_grad(n, self.ids, self.dx0, d0, d0, g["table"], self.rows, d0, self.ws, **st)

    def step(self, stream=None):
        self.gradients(stream)
        self.count += 1
        self.adamw.step(self.count, self.lr, B1, B2, ADAM_EPS, None, 21, self.status, stream)

    def reference(self):
        p = {k: v.double().requires_grad_() for k, v in self.p.items()}
        x0 = torch.where((self.ids >= 0)[:, None], p["table"][self.ids.clamp(min=0)], 0.0)
        typ = torch.repeat_interleave(torch.arange(self.types, device="cuda"), self.offsets.diff())

        def typed(x, W, bias=None):
            parts = [x[b:e] @ W[i] + (0 if bias is None else bias[i]) for i, (b, e) in enumerate(zip(self.off, self.off[1:]))]
            return torch.cat(parts)

        def norm(z):
            return (z - z.mean(1, keepdim=True)) / torch.sqrt(z.var(1, correction=0, keepdim=True) + EPS)

        x = typed(x0, p["W1"])
        r = x + self.alpha * p["gate"][typ] * norm(typed(x, p["W2"], p["b2"])) * p["post"]
        logp = torch.log_softmax(typed(norm(r) * p["gamma"] + p["beta"], p["W3"], p["b3"]), 1)
        given = self.labels >= 0
        loss = -logp[given, self.labels[given]].mean()
        loss.backward()
        return float(loss), {k: v.grad for k, v in p.items()}


def test_gradients_of_a_step():
    net = Net()
    net.gradients()
    loss, ref = net.reference()
    assert int(net.status) == 0
    got = float((net.logprob.double() * net.weight.double()).sum())
    # Nine operators one behind the other, each off by less than 200 roundings of its terms (rows of 48, sums over up to 2 100 rows in chains of less than 200): 1 800 u = 1.1e-4 of
    # the terms' size; terms of a sum cancel to a third of it at most in the norms compared here
    assert abs(got - loss) < 3.3e-4 * loss
    for k in ref:
        assert float((net.grads[k].double() - ref[k]).norm() / ref[k].norm()) < 3.3e-4, k


@pytest.mark.parametrize("eight", [False, True])
def test_steps_captured_as_a_graph_are_the_eager_ones(eight):
    a, b = Net(eight), Net(eight)
    b.step()                                          # (loads what a first call loads)
    torch.cuda.synchronize()
    b = Net(eight)
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=stream):
        b.step(stream)
    for _ in range(4):
        a.step()
        graph.replay()
    torch.cuda.synchronize()
    assert int(a.count) == int(b.count) == 4 and int(a.status) == 0 and int(b.status) == 0
    for k in a.p:
        assert torch.equal(a.p[k], b.p[k]), k
    assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a.m + a.v, b.m + b.v))


def test_two_nets_on_two_streams():
    """Calls that may run at the same time, each with a workspace of its own, give what they give alone."""
    alone = Net()
    for _ in range(3):
        alone.step()
    torch.cuda.synchronize()
    nets, streams = [Net(), Net()], [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(3):
        for net, s in zip(nets, streams):
            with torch.cuda.stream(s):
                net.step(s)
    torch.cuda.synchronize()
    for net in nets:
        assert all(torch.equal(net.p[k], alone.p[k]) for k in alone.p)


def test_an_answer_with_alternatives():
    """The same logits, answered: the label's log probability, the entropy and the best classes of each row."""
    net = Net()
    net.gradients()
    n, c = net.n, net.classes
    lp, H, top, cls = torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty(n, 3, device="cuda"), torch.empty(n, 3, dtype=torch.int64, device="cuda")
    tb.class_logprob(n, c, net.logits, c, net.labels, lp, H, None, 3, top, cls)
    assert torch.equal(lp, net.logprob) and torch.equal(H, net.entropy)
    want = torch.sort(net.logits, dim=1, descending=True, stable=True)
    assert torch.equal(cls, want.indices[:, :3])
    logp = torch.log_softmax(net.logits.double(), 1)
    assert (top.double() - logp.gather(1, cls)).abs().max() < 1e-5        # log p of at most 20, off by 2 u of it, the sum's logarithm by 30 u
