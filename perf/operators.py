"""Operators that stand before and between the layers of a graph network, as cases that can be timed.

embed         rows of a learned table, looked up by id and scaled (vertices without features of their own)
embed_grad    the gradient of that table
typed         one weight matrix per vertex type: rows grouped by type, ragged groups
typed_grad    gradients of the rows, of the weights and of the bias
norm          group norm with an activation over the rows of a batch of graphs, channels last
norm_train    the same with its gradients: a forward and a backward call

Where `own` is false `run` computes them from elementary torch operations in 32 bits; where it is true it makes the calls of
this library.  Ids follow a power law as degrees do, some are -1 (no entry); group and graph sizes are ragged, some empty.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
ACTS = {"none": 0, "relu": 1, "silu": 2}
EPS = 1e-5


def _embed(name, n, rows, width, type="f32", out="f32", grad=False):
    c = dict(kind="embed_grad" if grad else "embed", n=n, rows=rows, width=width, type=type, out=out)
    return dict(c, name=name) if name else c


def _typed(name, n, types, d_in, d_out, type="f32", out="f32", grad=False, bias=True):
    """out: type of the product (forward), of the weights' gradient (gradient)."""
    c = dict(kind="typed_grad" if grad else "typed", n=n, types=types, d_in=d_in, d_out=d_out, type=type, out=out, bias=bias)
    return dict(c, name=name) if name else c


def _norm(name, n, graphs, width, groups, type="f32", act="relu", train=False):
    c = dict(kind="norm_train" if train else "norm", n=n, graphs=graphs, width=width, groups=groups, type=type, act=act)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the row of one vertex that a query asks for: latency
        _embed("embed_one", 1, 10_000, 64),
        # a chunk of sources of the "mid" workload whose rows come from a table
        _embed("embed_chunk", 65_536, 2_450_000, 100),
        # every vertex of a large graph, table kept in 16 bits, rows of the "stress" width
        _embed("embed_graph_bf16", 1_200_000, 600_000, 512, "bf16"),
        # gradient of a table over one training batch with hubs
        _embed("embed_grad_hubs", 500_000, 400_000, 128, grad=True),
        # gradient of a small table of categories: odd width, few rows, many ids each
        _embed("embed_grad_categories", 120_001, 1_003, 47, "bf16", "bf16", grad=True),
        # vertices of one query, each with the weights of its type
        _typed("typed_few", 5, 8, 100, 256, "bf16", "bf16"),
        # the "gin_drain_ragged" sizes: odd widths, fp32 rows
        _typed("typed_ragged", 120_001, 7, 37, 130),
        # all vertices of a large heterogeneous graph, "stress" widths
        _typed("typed_graph_bf16", 1_200_000, 16, 512, 256, "bf16", "bf16"),
        # a training batch in fp32, "mid" widths, and one of many small types in fp16
        _typed("typed_grad_batch", 400_000, 5, 100, 256, grad=True),
        _typed("typed_grad_many_f16", 65_536, 200, 128, 128, "f16", "f32", grad=True),
        # a batch of small graphs
        _norm("norm_batch_bf16", 262_144, 9_001, 64, 8, "bf16", "silu"),
        # one large graph, a training step
        _norm("norm_train_graph", 1_000_000, 3, 256, 16, act="silu", train=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))


def draw(rng):
    kind = rng.choice(["embed", "embed_grad", "typed", "typed_grad", "norm", "norm_train"])
    type = rng.choice(list(TYPES))
    if kind.startswith("embed"):
        width = _log(rng, 1, 1024)
        n = _log(rng, 1, min(1_200_000, 500_000_000 // width))
        rows = _log(rng, 1, min(2_450_000, 250_000_000 // width))
        return _embed(None, n, rows, width, type, rng.choice(["f32", type]), kind == "embed_grad")
    if kind.startswith("typed"):
        d_in, d_out = _log(rng, 1, 1024), _log(rng, 1, 1024)
        cost = 450_000_000 if type == "f32" or kind == "typed_grad" else 900_000_000
        n = _log(rng, 1, min(1_200_000, cost // (d_in + d_out), cost * 60 // (d_in * d_out)))
        types = _log(rng, 1, max(1, min(1000, 100_000_000 // (d_in * d_out))))
        return _typed(None, n, types, d_in, d_out, type, rng.choice(["f32", type]), kind == "typed_grad", rng.random() < 0.7)
    per_group, groups = _log(rng, 1, 64), _log(rng, 1, 32)
    if per_group * groups > 1024:
        groups = 1024 // per_group
    n = _log(rng, 1, min(1_000_000, 250_000_000 // (per_group * groups)))
    # ReLU's slope jumps: what an element right at the border gets as its gradient says nothing, so training cases leave it out
    act = rng.choice(["none", "silu"] if kind == "norm_train" else list(ACTS))
    return _norm(None, n, _log(rng, 1, min(n, 50_000)), per_group * groups, groups, type, act, kind == "norm_train")


def _sizes(total, parts, g):
    """Ragged sizes that add up to total: shares spread over two orders of magnitude, one part in eight empty."""
    share = torch.exp(torch.rand(parts, generator=g, dtype=torch.float64) * 4.6)
    share[torch.rand(parts, generator=g, dtype=torch.float64) < 0.125] = 0
    if float(share.sum()) == 0:
        share[0] = 1
    ends = torch.floor(torch.cumsum(share, 0) / share.sum() * total + 0.5).to(torch.int64)
    ends[-1] = total
    return torch.cat([torch.zeros(1, dtype=torch.int64), ends])


def _inputs(case, seed):
    c = case
    g = torch.Generator().manual_seed(seed)
    d = torch.Generator("cuda").manual_seed(seed + 1)
    t = TYPES[c["type"]]

    def normal(*shape):
        return torch.randn(*shape, generator=d, device="cuda")

    s = {}
    if c["kind"].startswith("embed"):
        u = torch.rand(c["n"], generator=d, device="cuda", dtype=torch.float64)
        rank = (u ** 3 * c["rows"]).to(torch.int64).clamp_(max=c["rows"] - 1)
        step = 7919 if c["rows"] % 7919 else 7907
        ids = rank * step % c["rows"]                      # popular ids lie anywhere in the table
        ids[torch.rand(c["n"], generator=d, device="cuda") < 0.02] = -1
        s["ids"] = ids
        s["scale"] = math.sqrt(c["width"])
        if c["kind"] == "embed":
            s["table"] = (normal(c["rows"], c["width"]) * 0.02).to(t)
        else:
            s["grad"] = (normal(c["n"], c["width"]) * 1e-2).to(TYPES[c["out"]])
    elif c["kind"].startswith("typed"):
        off = _sizes(c["n"], c["types"], g)
        s["host_offsets"], s["offsets"] = off.tolist(), off.cuda()
        s["x"] = normal(c["n"], c["d_in"]).to(t)
        bound = math.sqrt(6.0 / (c["d_in"] + c["d_out"]))
        s["W"] = ((torch.rand(c["types"], c["d_in"], c["d_out"], generator=d, device="cuda") * 2 - 1) * bound).to(t)
        if c["kind"] == "typed":
            s["bias"] = normal(c["types"], c["d_out"]) * 0.1 if c["bias"] else None
        else:
            s["grad"] = (normal(c["n"], c["d_out"]) * 1e-2).to(t)
    else:
        off = _sizes(c["n"], c["graphs"], g)
        s["host_offsets"], s["offsets"] = off.tolist(), off.cuda()
        s["x"] = (normal(c["n"], c["width"]) * (0.5 + torch.rand(c["width"], generator=d, device="cuda")) + normal(c["width"]) * 0.5).to(t)
        s["gamma"] = 1 + 0.1 * normal(c["width"])
        s["beta"] = 0.1 * normal(c["width"])
        if c["kind"] == "norm_train":
            s["grad"] = (normal(c["n"], c["width"]) * 1e-2).to(t)
    return s


def prepare(case, seed):
    c = case
    s = _inputs(c, seed)
    s["case"] = c
    if not own:
        return s
    import paper_2607_17374_b200 as tb
    t, o = TYPES[c["type"]], TYPES[c["out"]] if "out" in c else None

    def empty(*shape, dtype):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    if c["kind"] == "embed":
        s["rows"], size = empty(c["n"], c["width"], dtype=o), 0
    elif c["kind"] == "embed_grad":
        s["grad_table"] = empty(c["rows"], c["width"], dtype=t)
        size = tb.embed_grad_workspace(c["n"], c["rows"], c["width"])
    elif c["kind"] == "typed":
        s["rows"] = empty(c["n"], c["d_out"], dtype=o)
        size = tb.typed_project_workspace(c["n"], c["types"], c["d_in"], c["d_out"], t)
    elif c["kind"] == "typed_grad":
        s["grad_x"], s["grad_W"] = empty(c["n"], c["d_in"], dtype=t), empty(c["types"], c["d_in"], c["d_out"], dtype=o)
        s["grad_bias"] = empty(c["types"], c["d_out"], dtype=torch.float32) if c["bias"] else None
        size = tb.typed_project_grad_workspace(c["n"], c["types"], c["d_in"], c["d_out"], t)
    else:
        s["rows"] = empty(c["n"], c["width"], dtype=t)
        size = tb.norm_rows_workspace(c["n"], c["graphs"], c["width"], c["groups"])
        if c["kind"] == "norm_train":
            s["mean"], s["rstd"] = (empty(c["graphs"], c["groups"], dtype=torch.float32) for _ in range(2))
            s["grad_x"] = empty(c["n"], c["width"], dtype=t)
            s["grad_gamma"], s["grad_beta"] = (empty(c["width"], dtype=torch.float32) for _ in range(2))
            size = max(size, tb.norm_rows_grad_workspace(c["n"], c["graphs"], c["width"], c["groups"]))
    s["workspace"] = empty(size, dtype=torch.uint8) if size else None
    s["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    return s


def _run_own(s):
    import paper_2607_17374_b200 as tb
    c = s["case"]
    st = dict(status=s["status"], stream=torch.cuda.current_stream())
    if c["kind"] == "embed":
        tb.embed_rows(c["n"], s["ids"], s["table"], c["rows"], c["width"], c["width"], s["rows"], c["width"], s["scale"], **st)
        return s["rows"]
    if c["kind"] == "embed_grad":
        tb.embed_grad(c["n"], s["ids"], s["grad"], c["width"], c["width"], s["grad_table"], c["rows"], c["width"], s["workspace"], s["scale"], **st)
        return s["grad_table"]
    if c["kind"] == "typed":
        tb.typed_project(c["n"], c["types"], s["offsets"], s["x"], c["d_in"], s["W"], s["bias"], c["d_in"], c["d_out"], s["rows"], c["d_out"],
                         s["workspace"], **st)
        return s["rows"]
    if c["kind"] == "typed_grad":
        tb.typed_project_grad(c["n"], c["types"], s["offsets"], s["x"], c["d_in"], s["W"], s["grad"], c["d_out"], c["d_in"], c["d_out"],
                              s["grad_x"], c["d_in"], s["grad_W"], s["grad_bias"], s["workspace"], **st)
        return [s["grad_x"], s["grad_W"], s["grad_bias"]] if c["bias"] else [s["grad_x"], s["grad_W"]]
    train = c["kind"] == "norm_train"
    tb.norm_rows(c["n"], c["graphs"], s["offsets"], s["x"], c["width"], c["width"], c["groups"], s["gamma"], s["beta"], EPS, ACTS[c["act"]],
                 s["rows"], c["width"], s["mean"] if train else None, s["rstd"] if train else None, s["workspace"], **st)
    if not train:
        return s["rows"]
    tb.norm_rows_grad(c["n"], c["graphs"], s["offsets"], s["x"], c["width"], c["width"], c["groups"], s["gamma"], s["beta"], ACTS[c["act"]],
                      s["mean"], s["rstd"], s["grad"], c["width"], s["grad_x"], c["width"], s["grad_gamma"], s["grad_beta"], s["workspace"], **st)
    return [s["rows"], s["grad_x"], s["grad_gamma"], s["grad_beta"]]


def _graph_of_rows(s, n):
    off = s["offsets"]
    return torch.bucketize(torch.arange(n, device="cuda"), off[1:], right=True)


def run(state):
    if own:
        return _run_own(state)
    s = state
    c = s["case"]
    t = TYPES[c["type"]]
    if c["kind"] == "embed":
        rows = s["table"][s["ids"].clamp(min=0)].float() * s["scale"]
        return torch.where((s["ids"] >= 0)[:, None], rows, 0.0).to(TYPES[c["out"]])
    if c["kind"] == "embed_grad":
        # long sums, so in 64 bits; -1 is a row behind the table's
        out = torch.zeros(c["rows"] + 1, c["width"], dtype=torch.float64, device="cuda")
        out.index_add_(0, torch.where(s["ids"] < 0, c["rows"], s["ids"]), s["grad"].double())
        return (out[:-1] * s["scale"]).to(t)
    if c["kind"].startswith("typed"):
        o = s["host_offsets"]
        x, W = s["x"].float(), s["W"].float()
        if c["kind"] == "typed":
            out = torch.empty(c["n"], c["d_out"], dtype=torch.float32, device="cuda")
            for g in range(c["types"]):
                if o[g + 1] > o[g]:
                    y = x[o[g]:o[g + 1]] @ W[g]
                    out[o[g]:o[g + 1]] = y + s["bias"][g] if c["bias"] else y
            return out.to(TYPES[c["out"]])
        dy = s["grad"].float()
        dx, dW = torch.empty_like(x), torch.zeros_like(W)
        db = torch.zeros(c["types"], c["d_out"], device="cuda")
        for g in range(c["types"]):
            if o[g + 1] > o[g]:
                part = dy[o[g]:o[g + 1]]
                dx[o[g]:o[g + 1]] = part @ W[g].T
                dW[g] = x[o[g]:o[g + 1]].T @ part
                db[g] = part.sum(0)
        return [dx.to(t), dW.to(TYPES[c["out"]]), db] if c["bias"] else [dx.to(t), dW.to(TYPES[c["out"]])]
    # norm: sums by graph of 32-bit rows, in 64 bits
    n, C, G = c["n"], c["width"], c["groups"]
    seg = _graph_of_rows(s, n)
    x = s["x"].float().view(n, G, C // G)
    count = ((s["offsets"][1:] - s["offsets"][:-1]) * (C // G)).double().clamp(min=1)[:, None]

    def by_graph(rows):
        if c["graphs"] <= 64:
            o = s["host_offsets"]
            return torch.stack([rows[b:e].sum(0, dtype=torch.float64) for b, e in zip(o, o[1:])])
        return torch.zeros(c["graphs"], G, dtype=torch.float64, device="cuda").index_add_(0, seg, rows.double())

    mean = (by_graph(x.sum(2)) / count).float()
    centred = x - mean[seg][:, :, None]
    rstd = torch.rsqrt(by_graph((centred * centred).sum(2)) / count + EPS).float()
    xh = centred * rstd[seg][:, :, None]
    gamma, beta = s["gamma"].view(G, C // G), s["beta"].view(G, C // G)
    z = xh * gamma + beta
    if c["act"] == "relu":
        y, slope = torch.where(z > 0, z, 0.0), (z > 0).float()
    elif c["act"] == "silu":
        sg = 1 / (1 + torch.exp(-z))
        y, slope = z * sg, sg * (1 + z * (1 - sg))
    else:
        y, slope = z, torch.ones_like(z)
    y = y.reshape(n, C).to(t)
    if c["kind"] == "norm":
        return y
    dz = s["grad"].float().view(n, G, C // G) * slope
    dgamma = (dz * xh).sum(0, dtype=torch.float64).reshape(C).float()
    dbeta = dz.sum(0, dtype=torch.float64).reshape(C).float()
    dxh = dz * gamma
    m1 = (by_graph(dxh.sum(2)) / count).float()[seg][:, :, None]
    m2 = (by_graph((dxh * xh).sum(2)) / count).float()[seg][:, :, None]
    dx = (dxh - m1 - xh * m2) * rstd[seg][:, :, None]
    return [y, dx.reshape(n, C).to(t), dgamma, dbeta]


def exact(case, seed):
    """The definitions in 64 bits, a graph / type / block of rows at a time."""
    c = case
    s = _inputs(c, seed)
    if c["kind"] == "embed":
        table = torch.cat([s["table"].double() * s["scale"], torch.zeros(1, c["width"], dtype=torch.float64, device="cuda")])
        return table[s["ids"]]                                            # -1 is the row of zeros at the end
    if c["kind"] == "embed_grad":
        # sorted ids, running sums, their differences at the ends of the segments
        ids, order = torch.sort(s["ids"], stable=True)
        first = torch.searchsorted(ids, torch.arange(c["rows"] + 1, device="cuda"))
        sums = torch.zeros(c["width"], c["n"] + 1, dtype=torch.float64, device="cuda")
        torch.cumsum(s["grad"][order].T.double(), 1, out=sums[:, 1:])
        return (sums[:, first[1:]] - sums[:, first[:-1]]).T * s["scale"]
    o = s["host_offsets"]
    spans = [(g, o[g], o[g + 1]) for g in range(len(o) - 1) if o[g + 1] > o[g]]
    if c["kind"] == "typed":
        out = torch.zeros(c["n"], c["d_out"], dtype=torch.float64, device="cuda")
        for g, b, e in spans:
            torch.matmul(s["x"][b:e].double(), s["W"][g].double(), out=out[b:e])
            if c["bias"]:
                out[b:e] += s["bias"][g].double()
        return out
    if c["kind"] == "typed_grad":
        dx = torch.zeros(c["n"], c["d_in"], dtype=torch.float64, device="cuda")
        dW = torch.zeros(c["types"], c["d_in"], c["d_out"], dtype=torch.float64, device="cuda")
        db = torch.zeros(c["types"], c["d_out"], dtype=torch.float64, device="cuda")
        for g, b, e in spans:
            dy = s["grad"][b:e].double()
            dx[b:e] = torch.einsum("rn,kn->rk", dy, s["W"][g].double())
            dW[g] = torch.einsum("rk,rn->kn", s["x"][b:e].double(), dy)
            db[g] = torch.einsum("rn->n", dy)
        return [dx, dW, db] if c["bias"] else [dx, dW]
    if len(spans) > 60_000:
        return None                                                      # a loop over graphs would take too long
    C, G = c["width"], c["groups"]
    gamma, beta = s["gamma"].double(), s["beta"].double()
    train = c["kind"] == "norm_train"
    y = torch.zeros(c["n"], C, dtype=torch.float64, device="cuda")
    dx, dgamma, dbeta = torch.zeros_like(y) if train else None, torch.zeros_like(gamma), torch.zeros_like(gamma)
    for _, b, e in spans:
        x = s["x"][b:e].double().reshape(e - b, G, -1)
        var, mean = torch.var_mean(x, dim=(0, 2), correction=0, keepdim=True)
        inv = (var + EPS) ** -0.5
        xh = ((x - mean) * inv).reshape(e - b, C)
        z = xh * gamma + beta
        gate = torch.sigmoid(z) if c["act"] == "silu" else (z > 0).double() if c["act"] == "relu" else None
        y[b:e] = z if gate is None else z * gate
        if train:
            dz = s["grad"][b:e].double()
            if gate is not None:
                dz = dz * (gate + z * gate * (1 - gate))                  # relu: gate is 0 or 1
            dgamma += (dz * xh).sum(0)
            dbeta += dz.sum(0)
            h, xg = (dz * gamma).reshape(e - b, G, -1), xh.reshape(e - b, G, -1)
            dx[b:e] = (inv * (h - h.mean((0, 2), keepdim=True) - xg * (h * xg).mean((0, 2), keepdim=True))).reshape(e - b, C)
    return [y, dx, dgamma, dbeta] if train else y


def work(case):
    c = case
    t = SIZE[c["type"]]
    if c["kind"] == "embed":
        return {"bytes": c["n"] * (8 + c["width"] * SIZE[c["out"]]) + min(c["n"], c["rows"]) * c["width"] * t, "flops": c["n"] * c["width"]}
    if c["kind"] == "embed_grad":
        return {"bytes": c["n"] * (8 + c["width"] * SIZE[c["out"]]) + c["rows"] * c["width"] * t, "flops": c["n"] * c["width"]}
    if c["kind"].startswith("typed"):
        n, k, m, g = c["n"], c["d_in"], c["d_out"], c["types"]
        weights = min(g, n) * k * m
        if c["kind"] == "typed":
            return {"bytes": n * (k * t + m * SIZE[c["out"]]) + weights * t + 8 * g, "flops": 2 * n * k * m}
        return {"bytes": n * (2 * k + m) * t + weights * t + g * k * m * SIZE[c["out"]] + 4 * g * m, "flops": 4 * n * k * m}
    e = c["n"] * c["width"]
    if c["kind"] == "norm":
        return {"bytes": 2 * e * t + 8 * c["graphs"], "flops": 8 * e}
    return {"bytes": 5 * e * t + 8 * c["graphs"] * (1 + c["groups"]), "flops": 24 * e}
