"""The rest of a program that trains an encoder on typed rows and answers with it, as cases that can be timed.

logprob         log probabilities of given classes with entropy and top alternatives, from rows of logits
logprob_train   the same with the gradient of the logits, in one call where the loss's weights of the rows are known ahead, else in two
block           norms before and after a block, fused with its gate by type and its residual scale
block_train     the same with its gradients
adamw           one AdamW step over many tensors, states in 32 bits or in 8

Where `own` is false `run` computes them from elementary torch operations in 32 bits; where it is true it makes the calls of this
library.  Some rows have no label, some classes (and a few rows wholly) are masked with -inf; groups of rows and sizes of tensors are
ragged, some empty; a part of the gradients is zero, as for rows of a table that no id named.
"""
import math
import random

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-5
BETA1, BETA2, ADAM_EPS, DECAY = 0.9, 0.999, 1e-8, 0.01
BLOCK = 256                      # elements that share a scale of the 8-bit states


def _named(name, c):
    return dict(c, name=name) if name else c


def _logprob(name, n, classes, type="f32", k=0, masked=False, train=False, late=False):
    """late: what the rows weigh in the loss is known after their log probabilities only."""
    return _named(name, dict(kind="logprob_train" if train else "logprob", n=n, classes=classes, type=type, k=k, masked=masked, late=late))


def _block(name, n, width, type="f32", res="f32", groups=1, layer=True, post=True, train=False):
    """res: type of the residual rows; groups: types of rows with a gate of their own, 0: no gate."""
    return _named(name, dict(kind="block_train" if train else "block", n=n, width=width, type=type, res=res, groups=groups, layer=layer, post=post))


def _adamw(name, tensors, total, type="f32", grad="f32", bits=32, master=False, step=100):
    return _named(name, dict(kind="adamw", tensors=tensors, total=total, type=type, grad=grad, bits=bits, master=master, step=step))


def listed():
    return [
        # the answer for one vertex: latency
        _logprob("answer_one", 1, 172, k=5),
        # every vertex of a graph, few classes
        _logprob("answer_graph", 1_200_000, 47, k=3),
        # a batch of queries against all items of a catalogue, odd width, a part of the items not allowed
        _logprob("answer_items_bf16", 2_000, 120_001, "bf16", k=10, masked=True),
        # three queries against a large catalogue
        _logprob("answer_few_f16", 3, 250_000, "f16", k=16),
        # the loss over one training batch and its gradient
        _logprob("loss_batch_bf16", 400_000, 172, "bf16", train=True),
        # the rows of one query between two layers
        _block("block_few", 5, 256, "bf16", "bf16", groups=3),
        # all vertices of a large heterogeneous graph, residual rows in 16 bits
        _block("block_graph_bf16", 1_200_000, 256, "bf16", "bf16", groups=16),
        # a training step over a batch of graphs, each with its own gate
        _block("block_train_graphs", 500_000, 256, groups=9_001, train=True),
        # fp16 blocks on fp32 residual rows, a ragged count of narrow rows
        _block("block_train_ragged", 120_001, 100, "f16", "f32", groups=7, layer=False, train=True),
        # biases, norms and small weights of a network: latency
        _adamw("step_small", 40, 30_000),
        # a table and typed weights, everything in 32 bits
        _adamw("step_table_f32", 12, 60_000_000),
        # a large table in 16 bits with states in 8
        _adamw("step_table_8bit", 30, 200_000_000, "bf16", "bf16", bits=8),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))


def draw(rng):
    kind = rng.choice(["logprob", "logprob_train", "block", "block_train", "adamw"])
    type = rng.choice(list(TYPES))
    if kind.startswith("logprob"):
        train = kind == "logprob_train"
        classes = _log(rng, 1, 250_000)
        n = _log(rng, 1, min(1_200_000, (60_000_000 if train else 200_000_000) // classes))
        return _logprob(None, n, classes, type, 0 if train else rng.randint(0, 16), rng.random() < 0.4, train, train and rng.random() < 0.4)
    if kind.startswith("block"):
        train = kind == "block_train"
        # of two channels or one nothing is left but rounding: a norm's gradient is then the difference of two equal numbers
        width = _log(rng, 4 if train else 1, 1024)
        n = _log(rng, 1, min(1_200_000, (125_000_000 if train else 300_000_000) // width))
        groups = 0 if rng.random() < 0.2 else _log(rng, 1, min(n, 50_000))
        return _block(None, n, width, type, rng.choice(["f32", type]), groups, rng.random() < 0.6, rng.random() < 0.7, train)
    bits, master = rng.choice([8, 32]), type != "f32" and rng.random() < 0.4
    tensors = _log(rng, 1, 300)
    total = _log(rng, tensors, 60_000_000 if bits == 32 else 150_000_000)
    return _adamw(None, tensors, total, type, rng.choice(["f32", type]), bits, master, _log(rng, 1, 100_000))


def _sizes(total, parts, g, empty):
    """Ragged sizes that add up to total: shares spread over two orders of magnitude, a part of them empty."""
    share = torch.exp(torch.rand(parts, generator=g, dtype=torch.float64) * 4.6)
    share[torch.rand(parts, generator=g, dtype=torch.float64) < empty] = 0
    if float(share.sum()) == 0:
        share[0] = 1
    ends = torch.floor(torch.cumsum(share, 0) / share.sum() * total + 0.5).to(torch.int64)
    ends[-1] = total
    return torch.cat([torch.zeros(1, dtype=torch.int64), ends])


def _tensor_sizes(c):
    """Elements of each tensor of an AdamW case: part of the case, not of its inputs."""
    rng = random.Random(c["total"] * 1009 + c["tensors"])
    share = [math.exp(rng.uniform(0, 6)) for _ in range(c["tensors"])]
    rest = c["total"] - c["tensors"]
    sizes = [1 + int(rest * s / sum(share)) for s in share]
    sizes[0] += c["total"] - sum(sizes)
    return sizes


def _power(e):
    """2 ** e for whole numbers e, exactly."""
    return ((e + 1023).to(torch.int64) << 52).view(torch.float64)


def _codes(x, n_blocks):
    """Blocks of 32-bit values as codes in 8 bits and a power of two for each block (to nearest: the state that training left)."""
    x = x.view(n_blocks, BLOCK)
    _, e = torch.frexp(x.abs().amax(1).clamp_(min=2.0 ** -119))
    scale = _power(e - 8).float()
    return (x / scale[:, None]).to(torch.float8_e4m3fn).view(-1), scale


def _inputs(case, seed):
    c = case
    g = torch.Generator().manual_seed(seed)
    d = torch.Generator("cuda").manual_seed(seed + 1)

    def normal(*shape):
        return torch.randn(*shape, generator=d, device="cuda")

    def uniform(*shape):
        return torch.rand(*shape, generator=d, device="cuda")

    s = {}
    if c["kind"].startswith("logprob"):
        n, C = c["n"], c["classes"]
        x = normal(n, C).mul_(2.0)
        s["labels"] = (uniform(n).double() * C).to(torch.int64).clamp_(max=C - 1)
        x[torch.arange(n, device="cuda"), s["labels"]] += 3.0
        s["labels"][uniform(n) < 0.1] = -1
        if c["masked"]:
            x[uniform(n, C) < 0.1] = -math.inf
            x[uniform(n) < 0.01] = -math.inf
        s["logits"] = x.to(TYPES[c["type"]])
        if c["kind"] == "logprob_train":
            s["grad_logprob"] = torch.full((n,), -1.0, device="cuda") * (0.5 + uniform(n))
            s["grad_entropy"] = -0.05 * (0.5 + uniform(n))
    elif c["kind"].startswith("block"):
        n, C, t, r = c["n"], c["width"], TYPES[c["type"]], TYPES[c["res"]]
        s["res"] = (normal(n, C) * (0.5 + uniform(C)) + 0.3 * normal(C)).to(r)
        s["block"] = (normal(n, C) * 0.7 + 0.2).to(t)
        s["post_gamma"] = 1 + 0.1 * normal(C) if c["post"] else None
        s["gamma"], s["beta"] = 1 + 0.1 * normal(C), 0.1 * normal(C) if c["layer"] else None
        s["gate"], s["offsets"] = None, None
        if c["groups"]:
            s["gate"] = 0.5 + 0.3 * normal(c["groups"], C)
            s["offsets"] = _sizes(n, c["groups"], g, 0.125).cuda()
        s["alpha"] = 0.7
        if c["kind"] == "block_train":
            s["grad_res"], s["grad_out"] = (normal(n, C) * 1e-2).to(r), (normal(n, C) * 1e-2).to(t)
    else:
        sizes = _tensor_sizes(c)
        starts, at = [], 0
        for n in sizes:
            starts.append(at)
            at += -(-n // BLOCK) * BLOCK
        used = torch.zeros(at, dtype=torch.bool, device="cuda")
        for b, n in zip(starts, sizes):
            used[b:b + n] = True
        s["sizes"], s["starts"] = sizes, starts
        live = used & (uniform(at // 64, 1) < 0.7).expand(-1, 64).reshape(-1)           # rows that some id named
        size = torch.exp(1.5 * normal(at // 64, 1)).expand(-1, 64).reshape(-1) * 1e-3
        grad = torch.where(live, normal(at) * size, 0.0)
        s["grad"] = (grad * 2).to(TYPES[c["grad"]])
        seen = used & (uniform(at // 64, 1) < 0.9).expand(-1, 64).reshape(-1)
        m = torch.where(seen, normal(at) * size * 0.3, 0.0)
        v = torch.where(seen, size * (0.5 + uniform(at)), 0.0)                            # its square root
        w = torch.where(used, normal(at) * 0.05, 0.0)
        s["param"] = w.to(TYPES[c["type"]])
        s["master"] = w if c["master"] else None
        if c["bits"] == 8:
            s["m"], s["m_scale"] = _codes(m, at // BLOCK)
            s["v"], s["v_scale"] = _codes(v, at // BLOCK)
        else:
            s["m"], s["v"], s["m_scale"], s["v_scale"] = m, v * v, None, None
        s["seed"] = seed * 7919 + 13
        s["lr"], s["step"] = torch.full((1,), 2e-3, device="cuda"), torch.full((1,), c["step"], dtype=torch.int64, device="cuda")
        s["grad_scale"] = torch.full((1,), 0.5, device="cuda")
        s["decay"] = [DECAY if n > 1024 else 0.0 for n in sizes]
    return s


def prepare(case, seed):
    c = case
    s = _inputs(c, seed)
    s["case"] = c

    def empty(*shape, dtype=torch.float32):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    s["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    if c["kind"] == "adamw":
        # what an element's tensor gives it: for the plain form, which takes all tensors as one array
        blocks = torch.tensor([-(-n // BLOCK) for n in s["sizes"]], device="cuda")
        keys = [_key(s["seed"], c["step"], t) for t in range(len(s["sizes"]))]
        s["block_decay"] = torch.tensor(s["decay"], device="cuda").repeat_interleave(blocks)
        s["block_key"] = torch.tensor([[k & 0xFFFFFFFF, k >> 32] for k in keys], device="cuda").repeat_interleave(blocks, 0)
        first = torch.tensor(s["starts"], device="cuda").repeat_interleave(blocks)
        s["block_first"] = torch.arange(len(first), device="cuda") * BLOCK - first
    if not own:
        return s
    import paper_2607_17374_b200 as tb
    size = 0
    if c["kind"].startswith("logprob"):
        n, k = c["n"], c["k"]
        s["logprob"], s["entropy"], s["stats"] = empty(n), empty(n), empty(n, 2)
        s["top_logprob"], s["top_class"] = (empty(n, k), empty(n, k, dtype=torch.int64)) if k else (None, None)
        if c["kind"] == "logprob_train":
            s["grad_logits"] = empty(n, c["classes"], dtype=TYPES[c["type"]])
        size = tb.class_logprob_workspace(n, c["classes"], k)
    elif c["kind"].startswith("block"):
        n, C, t, r = c["n"], c["width"], TYPES[c["type"]], TYPES[c["res"]]
        s["out_res"], s["out"] = empty(n, C, dtype=r), empty(n, C, dtype=t)
        s["stats"] = None
        if c["kind"] == "block_train":
            s["stats"] = empty(n, 4)
            s["d_res"], s["d_block"] = empty(n, C, dtype=r), empty(n, C, dtype=t)
            s["d_gamma"], s["d_beta"], s["d_post"] = empty(C), empty(C) if c["layer"] else None, empty(C) if c["post"] else None
            s["d_gate"] = empty(c["groups"], C) if c["groups"] else None
            size = tb.residual_norm_grad_workspace(n, C, c["groups"])
    else:
        def views(x):
            return None if x is None else [x[b:b + n] for b, n in zip(s["starts"], s["sizes"])]

        def scales(x):
            return None if x is None else [x[b // BLOCK:b // BLOCK + -(-n // BLOCK)] for b, n in zip(s["starts"], s["sizes"])]

        s["adamw"] = tb.AdamW(views(s["param"]), views(s["grad"]), views(s["m"]), views(s["v"]), scales(s["m_scale"]), scales(s["v_scale"]),
                              views(s["master"]), s["decay"])
    s["workspace"] = empty(size, dtype=torch.uint8) if size else None
    return s


def _state_of(s):
    return [s[k] for k in ("param", "master", "m", "v", "m_scale", "v_scale") if s[k] is not None]


def _run_own(s):
    import paper_2607_17374_b200 as tb
    c = s["case"]
    st = dict(status=s["status"], stream=torch.cuda.current_stream())
    if c["kind"] == "logprob_train" and not c["late"]:
        n, C = c["n"], c["classes"]
        tb.class_logprob_train(n, C, s["logits"], C, s["labels"], s["grad_logprob"], s["grad_entropy"], s["logprob"], s["entropy"], s["stats"], s["grad_logits"], C,
                               s["workspace"], **st)
        return [s["logprob"], s["entropy"], s["stats"], s["grad_logits"]]
    if c["kind"].startswith("logprob"):
        n, C = c["n"], c["classes"]
        tb.class_logprob(n, C, s["logits"], C, s["labels"], s["logprob"], s["entropy"], s["stats"], c["k"], s["top_logprob"], s["top_class"], s["workspace"], **st)
        if c["kind"] == "logprob_train":
            tb.class_logprob_grad(n, C, s["logits"], C, s["labels"], s["stats"], s["entropy"], s["grad_logprob"], s["grad_entropy"], s["grad_logits"], C, **st)
            return [s["logprob"], s["entropy"], s["stats"], s["grad_logits"]]
        top = [s["top_logprob"], s["top_class"]] if c["k"] else []
        return [s["logprob"], s["entropy"], s["stats"]] + top
    if c["kind"].startswith("block"):
        n, C, kind = c["n"], c["width"], tb.NORM_LAYER if c["layer"] else tb.NORM_RMS
        tb.residual_norm(n, C, s["res"], C, s["block"], C, kind, c["post"], s["post_gamma"], c["groups"], s["offsets"], s["gate"], s["alpha"], s["gamma"], s["beta"],
                         EPS, s["out_res"], C, s["out"], C, s["stats"], **st)
        if c["kind"] == "block":
            return [s["out_res"], s["out"]]
        tb.residual_norm_grad(n, C, s["res"], C, s["block"], C, kind, c["post"], s["post_gamma"], c["groups"], s["offsets"], s["gate"], s["alpha"], s["gamma"], s["stats"],
                              s["grad_res"], C, s["grad_out"], C, s["d_res"], C, s["d_block"], C, s["d_post"], s["d_gate"], s["d_gamma"], s["d_beta"], s["workspace"], **st)
        return [s["out_res"], s["out"]] + [s[k] for k in ("d_res", "d_block", "d_post", "d_gate", "d_gamma", "d_beta") if s[k] is not None]
    s["adamw"].step(s["step"], s["lr"], BETA1, BETA2, ADAM_EPS, s["grad_scale"], s["seed"], **st)
    return _state_of(s)


def _run_logprob(s):
    c = s["case"]
    x = s["logits"].float()
    m = x.amax(1)
    none = m == -math.inf                                                     # every class masked
    d = x - torch.where(none, 0.0, m)[:, None]
    e = torch.exp(d)
    total = torch.where(none, 1.0, e.sum(1, dtype=torch.float64))             # just above 1 where one class has nearly everything
    rest = torch.log(total)
    p = e / total.float()[:, None]
    logp = torch.where(d == -math.inf, 0.0, d - rest.float()[:, None])
    entropy = -(p * logp).sum(1, dtype=torch.float64)
    given, label = s["labels"] >= 0, s["labels"].clamp(min=0)[:, None]
    at = d.gather(1, label)[:, 0].double() - rest
    logprob = torch.where(given, at, 0.0).float()
    out = [logprob, entropy.float(), torch.stack([m, rest.float()], 1)]
    if c["kind"] == "logprob_train":
        g = torch.where(given, s["grad_logprob"], 0.0)
        dx = -g[:, None] * p
        dx.scatter_(1, label, (g * (total - e.gather(1, label)[:, 0]) / total).float()[:, None])
        dx -= s["grad_entropy"][:, None] * p * (logp + entropy.float()[:, None])
        return out + [torch.where(d == -math.inf, 0.0, dx).to(s["logits"].dtype)]
    k = c["k"]
    if k:
        values, order = torch.sort(x, dim=1, descending=True, stable=True)       # of equal ones the lowest class first
        values, order = values[:, :k], order[:, :k].clone()
        order[values == -math.inf] = -1
        top = torch.where(values == -math.inf, -math.inf, (values - m[:, None]).double() - rest[:, None]).float()
        if top.shape[1] < k:
            more = (0, k - top.shape[1])
            top, order = torch.nn.functional.pad(top, more, value=-math.inf), torch.nn.functional.pad(order, more, value=-1)
        out += [top, order]
    return out


def _group_of_rows(s, n):
    return torch.bucketize(torch.arange(n, device="cuda"), s["offsets"][1:], right=True)


def _normalised(x, layer):
    """(x - mean) rstd and rstd of each row; RMS: without the mean."""
    d = x - x.mean(1, keepdim=True) if layer else x
    rstd = torch.rsqrt((d * d).mean(1, keepdim=True) + EPS)
    return d * rstd, rstd


def _norm_back(dxh, xh, rstd, layer):
    d = dxh - xh * (dxh * xh).mean(1, keepdim=True)
    return (d - dxh.mean(1, keepdim=True) if layer else d) * rstd


def _run_block(s):
    c = s["case"]
    n, C, t, r = c["n"], c["width"], TYPES[c["type"]], TYPES[c["res"]]
    b = s["block"].float()
    if c["post"]:
        bh, rstd1 = _normalised(b, c["layer"])
        u = bh * s["post_gamma"]
    else:
        u = b
    group = _group_of_rows(s, n) if c["groups"] else None
    gate = s["gate"][group] * s["alpha"] if c["groups"] else s["alpha"]
    res = s["res"].float() + gate * u
    xh, rstd2 = _normalised(res, c["layer"])
    y = xh * s["gamma"]
    if c["layer"]:
        y = y + s["beta"]
    out = [res.to(r), y.to(t)]
    if c["kind"] == "block":
        return out
    dy = s["grad_out"].float()
    d_gamma, d_beta = (dy * xh).sum(0, dtype=torch.float64).float(), dy.sum(0, dtype=torch.float64).float()
    d_res = s["grad_res"].float() + _norm_back(dy * s["gamma"], xh, rstd2, c["layer"])
    du = d_res * gate
    out += [d_res.to(r)]
    if c["post"]:
        out += [_norm_back(du * s["post_gamma"], bh, rstd1, c["layer"]).to(t), (du * bh).sum(0, dtype=torch.float64).float()]
    else:
        out += [du.to(t)]
    if c["groups"]:
        d_gate = torch.zeros(c["groups"], C, dtype=torch.float64, device="cuda").index_add_(0, group, (d_res * u).double())
        out += [(d_gate * s["alpha"]).float()]
    return out + [d_gamma] + ([d_beta] if c["layer"] else [])


def _mix64(z):
    m = (1 << 64) - 1
    z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & m
    z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & m
    return z ^ (z >> 31)


def _key(seed, step, tensor):
    h = 0x243F6A8885A308D3
    for x in (seed, step, tensor):
        h = _mix64(h ^ (0x9E3779B97F4A7C15 * (x + 1) & ((1 << 64) - 1)))
    return h


def _random_bits(s):
    """32 bits for each element: a hash of (seed, step, tensor) and of its place in the tensor."""
    i = s["block_first"][:, None] + torch.arange(BLOCK, device="cuda")
    low = 0xFFFFFFFF
    x = ((i & low) ^ s["block_key"][:, :1]) + s["block_key"][:, 1:] + (i >> 32) * 0x85EBCA6B & low
    x = (x ^ (x >> 16)) * 0x7FEB352D & low
    x = (x ^ (x >> 15)) * 0x846CA68B & low
    return (x ^ (x >> 16)).view(-1)


def _rounded_codes(x, top, bits, keep):
    """Values as e4m3 codes and a power of two for each block, by the whole part of its largest logarithm: up with the probability of what is cut
    off; keep: what is not 0 stays so."""
    x = x.view(-1, BLOCK)
    scale = _power(top - 7).float()
    q = (x.abs() / scale[:, None]).double()
    _, e = torch.frexp(q)
    unit = _power((e - 1).clamp_(min=-6) - 3)
    whole = torch.floor((torch.floor(q / unit * 65536) + bits.view_as(q)) / 65536)
    if keep:
        whole = torch.where(q > 0, whole.clamp_(min=1.0), whole)
    return torch.copysign((whole * unit).float(), x).to(torch.float8_e4m3fn).view(-1), scale


def _run_adamw(s):
    c = s["case"]
    step = c["step"]
    g = s["grad"].float() * s["grad_scale"]
    eight = c["bits"] == 8

    def held(x, scale):
        return (x.float().view(-1, BLOCK) * scale[:, None]).view(-1) if eight else x

    m = BETA1 * held(s["m"], s["m_scale"]) + (1 - BETA1) * g
    v = held(s["v"], s["v_scale"])
    v = BETA2 * (v * v if eight else v) + (1 - BETA2) * g * g
    root = torch.sqrt(v)
    p = s["master"] if c["master"] else s["param"].float()
    decay = s["lr"] * s["block_decay"][:, None]
    update = (m / (1 - BETA1 ** step)) / (root / math.sqrt(1 - BETA2 ** step) + ADAM_EPS)
    p = (p.view(-1, BLOCK) - decay * p.view(-1, BLOCK)).view(-1) - s["lr"] * update
    s["param"].copy_(p)
    if c["master"]:
        s["master"].copy_(p)
    if eight:
        bits = _random_bits(s)
        top_m = torch.frexp(m.view(-1, BLOCK).abs().amax(1).clamp_(min=2.0 ** -119))[1] - 1
        top_v = (torch.frexp(v.view(-1, BLOCK).amax(1).clamp_(min=2.0 ** -126))[1] - 1) >> 1
        for name, x, top, r in (("m", m, top_m, bits & 0xFFFF), ("v", root, top_v, bits >> 16)):
            codes, scale = _rounded_codes(x, top, r, name == "v")
            s[name].copy_(codes)
            s[name + "_scale"].copy_(scale)
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
    return _state_of(s)


def run(state):
    if own:
        return _run_own(state)
    kind = state["case"]["kind"]
    return _run_logprob(state) if kind.startswith("logprob") else _run_block(state) if kind.startswith("block") else _run_adamw(state)


def _exact_logprob(c, s):
    n, C, k, train = c["n"], c["classes"], c["k"], c["kind"] == "logprob_train"
    rows = max(1, 50_000_000 // C)
    parts = []
    for b in range(0, n, rows):
        x, label = s["logits"][b:b + rows].double(), s["labels"][b:b + rows]
        most, lse = x.max(1).values, torch.logsumexp(x, 1)
        empty = torch.isinf(lse)
        logp = x - torch.where(empty, 0.0, lse)[:, None]
        p = torch.exp(logp)
        entropy = torch.special.entr(p).sum(1)
        lp = torch.where(empty[:, None], -math.inf, logp).gather(1, label.clamp(min=0)[:, None])[:, 0]
        part = [torch.where(label < 0, 0.0, lp), entropy, torch.stack([most, torch.where(empty, 0.0, lse - most)], 1)]
        if train:
            g = torch.where(label < 0, 0.0, s["grad_logprob"][b:b + rows].double())
            finite = torch.where(torch.isinf(logp), 0.0, logp)
            dx = -(g[:, None] + s["grad_entropy"][b:b + rows].double()[:, None] * (finite + entropy[:, None])) * p
            dx[torch.arange(len(dx), device="cuda"), label.clamp(min=0)] += g
            part.append(dx.masked_fill_(torch.isinf(x), 0.0))
        elif k:
            values = torch.topk(x, min(k, C), 1).values
            values = torch.nn.functional.pad(values, (0, k - values.shape[1]), value=-math.inf)
            part.append(torch.where(torch.isinf(values), values, values - torch.where(empty, 0.0, lse)[:, None]))
        parts.append(part)
    return [torch.cat(v) for v in zip(*parts)] + ([None] if k and not train else [])


def _exact_block(c, s):
    """The definition by blocks of rows, its gradients by the chain rule of each step, in 64 bits."""
    n, C, G, train = c["n"], c["width"], c["groups"], c["kind"] == "block_train"
    rows = max(1, 30_000_000 // C)
    gamma, alpha = s["gamma"].double(), s["alpha"]
    beta = s["beta"].double() if c["layer"] else 0.0
    post = s["post_gamma"].double() if c["post"] else None
    group = torch.repeat_interleave(torch.arange(G, device="cuda"), s["offsets"].diff()) if G else None
    sums = {k: torch.zeros(C, dtype=torch.float64, device="cuda") for k in ("post", "gamma", "beta")}
    d_gate = torch.zeros(max(G, 1), C, dtype=torch.float64, device="cuda")

    def norm(x):
        var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
        if not c["layer"]:
            var, mean = var + mean * mean, torch.zeros_like(mean)
        inv = (var + EPS) ** -0.5
        return (x - mean) * inv, inv

    def back(d, h, inv):
        first = d.sum(1, keepdim=True) / C if c["layer"] else 0.0
        return inv * (d - first - h * ((d * h).sum(1, keepdim=True) / C))

    parts = []
    for b in range(0, n, rows):
        res, blk = s["res"][b:b + rows].double(), s["block"][b:b + rows].double()
        ga = s["gate"].double()[group[b:b + rows]] * alpha if G else torch.full((1, 1), alpha, dtype=torch.float64, device="cuda")
        h1, inv1 = norm(blk) if c["post"] else (None, None)
        u = h1 * post if c["post"] else blk
        new = torch.addcmul(res, ga, u)
        h2, inv2 = norm(new)
        part = [new, torch.addcmul(torch.zeros_like(h2) + beta, h2, gamma)]
        if train:
            dy = s["grad_out"][b:b + rows].double()
            sums["gamma"] += torch.einsum("rc,rc->c", dy, h2)
            sums["beta"] += torch.einsum("rc->c", dy)
            dr = s["grad_res"][b:b + rows].double() + back(dy * gamma, h2, inv2)
            du = dr * ga
            if G:
                d_gate.index_add_(0, group[b:b + rows], dr * u, alpha=alpha)
            if c["post"]:
                sums["post"] += torch.einsum("rc,rc->c", du, h1)
            part += [dr, back(du * post, h1, inv1) if c["post"] else du]
        parts.append(part)
    out = [torch.cat(v) for v in zip(*parts)]
    if train:
        out += ([sums["post"]] if c["post"] else []) + ([d_gate] if G else []) + [sums["gamma"]] + ([sums["beta"]] if c["layer"] else [])
    return out


def _exact_adamw(c, s):
    """Tensor by tensor in 64 bits.  States in 8 bits have no value here: a hair on either side of a border makes a whole step of a code, or twice the scale."""
    t, eight = c["step"], c["bits"] == 8
    out = {k: torch.zeros(len(s["grad"]), dtype=torch.float64, device="cuda") for k in ("param", "m", "v")}
    lr, gs = float(s["lr"]), float(s["grad_scale"])
    for b, n, decay in zip(s["starts"], s["sizes"], s["decay"]):
        e = b + -(-n // BLOCK) * BLOCK
        g = s["grad"][b:e].double() * gs
        m, v = s["m"][b:e].double(), s["v"][b:e].double()
        if eight:
            m *= s["m_scale"][b // BLOCK:e // BLOCK].double().repeat_interleave(BLOCK)
            v = (v * s["v_scale"][b // BLOCK:e // BLOCK].double().repeat_interleave(BLOCK)) ** 2
        m.lerp_(g, 1 - BETA1)
        v.lerp_(g.square(), 1 - BETA2)
        w = (s["master"] if c["master"] else s["param"])[b:e].double()
        top, root = m / (1 - BETA1 ** t), (v / (1 - BETA2 ** t)).sqrt()
        out["param"][b:e] = w * (1 - lr * decay) - lr * top / (root + ADAM_EPS)
        out["m"][b:e], out["v"][b:e] = m, v
    params = [out["param"]] + ([out["param"]] if c["master"] else [])
    return params + ([None, None, None, None] if eight else [out["m"], out["v"]])


def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    return _exact_logprob(case, s) if kind.startswith("logprob") else _exact_block(case, s) if kind.startswith("block") else _exact_adamw(case, s)


def work(case):
    c = case
    if c["kind"].startswith("logprob"):
        n, C, t = c["n"], c["classes"], SIZE[c["type"]]
        if c["kind"] == "logprob":
            return {"bytes": n * (C * t + 8 + 12 + 12 * c["k"]), "flops": 5 * n * C}
        return {"bytes": n * ((3 if c["late"] else 2) * C * t + 8 + 12 + 8), "flops": 12 * n * C}
    if c["kind"].startswith("block"):
        n, C, t, r = c["n"], c["width"], SIZE[c["type"]], SIZE[c["res"]]
        sides = 8 + 4 * C
        if c["kind"] == "block":
            return {"bytes": 2 * n * C * (t + r) + c["groups"] * sides + 12 * C, "flops": 14 * n * C}
        return {"bytes": 4 * n * C * (t + r) + c["groups"] * (sides + 4 * C) + 24 * C, "flops": 45 * n * C}
    e, p = c["total"], SIZE[c["type"]]
    state = 4 if c["bits"] == 8 else 16
    return {"bytes": e * (2 * p + SIZE[c["grad"]] + state + (8 - p if c["master"] else 0)) + (16 * e // BLOCK if c["bits"] == 8 else 0), "flops": 20 * e}
