"""The timed workloads of a training step's remaining parts around the MoE layer: the embedding with its gradient, the norms in front of
and behind the block, and the Muon update of the layer's matrices.

kinds
  embed       rows of an embedding for a batch of tokens, scaled
  embed_grad  the gradient of the embedding from the rows' gradients, written or added to what is there (a matrix shared with the loss)
  norm        the end of one block and the start of the next: residual stream, normed and gated block output, norm in front of the next
  norm_grad   all its gradients
  orth        a batch of matrices orthogonalised by five quintic Newton-Schulz steps
  muon        one Muon update: momentum, orthogonalised, added to the parameters with decay, in place

Widths are those of this repository's layers (synth/moe_inputs.py) and generic odd ones; vocabularies are generic.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
EPS = 1e-6
STEPS = ((3.4445, -4.7750, 2.0315),) * 5
MOMENTUM, DECAY, LR = 0.95, 0.1, 3e-4


# padding: share of tokens that have no row; add: the gradient is added to what is there
def _embed(name, kind, T, d, V, dtype="bf16", scale=1.0, padding=0.0, add=0):
    return dict(name=name, kind=kind, T=T, d=d, V=V, dtype=dtype, scale=scale, padding=padding, add=add)


# residual: there is a block output to add; after: it is normed; gate_rows: tokens that share a row of the gate (0: no gate);
# before: the norm in front of the next block
def _norm(name, kind, T, d, dtype="bf16", residual=1, after=1, gate_rows=0, before=1, alpha=1.0):
    return dict(name=name, kind=kind, T=T, d=d, dtype=dtype, residual=residual, after=after, gate_rows=gate_rows, before=before, alpha=alpha)


# decay: singular values of the gradients' common part fall as the index to minus this
def _matrices(name, kind, batch, rows, cols, dtype, decay=0.5):
    return dict(name=name, kind=kind, batch=batch, rows=rows, cols=cols, dtype=dtype, decay=decay)


def listed():
    return [
        # the next token while serving: one row
        _embed("embed_1_token", "embed", 1, 4096, 32000),
        # a training batch of the fine-grained layer over a large vocabulary, padded at its end
        _embed("embed_16384_tokens", "embed", 16384, 2048, 102400, scale=45.25, padding=0.06),
        # a small fp32 model with odd sizes
        _embed("embed_grad_f32_1009_tokens", "embed_grad", 1009, 1040, 5003, dtype="f32", scale=32.25, padding=0.1),
        # the micro-batch of the headline layer of bench.py
        _embed("embed_grad_8192_tokens", "embed_grad", 8192, 4096, 32000),
        # serving one token: launches, not bytes
        _norm("norm_1_token", "norm", 1, 4096),
        # a training batch of the fine-grained layer, the gate a vector
        _norm("norm_16384_tokens", "norm", 16384, 2048, gate_rows=16384),
        # a small fp32 model with odd sizes, a gate for each sequence
        _norm("norm_grad_f32_777_tokens", "norm_grad", 777, 1040, dtype="f32", gate_rows=111, alpha=0.75),
        # the micro-batch of the headline layer
        _norm("norm_grad_8192_tokens", "norm_grad", 8192, 4096, gate_rows=8192),
        # the router of the fine-grained layer: one small matrix
        _matrices("orth_router", "orth", 1, 64, 2048, "f32"),
        # down projections of the fine-grained layer's experts
        _matrices("orth_64_experts", "orth", 64, 2048, 1408, "bf16"),
        # the tiny layer's up projections
        _matrices("muon_tiny_layer", "muon", 16, 256, 128, "f32"),
        # two down projections of the headline layer
        _matrices("muon_2_experts", "muon", 2, 4096, 14336, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["embed", "embed_grad", "norm", "norm_grad", "orth", "muon"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind in ("embed", "embed_grad"):
        while True:
            T, d, V = _log_int(rng, 1, 65536), 16 * _log_int(rng, 4, 256), _log_int(rng, 300, 131072)
            if T * d <= 8192 * 4096 and V * d <= 210_000_000:
                break
        return dict(kind=kind, T=T, d=d, V=V, dtype=dtype, scale=rng.choice([1.0, math.sqrt(d)]), padding=rng.choice([0.0, 0.0, 0.3]),
                    add=rng.randint(0, 1) if kind == "embed_grad" else 0)
    if kind in ("norm", "norm_grad"):
        while True:
            T, d = _log_int(rng, 1, 32768), 16 * _log_int(rng, 4, 512)
            if T * d <= 8192 * 4096:
                break
        residual = int(rng.random() < 0.85)
        gate_rows = rng.choice([0, 1, T, max(1, T // rng.randint(2, 9))]) if residual else 0
        return dict(kind=kind, T=T, d=d, dtype=dtype, residual=residual, after=rng.randint(0, 1) if residual else 0, gate_rows=gate_rows,
                    before=1 if not residual else rng.randint(0, 1), alpha=rng.choice([1.0, 1.0, 0.5]) if residual else 1.0)
    while True:
        batch, rows, cols = _log_int(rng, 1, 128), _log_int(rng, 8, 8192), _log_int(rng, 8, 16384)
        m, n = min(rows, cols), max(rows, cols)
        if batch * m * m * (3 * n + m) <= 8e11 and batch * m * n <= 120_000_000:
            break
    return dict(kind=kind, batch=batch, rows=rows, cols=cols, dtype=dtype, decay=rng.choice([0.0, 0.3, 0.5, 0.7]))


# ---- inputs ------------------------------------------------------------------------------------------------------------
def _dtype(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _tokens(c, g):
    """Words by rank: the share of the word of rank r falls as 1 / r; the ranks lie anywhere in the vocabulary."""
    rank = torch.exp(torch.rand((c["T"],), device=DEV, generator=g, dtype=torch.float64) * math.log(c["V"] + 1.0)).long() - 1
    tokens = torch.randperm(c["V"], device=DEV, generator=g)[rank.clamp(0, c["V"] - 1)]
    none = torch.rand((c["T"],), device=DEV, generator=g) < c["padding"]
    return torch.where(none, torch.full_like(tokens, -1), tokens).to(torch.int32)


def _embed_inputs(c, seed):
    g = _generator(seed)
    tokens = _tokens(c, g)
    if c["kind"] == "embed":
        return tokens, torch.randn((c["V"], c["d"]), device=DEV, generator=g).mul_(0.02).to(_dtype(c["dtype"]))
    dy = torch.randn((c["T"], c["d"]), device=DEV, generator=g).mul_(1e-3).to(_dtype(c["dtype"]))
    d_table = torch.zeros((c["V"], c["d"]), device=DEV)
    if c["add"]:
        d_table.normal_(0.0, 1e-4, generator=g)
    return tokens, dy, d_table


def _norm_inputs(c, seed):
    g = _generator(seed)
    T, d, dt = c["T"], c["d"], _dtype(c["dtype"])

    def rows(std):
        # a few channels carry much more than the others, tokens differ in size
        channel = 1.0 + 9.0 * (torch.rand((d,), device=DEV, generator=g) < 0.01)
        token = torch.exp(0.5 * torch.randn((T, 1), device=DEV, generator=g))
        return (torch.randn((T, d), device=DEV, generator=g) * channel * token * std).to(dt)

    def weight():
        return 1.0 + 0.2 * torch.randn((d,), device=DEV, generator=g)

    x, y = rows(2.0), rows(0.7) if c["residual"] else None
    w_after = weight() if c["after"] else None
    groups = -(-T // c["gate_rows"]) if c["gate_rows"] else 0
    gate = 0.3 + 0.2 * torch.randn((groups, d), device=DEV, generator=g) if groups else None
    w_before = weight() if c["before"] else None
    d_out = rows(1e-3) if c["residual"] else None
    d_h = rows(1e-3) if c["before"] else None
    return x, y, w_after, gate, w_before, d_out, d_h


def _matrix_inputs(c, seed):
    g = _generator(seed)
    batch, rows, cols = c["batch"], c["rows"], c["cols"]
    r = min(rows, cols)
    value = torch.arange(1, r + 1, device=DEV, dtype=torch.float32) ** -c["decay"]
    shape = (batch, rows, cols)
    m = torch.empty(shape, device=DEV)
    for i in range(batch):
        left = torch.randn((rows, r), device=DEV, generator=g) * value
        torch.mm(left, torch.randn((r, cols), device=DEV, generator=g), out=m[i])
        m[i] *= 3e-4 / (m[i].square().mean().sqrt() + 1e-30)
    grad = torch.randn(shape, device=DEV, generator=g).mul_(1e-4).add_(m, alpha=0.1).to(_dtype(c["dtype"]))
    if c["kind"] == "orth":
        return (m.to(_dtype(c["dtype"])),)
    p = torch.randn(shape, device=DEV, generator=g).mul_(0.02)              # (the layers' w_std)
    return p, grad, m


def prepare(case, seed):
    c = dict(case)
    if c["kind"] == "embed":
        tokens, table = _embed_inputs(c, seed)
        return dict(c, tokens=tokens, table=table)
    if c["kind"] == "embed_grad":
        tokens, dy, d_table = _embed_inputs(c, seed)
        return dict(c, tokens=tokens, dy=dy, d_table=d_table)
    if c["kind"] in ("norm", "norm_grad"):
        x, y, w_after, gate, w_before, d_out, d_h = _norm_inputs(c, seed)
        s = dict(c, x=x, y=y, w_after=w_after, gate=gate, w_before=w_before, d_out=d_out, d_h=d_h)
        if c["kind"] == "norm_grad":           # the stream that the forward pass has left behind
            s["out"], _ = _forward(s)
        return s
    if c["kind"] == "orth":
        return dict(c, x=_matrix_inputs(c, seed)[0])
    p, grad, m = _matrix_inputs(c, seed)
    return dict(c, p=p, g=grad, m=m, w16=torch.empty_like(p, dtype=torch.bfloat16), lr=torch.full((1,), LR, device=DEV))


# ---- plain forms -------------------------------------------------------------------------------------------------------
def _kept(s):
    return ((s["tokens"] >= 0) & (s["tokens"] < s["V"])).unsqueeze(1)


def _plain_embed(s):
    rows = s["table"][s["tokens"].clamp(min=0).long()].float() * s["scale"]
    return {"out": torch.where(_kept(s), rows, torch.zeros_like(rows)).to(s["table"].dtype)}


def _plain_embed_grad(s):
    rows = s["dy"].float() * s["scale"]
    rows = torch.where(_kept(s), rows, torch.zeros_like(rows))
    if not s["add"]:
        s["d_table"].zero_()
    s["d_table"].index_add_(0, s["tokens"].clamp(min=0).long(), rows)
    return {"d_table": s["d_table"]}


def _unit(v):
    """v over its root mean square, and one over that."""
    r = (v.square().mean(1, keepdim=True) + EPS).rsqrt()
    return v * r, r


def _gate_of_tokens(s):
    return s["gate"].repeat_interleave(s["gate_rows"], 0)[: s["T"]]


def _forward(s):
    out, dt = s["x"], s["x"].dtype
    if s["residual"]:
        n = s["y"].float()
        if s["after"]:
            n = _unit(n)[0] * s["w_after"]
        if s["gate_rows"]:
            n = n * _gate_of_tokens(s)
        out = (s["alpha"] * s["x"].float() + n).to(dt)
    # the next block's norm is that of the stream as it is kept
    return out, (_unit(out.float())[0] * s["w_before"]).to(dt) if s["before"] else None


def _plain_norm(s):
    out, h = _forward(s)
    return {"out": out if s["residual"] else None, "h": h}


def _norm_back(unit, r, w, d_n):
    """Gradients of unit(v) * w: of v, and of w by token."""
    u = d_n * w
    return (u - unit * (u * unit).mean(1, keepdim=True)) * r, d_n * unit


def _plain_norm_grad(s):
    dt, got = s["x"].dtype, {}
    g = s["d_out"].float() if s["residual"] else torch.zeros((), device=DEV)
    if s["before"]:
        unit, r = _unit(s["out"].float())
        back, d_w = _norm_back(unit, r, s["w_before"], s["d_h"].float())
        g = g + back
        got["d_w_before"] = d_w.sum(0)
    got["dx"] = (s["alpha"] * g).to(dt)
    if s["residual"]:
        n = s["y"].float()
        if s["after"]:
            unit, r = _unit(n)
            n = unit * s["w_after"]
        if s["gate_rows"]:
            gn = g * n
            short = s["gate"].shape[0] * s["gate_rows"] - s["T"]
            got["d_gate"] = torch.nn.functional.pad(gn, (0, 0, 0, short)).view(s["gate"].shape[0], s["gate_rows"], s["d"]).sum(1)
            g = g * _gate_of_tokens(s)
        if s["after"]:
            g, d_w = _norm_back(unit, r, s["w_after"], g)
            got["d_w_after"] = d_w.sum(0)
        got["dy"] = g.to(dt)
    return got


def _plain_orthogonal(u):
    """Five steps X <- a X + b (X X^T) X + c (X X^T)^2 X from u / |u|, on the side where X X^T is smaller."""
    tall = u.shape[1] > u.shape[2]
    x = u.transpose(1, 2).contiguous() if tall else u
    x = x / x.double().square().sum((1, 2), keepdim=True).sqrt().float().clamp(min=1e-38)
    for a, b, c in STEPS:
        gram = torch.bmm(x, x.transpose(1, 2).contiguous())
        x = a * x + torch.bmm(b * gram + c * torch.bmm(gram, gram), x)
    return x.transpose(1, 2) if tall else x


def _plain_orth(s):
    return {"out": _plain_orthogonal(s["x"].float()).to(torch.bfloat16).contiguous()}


def _plain_muon(s):
    g = s["g"].float()
    s["m"].mul_(MOMENTUM).add_(g)
    update = _plain_orthogonal(g + MOMENTUM * s["m"])
    s["p"].mul_(1.0 - s["lr"] * DECAY).sub_(s["lr"] * (0.2 * math.sqrt(max(s["rows"], s["cols"]))) * update)
    s["w16"].copy_(s["p"])
    return {"p": s["p"], "m": s["m"], "w16": s["w16"]}


# ---- the framework's calls: the handle (buffers, workspaces) is made once per state, as a user's program does --------------
def _own_embed(s):
    from paper_2505_11432_amd.embedding import Embedding
    if "op" not in s:
        s["op"] = Embedding(s["T"], s["d"], s["V"], dtype=_dtype(s["dtype"]), scale=s["scale"], gradients=s["kind"] == "embed_grad", device=DEV,
                            d_table=s.get("d_table"))
    if s["kind"] == "embed":
        return {"out": s["op"].lookup(s["table"], s["tokens"])}
    return {"d_table": s["op"].backward(s["tokens"], s["dy"], accumulate=bool(s["add"]))}


def _own_norm(s):
    from paper_2505_11432_amd.norm import BlockNorm
    if "op" not in s:
        s["op"] = BlockNorm(s["T"], s["d"], dtype=_dtype(s["dtype"]), eps=EPS, alpha=s["alpha"], residual=bool(s["residual"]), after=bool(s["after"]),
                            gate_rows=s["gate_rows"], before=bool(s["before"]), gradients=s["kind"] == "norm_grad", device=DEV)
    op = s["op"]
    if s["kind"] == "norm":
        out, h = op.forward(s["x"], s["y"], s["w_after"], s["gate"], s["w_before"])
        return {"out": out if s["residual"] else None, "h": h}
    op.backward(s["out"], s["y"], s["w_after"], s["gate"], s["w_before"], s["d_out"], s["d_h"])
    got = {"dx": op.dx, "dy": op.dy, "d_w_after": op.d_w_after, "d_gate": op.d_gate, "d_w_before": op.d_w_before}
    return {k: v for k, v in got.items() if v is not None}


def _own_orth(s):
    from paper_2505_11432_amd.optim import Orthogonal
    if "op" not in s:
        s["op"] = Orthogonal(s["batch"], s["rows"], s["cols"], out_dtype=torch.bfloat16, coefficients=STEPS, device=DEV)
    return {"out": s["op"].apply(s["x"])}


def _own_muon(s):
    from paper_2505_11432_amd.optim import Muon
    if "op" not in s:
        s["op"] = Muon([s["p"]], [s["g"]], [s["m"]], weights=[s["w16"]], lr=s["lr"], momentum=MOMENTUM, nesterov=True, weight_decay=DECAY,
                       coefficients=STEPS)
    s["op"].step()
    return {"p": s["p"], "m": s["m"], "w16": s["w16"]}


def run(state):
    if own:
        return {"embed": _own_embed, "embed_grad": _own_embed, "norm": _own_norm, "norm_grad": _own_norm, "orth": _own_orth,
                "muon": _own_muon}[state["kind"]](state)
    return {"embed": _plain_embed, "embed_grad": _plain_embed_grad, "norm": _plain_norm, "norm_grad": _plain_norm_grad, "orth": _plain_orth,
            "muon": _plain_muon}[state["kind"]](state)


# ---- what a pass cannot do without ---------------------------------------------------------------------------------------
def _distinct(c):
    """Expected number of different words among the tokens (shares 1 / r)."""
    T, V = c["T"] * (1.0 - c["padding"]), c["V"]
    total, r = 0.0, 1
    while r <= V:
        step = max(1, r // 16)
        step = min(step, V - r + 1)
        share = math.log1p(step / r) / math.log(V + 1.0) / step
        total += step * -math.expm1(T * math.log1p(-min(share, 0.999999)))
        r += step
    return max(1.0, total)


def work(case):
    c = case
    es = 4 if c["dtype"] == "f32" else 2
    if c["kind"] == "embed":
        T, d = c["T"], c["d"]
        return {"bytes": 4.0 * T + _distinct(c) * d * es + T * d * es, "flops": float(T * d)}
    if c["kind"] == "embed_grad":
        T, d = c["T"] * (1.0 - c["padding"]), c["d"]
        table = 2.0 * _distinct(c) if c["add"] else float(c["V"])
        return {"bytes": 4.0 * c["T"] + T * d * es + table * d * 4, "flops": 2.0 * T * d}
    if c["kind"] in ("norm", "norm_grad"):
        T, d = c["T"], c["d"]
        groups = -(-T // c["gate_rows"]) if c["gate_rows"] else 0
        vectors = (c["after"] + groups + c["before"]) * d * 4.0
        if c["kind"] == "norm":
            return {"bytes": T * d * es * (1.0 + 2 * c["residual"] + c["before"]) + vectors, "flops": 10.0 * T * d}
        needs_y = c["residual"] and (c["after"] or c["gate_rows"])
        rows = 2 * c["before"] + 1 + 2 * c["residual"] + (1 if needs_y else 0)          # stream, d_h; dx; d_out, dy; y
        return {"bytes": T * d * es * float(rows) + 2 * vectors, "flops": 25.0 * T * d}
    # X X^T and its square are symmetric: half their products
    m, n = min(c["rows"], c["cols"]), max(c["rows"], c["cols"])
    flops = float(c["batch"]) * len(STEPS) * m * m * (3.0 * n + m)
    size = float(c["batch"]) * m * n
    if c["kind"] == "orth":
        return {"bytes": size * (es + 2), "flops": flops}
    return {"bytes": size * (es + 18), "flops": flops}


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------------
def _exact_embed(c, seed):
    tokens, table = _embed_inputs(c, seed)
    out = torch.zeros((c["T"], c["d"]), dtype=torch.float64, device=DEV)
    at = (tokens >= 0).nonzero().squeeze(1)
    out[at] = table.double()[tokens[at].long()] * c["scale"]
    return {"out": out}


def _exact_embed_grad(c, seed):
    tokens, dy, d_table = _embed_inputs(c, seed)
    total = d_table.double() if c["add"] else torch.zeros_like(d_table, dtype=torch.float64)
    order = torch.argsort(tokens, stable=True)
    order = order[tokens[order] >= 0]
    words, counts = torch.unique_consecutive(tokens[order], return_counts=True)
    if not len(words):
        return {"d_table": total}
    for cols in torch.arange(c["d"], device=DEV).split(512):
        run = torch.zeros((len(order) + 1, len(cols)), dtype=torch.float64, device=DEV)
        torch.cumsum(dy[:, cols].double()[order], 0, out=run[1:])
        ends = counts.cumsum(0)
        total[words.long()[:, None], cols] += c["scale"] * (run[ends] - run[ends - counts])
    return {"d_table": total}


def _exact_norm_parts(c, seed):
    parts = _norm_inputs(c, seed)
    x, y, w_after, gate, w_before = (None if t is None else t.double().requires_grad_(c["kind"] == "norm_grad") for t in parts[:5])
    row = (torch.arange(c["T"], device=DEV) // c["gate_rows"]) if c["gate_rows"] else None

    def rms_norm(v, w):
        return v / torch.sqrt(v.pow(2).sum(-1, keepdim=True) / c["d"] + EPS) * w

    out = x
    if y is not None:
        branch = rms_norm(y, w_after) if w_after is not None else y
        out = x * c["alpha"] + (branch * gate[row] if gate is not None else branch)
    h = rms_norm(out, w_before) if w_before is not None else None
    return (x, y, w_after, gate, w_before), out, h, parts[5], parts[6]


def _exact_norm(c, seed):
    _, out, h, _, _ = _exact_norm_parts(c, seed)
    return {"out": out if c["residual"] else None, "h": h}


def _exact_norm_grad(c, seed):
    leaves, out, h, d_out, d_h = _exact_norm_parts(c, seed)
    # (the stream of the forward pass is kept rounded, and the derivative is taken there: it is moved to that place)
    if h is not None and c["residual"]:
        kept = out.detach().to(_dtype(c["dtype"])).double()
        here = kept.requires_grad_()
        h = here / torch.sqrt(here.pow(2).sum(-1, keepdim=True) / c["d"] + EPS) * leaves[4]
        at_h = torch.autograd.grad(h, [here, leaves[4]], d_h.double())
        total, d_w_before = d_out.double() + at_h[0], at_h[1]
    elif h is not None:
        g = torch.autograd.grad(h, [leaves[0], leaves[4]], d_h.double())
        return {"dx": g[0], "d_w_before": g[1]}
    else:
        total, d_w_before = d_out.double(), None
    names = ["dx", "dy", "d_w_after", "d_gate"]
    asked = [(k, t) for k, t in zip(names, leaves[:4]) if t is not None]
    got = dict(zip([k for k, _ in asked], torch.autograd.grad(out, [t for _, t in asked], total)))
    if d_w_before is not None:
        got["d_w_before"] = d_w_before
    return got


def _exact_orthogonal(u):
    """By the definition on the singular values' side that is given, one matrix at a time."""
    done = []
    for x in u:
        size = torch.linalg.vector_norm(x)
        x = x / size if float(size) > 0 else x
        for a, b, c in STEPS:
            if x.shape[0] <= x.shape[1]:
                xx = x @ x.t()
                x = a * x + b * (xx @ x) + c * (xx @ (xx @ x)) if x.shape[1] < 2 * x.shape[0] else a * x + (b * xx + c * xx @ xx) @ x
            else:
                xx = x.t() @ x
                x = a * x + x @ (b * xx + c * xx @ xx)
        done.append(x)
    return torch.stack(done)


def _exact_orth(c, seed):
    return {"out": _exact_orthogonal(_matrix_inputs(c, seed)[0].double())}


def _exact_muon(c, seed):
    p, grad, m = (t.double() for t in _matrix_inputs(c, seed))
    m = MOMENTUM * m + grad
    update = _exact_orthogonal(grad + MOMENTUM * m)
    lr = float(torch.tensor(LR))
    p = p - lr * DECAY * p - lr * 0.2 * max(c["rows"], c["cols"]) ** 0.5 * update
    return {"p": p, "m": m, "w16": p}


def exact(case, seed):
    return {"embed": _exact_embed, "embed_grad": _exact_embed_grad, "norm": _exact_norm, "norm_grad": _exact_norm_grad, "orth": _exact_orth,
            "muon": _exact_muon}[case["kind"]](dict(case), seed)
