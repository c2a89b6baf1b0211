"""The timed workloads of what follows the MoE layer in a training step: the vocabulary loss with its gradients, the global
gradient norm with clipping, and the AdamW update.

kinds
  score   loss and log-sum-exp of every token's logits over the vocabulary, forward only (evaluation, serving)
  loss    the same with the gradients of the hidden rows and of the vocabulary matrix (a micro-batch of a training step)
  clip    gradient norm over a list of tensors and the clipped gradients
  adamw   one update of a list of tensors from their gradients and the clip factor, in place

Widths are those of this repository's layers (synth/moe_inputs.py) and generic odd ones; vocabularies are generic.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda:0"
EPS_CLIP = 1e-6
BETA1, BETA2, EPS, DECAY, LR = 0.9, 0.95, 1e-8, 0.1, 3e-4


# ignored: share of tokens whose target is left out; weights: 1 = a weight per token, 0 = the mean over counted tokens
def _loss(name, kind, T, d, V, dtype="bf16", ignored=0.0, weights=0):
    return dict(name=name, kind=kind, T=T, d=d, V=V, dtype=dtype, ignored=ignored, weights=weights)


# bf16: share of the elements that lie in bf16 tensors; limit: max_norm over the expected norm (below 1: clipped)
def _clip(name, n, numel, bf16, limit):
    return dict(name=name, kind="clip", n=n, numel=numel, bf16=bf16, limit=limit)


# grad: type of the gradients; steps: updates taken before this one
def _adamw(name, n, numel, grad, steps):
    return dict(name=name, kind="adamw", n=n, numel=numel, grad=grad, steps=steps)


def listed():
    return [
        # log-probability of one token while serving: the vocabulary matrix is read for a single row
        _loss("score_1_token", "score", 1, 4096, 32000),
        # a small evaluation batch; no size is a multiple of a tile
        _loss("score_257_tokens", "score", 257, 2048, 50257),
        # evaluation of answers: the prompt's tokens are left out
        _loss("score_4096_tokens", "score", 4096, 4096, 32000, ignored=0.3),
        # the smallest training step: a small fp32 model with odd sizes
        _loss("loss_f32_131_tokens", "loss", 131, 1040, 5003, dtype="f32", ignored=0.1),
        # a single-precision step of ordinary size
        _loss("loss_f32_1000_tokens", "loss", 1000, 1024, 32000, dtype="f32", weights=1),
        # the micro-batch of the headline layer of bench.py
        _loss("loss_8192_tokens", "loss", 8192, 4096, 32000),
        # packed instruction data on the fine-grained layer: a large vocabulary, weighted tokens, half of them left out
        _loss("loss_16384_tokens_half", "loss", 16384, 2048, 102400, ignored=0.5, weights=1),
        # the gradients of the tiny fp32 layer: launches, not bytes
        _clip("clip_tiny_layer", 5, 460_000, 0.0, 0.37),
        # a whole model's list: many tensors of all sizes, matrices in bf16, the rest in fp32
        _clip("clip_400_tensors", 400, 300_000_000, 0.9, 0.37),
        # fp32 main gradients of the eight experts of the headline layer, within the limit
        _clip("clip_experts", 18, 1_409_000_000, 0.0, 2.0),
        # the tiny layer's update
        _adamw("adamw_tiny_layer", 5, 460_000, "f32", 0),
        # matrices of the headline layer and some hundred smaller tensors, bf16 gradients
        _adamw("adamw_120_tensors", 120, 400_000_000, "bf16", 999),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["score", "score", "loss", "loss", "loss", "loss_f32", "clip", "clip", "adamw"])
    if kind == "clip":
        return dict(kind="clip", n=_log_int(rng, 1, 500), numel=_log_int(rng, 1000, 1_000_000_000), bf16=rng.choice([0.0, 0.5, 1.0]),
                    limit=rng.choice([0.3, 0.9, 3.0]))
    if kind == "adamw":
        return dict(kind="adamw", n=_log_int(rng, 1, 300), numel=_log_int(rng, 1000, 400_000_000), grad=rng.choice(["bf16", "f32"]),
                    steps=rng.choice([0, 1, 17, 5000]))
    f32 = kind == "loss_f32" or (kind == "score" and rng.random() < 0.2)
    most = 2.5e11 if f32 else 3.4e12
    while True:
        T, d, V = _log_int(rng, 1, 16384), 16 * _log_int(rng, 8, 256), _log_int(rng, 500, 131072)
        if T * d * V <= most:
            break
    return dict(kind="score" if kind == "score" else "loss", T=T, d=d, V=V, dtype="f32" if f32 else "bf16",
                ignored=rng.choice([0.0, 0.0, 0.25, 0.8]), weights=rng.randint(0, 1))


# ---- inputs ------------------------------------------------------------------------------------------------------------
def _dtype(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _loss_inputs(c, seed):
    g = _generator(seed)
    T, d, V, dt = c["T"], c["d"], c["V"], _dtype(c["dtype"])
    w = torch.randn((V, d), device=DEV, generator=g).mul_(1.28 / math.sqrt(d))
    target = torch.randint(0, V, (T,), device=DEV, generator=g)
    # normalised hidden rows that lean towards their target's row by varying amounts: losses from near 0 to past log V
    lean = torch.rand((T, 1), device=DEV, generator=g) * 8.0
    x = torch.randn((T, d), device=DEV, generator=g).addcmul_(lean, w[target])
    left_out = torch.rand((T,), device=DEV, generator=g) < c["ignored"]
    target = torch.where(left_out, torch.full_like(target, -100), target).to(torch.int32)
    token_w = torch.rand((T,), device=DEV, generator=g).add_(0.25).div_(T) if c["weights"] else None
    return x.to(dt), w.to(dt), target, token_w


def _sizes(n, numel):
    """n sizes that add up to numel, spread over their logarithm, odd ones and one empty tensor among them."""
    if n == 0:
        return []
    rng = random.Random(n * 1_000_003 + numel)
    share = [math.exp(rng.uniform(0.0, 9.0)) for _ in range(n)]
    total = sum(share)
    sizes = [int(numel * s / total) for s in share]
    if n > 3:
        sizes[1] = 0
    sizes[0] += numel - sum(sizes)
    return sizes


def _flat(sizes, scales, dtype, g):
    """One buffer with the tensors one after another, and the tensors: views at whatever offset they come to."""
    buf = torch.empty((sum(sizes),), dtype=dtype, device=DEV)
    views = list(buf.split(sizes)) if sizes else []
    for v, s in zip(views, scales):
        v.normal_(0.0, s, generator=g)
    return buf, views


def _clip_inputs(c, seed):
    g = _generator(seed)
    n16 = int(round(c["n"] * c["bf16"])) if c["n"] > 1 else int(c["bf16"] >= 0.5)
    numel16 = 0 if n16 == 0 else c["numel"] if n16 == c["n"] else int(c["numel"] * c["bf16"])
    s16, s32 = _sizes(n16, numel16), _sizes(c["n"] - n16, c["numel"] - numel16)
    rng = random.Random(seed)
    scales = [10.0 ** rng.uniform(-4.0, -1.0) for _ in range(c["n"])]
    norm = math.sqrt(sum(n * s * s for n, s in zip(s16 + s32, scales)))
    b16, v16 = _flat(s16, scales[:n16], torch.bfloat16, g)
    b32, v32 = _flat(s32, scales[n16:], torch.float32, g)
    return b16, v16, s16, b32, v32, s32, c["limit"] * norm


def _adamw_inputs(c, seed):
    g = _generator(seed)
    sizes, dt = _sizes(c["n"], c["numel"]), _dtype(c["grad"])
    p, _ = _flat(sizes, [0.02] * len(sizes), torch.float32, g)
    grad, _ = _flat(sizes, [1e-3] * len(sizes), dt, g)
    m, _ = _flat(sizes, [3e-4] * len(sizes), torch.float32, g)
    v, _ = _flat(sizes, [1e-3] * len(sizes), torch.float32, g)
    if c["steps"] == 0:
        m.zero_()
        v.zero_()
    else:
        v.square_()
    coef = torch.rand((1,), device=DEV, generator=g)
    return sizes, p, grad, m, v, coef


def prepare(case, seed):
    c = dict(case)
    if c["kind"] in ("score", "loss"):
        x, w, target, token_w = _loss_inputs(c, seed)
        return dict(c, x=x, w=w, target=target, token_w=token_w)
    if c["kind"] == "clip":
        b16, v16, s16, b32, v32, s32, max_norm = _clip_inputs(c, seed)
        o16, o32 = torch.empty_like(b16), torch.empty_like(b32)
        outs = (list(o16.split(s16)) if s16 else []) + (list(o32.split(s32)) if s32 else [])
        return dict(c, b16=b16, b32=b32, o16=o16, o32=o32, grads=v16 + v32, outs=outs, max_norm=max_norm)
    sizes, p, grad, m, v, coef = _adamw_inputs(c, seed)
    views = [list(b.split(sizes)) for b in (p, grad, m, v)]
    w16 = torch.empty_like(p, dtype=torch.bfloat16)
    return dict(c, p=p, g=grad, m=m, v=v, w16=w16, coef=coef, params=views[0], grads=views[1], ms=views[2], vs=views[3],
                weights=list(w16.split(sizes)), lr=torch.full((1,), LR, device=DEV),
                step=torch.full((1,), c["steps"], dtype=torch.int32, device=DEV))


# ---- plain forms -------------------------------------------------------------------------------------------------------
def _plain_loss(s):
    x, w = s["x"].float(), s["w"].float()
    kept = s["target"] >= 0
    at = s["target"].clamp(min=0).long().unsqueeze(1)
    z = x @ w.t()
    top = z.amax(1, keepdim=True)
    lse = top + (z - top).exp().sum(1, keepdim=True).log()
    zero = torch.zeros((), device=x.device)
    loss = torch.where(kept, (lse - z.gather(1, at)).squeeze(1), zero)
    lse_out = torch.where(kept, lse.squeeze(1), zero)
    if s["kind"] == "score":
        return {"loss": loss, "lse": lse_out}
    share = s["token_w"] if s["token_w"] is not None else 1.0 / kept.sum().clamp(min=1).float()
    c = torch.where(kept, share, zero)
    g = (z - lse).exp()
    g.scatter_add_(1, at, torch.full_like(at, -1.0, dtype=torch.float32))
    g *= c.unsqueeze(1)
    return {"total": (c * loss).sum(dtype=torch.float64).float(), "loss": loss, "lse": lse_out,
            "dx": (g @ w).to(s["x"].dtype), "d_w": (g.t() @ x).to(s["w"].dtype)}


def _plain_clip(s):
    a, b = s["b16"].float(), s["b32"]
    norm = ((a * a).sum(dtype=torch.float64) + (b * b).sum(dtype=torch.float64)).sqrt()
    coef = (s["max_norm"] / (norm + EPS_CLIP)).clamp(max=1.0)
    return {"norm": norm.float(), "coef": coef.float(), "out16": (a * coef.float()).to(torch.bfloat16), "out32": b * coef.float()}


def _plain_adamw(s):
    s["step"] += 1
    t = s["step"].double()
    c1, c2 = (1.0 - BETA1 ** t).float(), (1.0 - BETA2 ** t).float()
    g = s["g"].float() * s["coef"]
    s["m"].mul_(BETA1).add_(g * (1.0 - BETA1))
    s["v"].mul_(BETA2).add_(g * g * (1.0 - BETA2))
    s["p"].mul_(1.0 - s["lr"] * DECAY).sub_(s["lr"] * (s["m"] / c1) / ((s["v"] / c2).sqrt() + EPS))
    s["w16"].copy_(s["p"])
    return {"p": s["p"], "m": s["m"], "v": s["v"], "w16": s["w16"], "step": s["step"]}


# ---- the framework's calls: the handle (buffers, tables) is made once per state, as a user's program does ----------------
def _own_loss(s):
    from paper_2505_11432_amd.head import VocabLoss
    if "op" not in s:
        s["op"] = VocabLoss(s["T"], s["d"], s["V"], dtype=s["x"].dtype, grad_dtype=s["w"].dtype, device=DEV,
                            gradients=s["kind"] == "loss")
    op = s["op"]
    if s["kind"] == "score":
        loss, lse = op.score(s["x"], s["w"], s["target"])
        return {"loss": loss, "lse": lse}
    total = op.step(s["x"], s["w"], s["target"], token_w=s["token_w"])
    return {"total": total.view(()), "loss": op.loss, "lse": op.lse, "dx": op.dx, "d_w": op.d_w}


def _own_clip(s):
    from paper_2505_11432_amd.optim import GradClip
    if "op" not in s:
        s["op"] = GradClip(s["grads"], max_norm=s["max_norm"], out=s["outs"])
    op = s["op"]
    op.clip()
    return {"norm": op.norm.view(()), "coef": op.coef.view(()), "out16": s["o16"], "out32": s["o32"]}


def _own_adamw(s):
    from paper_2505_11432_amd.optim import AdamW
    if "op" not in s:
        s["op"] = AdamW(s["params"], s["grads"], s["ms"], s["vs"], weights=s["weights"], lr=s["lr"], betas=(BETA1, BETA2), eps=EPS,
                        weight_decay=DECAY, step=s["step"])
    s["op"].step(coef=s["coef"])
    return {"p": s["p"], "m": s["m"], "v": s["v"], "w16": s["w16"], "step": s["step"]}


def run(state):
    if own:
        return {"score": _own_loss, "loss": _own_loss, "clip": _own_clip, "adamw": _own_adamw}[state["kind"]](state)
    return {"score": _plain_loss, "loss": _plain_loss, "clip": _plain_clip, "adamw": _plain_adamw}[state["kind"]](state)


# ---- what a pass cannot do without ---------------------------------------------------------------------------------------
def work(case):
    c = case
    if c["kind"] in ("score", "loss"):
        T, d, V, es = c["T"], c["d"], c["V"], 4 if c["dtype"] == "f32" else 2
        rows = max(1.0, T * (1.0 - c["ignored"]))          # rows that count: the others give zeros
        read = rows * d * es + V * d * es + T * 4 + (T * 4 if c["weights"] and c["kind"] == "loss" else 0)
        if c["kind"] == "score":
            return {"bytes": read + 8 * T, "flops": 2.0 * rows * V * d}
        return {"bytes": read + 8 * T + T * d * es + V * d * es, "flops": 6.0 * rows * V * d}
    if c["kind"] == "clip":
        es = 4 - 2 * c["bf16"]
        return {"bytes": 2.0 * c["numel"] * es, "flops": 3.0 * c["numel"]}
    return {"bytes": c["numel"] * (26.0 + (4 if c["grad"] == "f32" else 2)), "flops": 15.0 * c["numel"]}


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------------
def _exact_loss(c, seed):
    x, w, target, token_w = _loss_inputs(c, seed)
    T, d, V = c["T"], c["d"], c["V"]
    W = w.double()
    loss, lse = torch.zeros(T, dtype=torch.float64, device=DEV), torch.zeros(T, dtype=torch.float64, device=DEV)
    grads = c["kind"] == "loss"
    counted = (target >= 0).nonzero().squeeze(1)
    dx = torch.zeros((T, d), dtype=torch.float64, device=DEV) if grads else None
    d_w = torch.zeros((V, d), dtype=torch.float64, device=DEV) if grads else None
    total = torch.zeros((), dtype=torch.float64, device=DEV)
    for rows in counted.split(max(1, 2 ** 29 // V)):
        xr, tr = x[rows].double(), target[rows].long()
        logp = torch.log_softmax(xr @ W.t(), dim=1)
        first = xr @ W[:1].t()
        at = torch.arange(len(rows), device=DEV)
        loss[rows] = -logp[at, tr]
        lse[rows] = (first - logp[:, :1]).squeeze(1)
        if grads:
            share = token_w[rows].double() if token_w is not None else torch.full_like(loss[rows], 1.0 / max(1, len(counted)))
            total += (share * loss[rows]).sum()
            logp.exp_()
            logp[at, tr] -= 1.0
            logp *= share[:, None]
            dx[rows] = logp @ W
            d_w += logp.t() @ xr
    if not grads:
        return {"loss": loss, "lse": lse}
    return {"total": total, "loss": loss, "lse": lse, "dx": dx, "d_w": d_w}


def _exact_clip(c, seed):
    b16, _, _, b32, _, _, max_norm = _clip_inputs(c, seed)
    norm = torch.sqrt(sum(t.double().square().sum() for b in (b16, b32) for t in b.split(2 ** 27)))
    coef = torch.minimum(torch.ones_like(norm), max_norm / (norm + EPS_CLIP))
    return {"norm": norm, "coef": coef, "out16": b16.double() * coef, "out32": b32.double() * coef}


def _exact_adamw(c, seed):
    _, p, grad, m, v, coef = _adamw_inputs(c, seed)
    t = c["steps"] + 1
    g = grad.double() * coef.double()
    m = m.double() * BETA1 + g * (1.0 - BETA1)
    v = v.double() * BETA2 + g.square() * (1.0 - BETA2)
    lr = float(torch.tensor(LR))
    p = p.double() * (1.0 - lr * DECAY) - lr * (m / (1.0 - BETA1 ** t)) / (torch.sqrt(v / (1.0 - BETA2 ** t)) + EPS)
    return {"p": p, "m": m, "v": v, "w16": p, "step": None}


def exact(case, seed):
    return {"score": _exact_loss, "loss": _exact_loss, "clip": _exact_clip, "adamw": _exact_adamw}[case["kind"]](dict(case), seed)
