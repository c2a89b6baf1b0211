"""The step of train.py: layer, vocabulary loss, clipping and update together."""
import math

import pytest
import torch

DEV = "cuda:0"


def batches(T, V, n, seed=1):
    g = torch.Generator(device=DEV).manual_seed(seed)
    follow = torch.randperm(V, device=DEV, generator=g)
    for _ in range(n):
        tokens = torch.randint(0, V, (T,), device=DEV, generator=g)
        target = follow[tokens]
        target[torch.rand((T,), device=DEV, generator=g) < 0.1] = -100
        yield tokens, target


def make(T, V, dtype):
    from paper_2505_11432_amd.train import TrainStep
    return TrainStep(T, 128, 4, 2, 144, V, dtype=dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_it_learns(dtype):
    """A permutation of 300 words from 400 tokens a step: from about log 300 to under half of it within 40 steps."""
    T, V = 400, 300
    model = make(T, V, dtype)
    losses = []
    for tokens, target in batches(T, V, 40):
        model.load(tokens, target)
        loss, norm = model.step()
        losses.append(float(loss))
        assert math.isfinite(float(norm)) and float(norm) > 0
    assert losses[0] > math.log(V) - 1.0
    assert losses[-1] < losses[0] / 2
    assert int(model.adamw.step_count) == 40


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_one_step_against_64_bits(dtype):
    """The first update of the vocabulary matrix from the hidden rows that the step made: loss, gradient, norm over all gradients, factor and
    AdamW by their formulas.  d_w is G^T hidden with G rounded to bf16 once (2^-8), in fp32 data 2^-16; the first AdamW step is
    lr g / (|g| + eps'), so it is compared where |g| is well above its error."""
    T, V = 200, 150
    model = make(T, V, dtype)
    was = [p.clone() for p in model.masters]
    w_used = model.params[3].clone()
    tokens, target = next(batches(T, V, 1))
    model.load(tokens, target)
    loss, norm = model.step()
    h, w, tg = model.hidden.double().cpu(), w_used.double().cpu(), target.cpu()
    keep = (tg >= 0).nonzero().squeeze(1)
    z = h[keep] @ w.t()
    logp = torch.log_softmax(z, 1)
    want = -logp[torch.arange(len(keep)), tg[keep]].mean()
    assert abs(float(loss) - float(want)) <= 2.0 ** -16 * max(1.0, float(z.abs().max()))
    g = logp.exp()
    g[torch.arange(len(keep)), tg[keep]] -= 1
    d_w = (g / len(keep)).t() @ h[keep]
    tol = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -16
    got = model.head.d_w.double().cpu()
    assert float((got - d_w).norm()) <= tol * float(d_w.norm())
    grads = [t.double() for t in (model.layer.d_w_r, model.layer.d_w1, model.layer.d_w2, model.head.d_w)]
    full = math.sqrt(sum(float(t.square().sum()) for t in grads))
    assert abs(float(norm) - full) <= 2.0 ** -23 * full
    coef = min(1.0, 1.0 / (full + 1e-6))
    lr = float(model.lr)
    for p, old, t in zip(model.masters, was, grads):
        c = t * coef
        step = lr * c / (c.abs() + 1e-8)
        # the update: some roundings of it, and what eps makes of a gradient near it
        assert float((p.double() - (old.double() - step)).abs().max()) <= 2.0 ** -21 * (float(old.abs().max()) + lr)
    if dtype == torch.bfloat16:
        for p, q in zip(model.params, model.masters):
            assert torch.equal(p, q.to(dtype))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_replayed_from_a_graph(dtype):
    T, V = 300, 200
    eager, graph = make(T, V, dtype), make(T, V, dtype)
    for i, (tokens, target) in enumerate(batches(T, V, 6)):
        for m in (eager, graph):
            m.load(tokens, target)
        if i == 1:
            graph.capture()
        a = [t.clone() for t in eager.step()]
        b = [t.clone() for t in graph.step()]
        torch.cuda.synchronize()
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        for p, q in zip(eager.masters, graph.masters):
            assert torch.equal(p, q)
