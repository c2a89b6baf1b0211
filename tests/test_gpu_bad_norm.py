"""A step whose gradient norm is infinite or NaN changes nothing, eagerly and from a graph, and the next one goes on."""
import math

import pytest
import torch

DEV = "cuda:0"


def lists(sizes, grad_dtype):
    g = torch.Generator(device=DEV).manual_seed(3)
    p, m, v = ([torch.randn((n,), device=DEV, generator=g) * 0.02 for n in sizes] for _ in range(3))
    return p, [torch.randn((n,), device=DEV, generator=g).to(grad_dtype) for n in sizes], m, [t.square_() for t in v]


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", [[5], [40_003, 0, 17], [3_000_001]])
@pytest.mark.parametrize("grad_dtype", [torch.float32, torch.bfloat16])
def test_update_left_out(sizes, grad_dtype):
    from paper_2505_11432_amd.optim import AdamW
    p, g, m, v = lists(sizes, grad_dtype)
    w = [t.to(torch.bfloat16) for t in p]
    g[0][1] = float("inf")
    op = AdamW(p, g, m, v, weights=w)
    was = [t.clone() for t in p + m + v + w]
    coef = torch.full((1,), float("nan"), device=DEV)
    for _ in range(3):
        op.step(coef=coef)
    assert int(op.step_count) == 0 and not bool(op.workspace.any())
    assert all(torch.equal(a, b) for a, b in zip(was, p + m + v + w))
    g[0][1] = 0.5
    coef.fill_(0.5)
    other = AdamW(*[[t.clone() for t in x] for x in (p, g, m, v)])
    op.step(coef=coef)
    other.step(coef=coef)
    assert int(op.step_count) == 1 and all(torch.equal(a, b) for a, b in zip(p + m + v, other.params + other.m + other.v))
    assert not torch.equal(was[0], p[0])


def trainer(dtype):
    from paper_2505_11432_amd.train import TrainStep
    return TrainStep(300, 128, 4, 2, 144, 200, dtype=dtype)


def state(model):
    return [t.clone() for t in model.masters + model.adamw.m + model.adamw.v + model.params]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("graph", [0, 1])
def test_training_goes_on(dtype, graph):
    model, clean = trainer(dtype), trainer(dtype)
    g = torch.Generator(device=DEV).manual_seed(1)
    batches = [(torch.randint(0, 200, (300,), device=DEV, generator=g), torch.randint(0, 200, (300,), device=DEV, generator=g)) for _ in range(5)]
    for i, (tokens, target) in enumerate(batches):
        for m in (model, clean):
            m.load(tokens, target)
        if i == 1 and graph:
            model.capture()
        if i == 2:                           # the bad one
            before = state(model)
            model.x[5] = float("nan")
            loss, norm = model.step()
            assert math.isnan(float(loss)) and not math.isfinite(float(norm))
            assert int(model.adamw.step_count) == 2 and all(torch.equal(a, b) for a, b in zip(before, state(model)))
            continue
        model.step()
        clean.step()
        torch.cuda.synchronize()
    assert int(model.adamw.step_count) == int(clean.adamw.step_count) == 4
    assert all(torch.equal(a, b) for a, b in zip(state(model), state(clean)))


@pytest.mark.gpu
def test_infinite_norm(monkeypatch):
    """The factor of an infinite norm is 0, with which infinite gradients would make NaN."""
    model = trainer(torch.float32)
    model.load(torch.arange(300, device=DEV) % 200, torch.arange(300, device=DEV) % 200)
    before = state(model)
    clip = model.clip.clip

    def overflowed():
        model.layer.d_w1.view(-1)[7] = float("inf")
        return clip()

    monkeypatch.setattr(model.clip, "clip", overflowed)
    _, norm = model.step()
    assert float(norm) == math.inf and float(model.clip.coef) == 0.0
    assert int(model.adamw.step_count) == 0 and all(torch.equal(a, b) for a, b in zip(before, state(model)))
