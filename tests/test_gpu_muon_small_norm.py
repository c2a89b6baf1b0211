"""Muon of matrices whose update is next to nothing: X = u / max(|u|, eps), so it fades where there is no gradient (an expert without tokens).

Tolerance: that of an orthogonalised matrix (test_gpu_muon: `rounded`, the steps with what is kept changed by its rounding), and what 16 bits leave of small
numbers.  In units of 2^12 those below 2^-14 are multiples of 2^-24, off by up to 2^-25: of A and R, m entries each, 2^-37 m of A (2-norm), with b / a = 1.4 and five
steps less than 2^-34 m of the outcome; of X, whose rest is times 2^11 in a number of its own, 2^-48 of an element, multiplied by at most 485."""
import math

import pytest
import torch

from test_gpu_muon import DEV, STEPS, formula, rounded

EPS = 1e-7
SHAPES = [(3, 40, 100), (2, 300, 64), (2, 130, 70), (1, 260, 300), (1, 1500, 2100)]


def make(shape, m, grad, **k):
    from paper_2505_11432_amd.optim import Muon
    p = torch.zeros(shape, device=DEV)
    return p, Muon([p], [grad], [m], lr=1.0, weight_decay=0.0, scale=1.0, **k)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES)
def test_no_gradient_and_what_is_left_of_the_momentum(shape):
    """0.95 times nine of the smallest numbers is nine of them again: such a momentum stays for good, and moves nothing."""
    g = torch.Generator(device=DEV).manual_seed(1)
    m = torch.where(torch.rand(shape, device=DEV, generator=g) < 0.5, -1.0, 1.0) * 9 * 2.0 ** -149
    was = m.clone()
    p, op = make(shape, m, torch.zeros_like(m))
    p.normal_(generator=g)
    before = p.clone()
    op.step()
    assert torch.equal(m, was) and bool((m != 0).all())
    assert torch.equal(p, before)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("size", [4.0, 1.0, 0.5, 1e-2, 1e-4])
def test_norms_around_eps(shape, size):
    """p = 0, lr = scale = 1 and no momentum: p becomes -O(grad)."""
    g = torch.Generator(device=DEV).manual_seed(2)
    grad = torch.randn(shape, device=DEV, generator=g)
    grad *= size * EPS / grad.double().square().sum((1, 2), keepdim=True).sqrt().float()
    p, op = make(shape, torch.zeros(shape, device=DEV), grad, momentum=0.0)
    op.step()
    for i in range(shape[0]):
        u = grad[i].double()
        flip = u.shape[0] > u.shape[1]
        x = (u.t().contiguous() if flip else u) / max(float(u.norm()), EPS)
        want = formula(x, STEPS)
        norm, m = float(want.norm()), min(x.shape)
        tol = 2.0 * float((rounded(x, STEPS, False) - want).norm()) + (2.0 ** -22 * math.sqrt(max(x.shape)) + 2.0 ** -34 * m) * norm
        tol += 485 * 2.0 ** -48 * math.sqrt(x.numel())
        got = -(p[i].double().t() if flip else p[i].double())
        assert float((got - want).norm()) <= tol


@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES[:4])
def test_eps_of_the_caller(shape):
    """eps = 0: a direction of any length; above eps its value changes nothing."""
    g = torch.Generator(device=DEV).manual_seed(3)
    grad = torch.randn(shape, device=DEV, generator=g) * 2.0 ** -60
    outs = []
    for u, eps in ((grad, 0.0), (grad * 2.0 ** 60, 0.0), (grad * 2.0 ** 60, EPS)):
        p, op = make(shape, torch.zeros(shape, device=DEV), u, momentum=0.0, eps=eps)
        op.step()
        outs.append(p)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[1], outs[2]) and bool((outs[0] != 0).any())
