"""Orthogonalised updates and Muon against their formulas in 64 bits.

Tolerance of an orthogonalised matrix, in the 2-norm of all elements: what a step adds and what it multiplies earlier errors by.  A step keeps
A = X X^T and R = b A + c A^2 in 11 bits: a rounding is at most half a step of 2^-11 of its element, 2^-11 / sqrt(3) in the root mean square over
many elements that round independently.  With s the largest singular value of X and |.| the 2-norm of all elements:
  dA <= r sqrt(|A|^2 + 2 s^2 |X|^2)  (A's own rounding, and that of the operand on either side),  r = 2^-11 / sqrt(3)
  dR <= (|b| + 2 |c| s^2) dA + r |R|
  added: s dR + r |R X| (the operand of R X) + 2^-21 |X| (X itself is carried in 22 bits)
Earlier errors are multiplied by at most the largest slope of a s + b s^3 + c s^5 on the singular values' range (Lipschitz constant of the matrix function).
Two adjacent steps may be taken on the powers of one A, whose error then passes through both polynomials: twice the above.  fp32
accumulation adds up to 2^-24 sqrt(n) of the products' sizes, which a factor of 1.1 covers.  A result in bf16 adds half a step, 2^-8 of each element."""
import math

import pytest
import torch

DEV = "cuda:0"
STEPS = ((3.4445, -4.7750, 2.0315),) * 5
R16 = 2.0 ** -11 / math.sqrt(3.0)


def exact(u, steps=STEPS):
    """(orthogonalised matrix, its tolerance) in 64 bits."""
    u = u.double()
    flip = u.shape[0] > u.shape[1]
    x = u.t() if flip else u
    size = x.norm()
    x = x / size if float(size) > 0 else x
    off = 0.0
    for a, b, c in steps:
        s = float(torch.linalg.matrix_norm(x, 2)) if float(size) > 0 else 0.0
        gram = x @ x.t()
        r = b * gram + c * gram @ gram
        d_gram = R16 * math.sqrt(float(gram.norm()) ** 2 + 2 * s ** 2 * float(x.norm()) ** 2)
        d_r = (abs(b) + 2 * abs(c) * s ** 2) * d_gram + R16 * float(r.norm())
        v = torch.linspace(0, max(s, 1e-3), 2001, dtype=torch.float64)
        slope = float((a + 3 * b * v ** 2 + 5 * c * v ** 4).abs().max())
        off = slope * off + s * d_r + R16 * float((r @ x).norm()) + 2.0 ** -21 * float(x.norm())
        x = a * x + r @ x
    return (x.t() if flip else x), 2.2 * off


def matrices(batch, rows, cols, kind, seed=0, dtype=torch.float32):
    g = torch.Generator(device=DEV).manual_seed(seed)
    r = min(rows, cols)
    i = torch.arange(1, r + 1, device=DEV, dtype=torch.float32)
    value = {"flat": i ** 0, "falling": i ** -0.5, "steep": i ** -1.5, "low rank": (i <= max(1, r // 8)).float()}[kind]
    x = torch.randn((batch, rows, r), device=DEV, generator=g) * value @ torch.randn((batch, r, cols), device=DEV, generator=g)
    return (x * 10.0 ** torch.randint(-7, 3, (batch, 1, 1), device=DEV, generator=g)).to(dtype)


SHAPES = [(1, 1, 1), (3, 1, 7), (2, 5, 1), (2, 16, 16), (1, 64, 2048), (5, 100, 131), (3, 257, 129), (2, 128, 128), (2, 384, 256), (1, 300, 1000), (1, 1030, 515),
          (9, 65, 64)]


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["flat", "falling", "steep", "low rank"])
@pytest.mark.parametrize("batch,rows,cols", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_orthogonal(batch, rows, cols, kind, dtype):
    from paper_2505_11432_amd.optim import Orthogonal
    x = matrices(batch, rows, cols, kind, dtype=dtype)
    op = Orthogonal(batch, rows, cols, out_dtype=torch.float32, device=DEV)
    op.workspace.fill_(255)
    out = op.apply(x).clone()
    for i in range(batch):
        want, tol = exact(x[i])
        assert float((out[i].double() - want).norm()) <= tol, i
    short = Orthogonal(batch, rows, cols, out_dtype=torch.bfloat16, max_bytes=1, device=DEV)          # a matrix at a time
    assert torch.equal(short.apply(x), out.to(torch.bfloat16))
    op.workspace.zero_()
    assert torch.equal(op.apply(x), out)


@pytest.mark.gpu
def test_zeros_scale_and_bad_matrices():
    """A matrix of zeros stays one; a power of two in front changes nothing; an infinite or NaN element spoils its own matrix alone."""
    from paper_2505_11432_amd.optim import Orthogonal
    x = matrices(5, 70, 90, "falling")
    x /= x.square().sum((1, 2), keepdim=True).sqrt()
    op = Orthogonal(5, 70, 90, out_dtype=torch.float32, device=DEV)
    want = op.apply(x).clone()
    for k in (-100, -40, 50):
        assert torch.equal(op.apply(x * 2.0 ** k), want)
    x[1] = 0
    x[2, 3, 4] = float("inf")
    x[3, 0, 0] = float("nan")
    out = op.apply(x)
    assert torch.equal(out[0], want[0]) and torch.equal(out[4], want[4]) and bool((out[1] == 0).all())
    assert bool(torch.isnan(out[2]).any()) and bool(torch.isnan(out[3]).any())


@pytest.mark.gpu
@pytest.mark.parametrize("steps", [((2.0, -1.5, 0.5),), ((1.5, -0.5, 0.0),) * 12, ((3.4445, -4.7750, 2.0315),) * 2 + ((2.0, -1.5, 0.5),) * 3, ((1.0, 0.0, 0.0),) * 16])
def test_other_coefficients(steps):
    from paper_2505_11432_amd.optim import Orthogonal
    x = matrices(2, 130, 200, "flat")
    out = Orthogonal(2, 130, 200, out_dtype=torch.float32, coefficients=steps, device=DEV).apply(x)
    for i in range(2):
        want, tol = exact(x[i], steps)
        assert float((out[i].double() - want).norm()) <= tol


@pytest.mark.gpu
@pytest.mark.parametrize("batch,rows,cols", [(1, 3, 2), (4, 40, 100), (2, 257, 129), (1, 129, 515), (3, 128, 256)])
@pytest.mark.parametrize("grad_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("offset", [0, 1])
def test_muon(batch, rows, cols, grad_dtype, nesterov, offset):
    """m: two products, one sum: 3 * 2^-24 of its terms.  p: 2^-22 of |p| and the orthogonalised update's tolerance times lr scale, the update from the
    momentum as it was written."""
    from paper_2505_11432_amd.optim import Muon
    n = batch * rows * cols
    shape = (batch, rows, cols) if batch > 1 else (rows, cols)
    g = torch.Generator(device=DEV).manual_seed(4)
    make = lambda dt, s: ((torch.randn((n + 4,), device=DEV, generator=g) * s).to(dt))
    bufs = [make(torch.float32, 0.05), make(grad_dtype, 1e-3), make(torch.float32, 1e-3), make(torch.bfloat16, 1.0)]
    p, grad, m, w = (b[offset:offset + n].view(shape) for b in bufs)
    lr, mu, wd, coef = float(torch.tensor(0.02)), 0.9, 0.1, 0.625
    ends = [b[[0, -1]].clone() if offset else b[-4:].clone() for b in bufs]
    op = Muon([p], [grad], [m], weights=[w], lr=lr, momentum=mu, nesterov=nesterov, weight_decay=wd, device=DEV)
    factor = torch.full((1,), coef, device=DEV)
    for _ in range(2):
        p0, m0, g0 = p.double().clone(), m.double().clone(), grad.double() * coef
        op.step(coef=factor)
        assert bool(((m.double() - (mu32 := float(torch.tensor(mu))) * m0 - g0).abs() <= 3 * 2.0 ** -24 * (mu * m0.abs() + g0.abs())).all())
        u = g0 + mu32 * m.double() if nesterov else m.double()
        scale = 0.2 * max(rows, cols) ** 0.5
        for i in range(batch):
            at = (lambda t: t[i]) if batch > 1 else (lambda t: t)
            o, tol = exact(at(u))
            want = at(p0) * (1 - lr * wd) - lr * scale * o
            # (u itself is rounded: 2^-23 of its terms, which the steps multiply by at most 4^5)
            extra = 1024 * 2.0 ** -23 * float((at(g0).abs() + at(m).double().abs()).norm() / at(u).norm())
            assert float((at(p).double() - want).norm()) <= 2.0 ** -22 * float(at(p0).norm()) + lr * scale * (tol + extra)
        assert torch.equal(w, p.to(torch.bfloat16))
    for b, e in zip(bufs, ends):
        assert torch.equal(b[[0, -1]] if offset else b[-4:], e)


@pytest.mark.gpu
def test_list_and_left_out_update():
    from paper_2505_11432_amd.optim import Muon
    shapes = [(4, 64, 48), (30, 70), (2, 3, 16, 40), (0, 8, 8)]
    dts = [torch.bfloat16, torch.float32, torch.float32, torch.float32]
    p = [torch.randn(s, device=DEV) for s in shapes]
    g = [torch.randn(s, device=DEV).to(t) for s, t in zip(shapes, dts)]
    m = [torch.zeros_like(t) for t in p]
    w = [torch.zeros_like(p[0], dtype=torch.bfloat16), None, torch.zeros_like(p[2], dtype=torch.bfloat16), None]
    op = Muon(p, g, m, weights=w, lr=torch.full((1,), 0.1, device=DEV))
    was = [t.clone() for t in p + m + w[::2]]
    op.step(coef=torch.full((1,), float("nan"), device=DEV))
    for a, b in zip(was, p + m + w[::2]):
        assert torch.equal(a, b)
    op.step()
    for i, s in enumerate(shapes[:3]):
        alone = Muon([q := was[i].clone()], [g[i]], [torch.zeros_like(m[i])], lr=0.1)
        alone.step()
        assert torch.equal(q, p[i]) and not torch.equal(q, was[i])
        if w[i] is not None:
            assert torch.equal(w[i], p[i].to(torch.bfloat16))
    op = Muon([], [], [])
    op.step()


@pytest.mark.gpu
def test_captured_twice_and_replayed():
    from paper_2505_11432_amd.optim import GradClip, Muon

    def state(seed):
        g = torch.Generator(device=DEV).manual_seed(seed)
        p, grad, m = (torch.randn((3, 130, 70), device=DEV, generator=g) for _ in range(3))
        clip, lr = GradClip([grad], 5.0), torch.full((1,), 1e-2, device=DEV)
        return p, grad, m, lr, clip, Muon([p], [grad], [m], lr=lr)

    def step(s):
        s[4].clip()
        s[5].step(coef=s[4].coef)

    eager, replayed = [state(1), state(2)], [state(1), state(2)]
    graphs = []
    for a, b in zip(eager, replayed):
        step(a)
        step(b)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(b)
        graphs.append(graph)
    for r in range(3):
        for i, (a, b) in enumerate(zip(eager, replayed)):
            b[1].copy_(a[1].normal_())
            a[3].fill_(1e-2 / (r + 1))
            b[3].copy_(a[3])
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager, replayed):
            step(a)
            assert torch.equal(a[0], b[0]) and torch.equal(a[2], b[2])


@pytest.mark.gpu
def test_refused():
    from paper_2505_11432_amd import binding as B
    from paper_2505_11432_amd.optim import Muon, Orthogonal
    x = torch.randn((2, 8, 8), device=DEV)
    y, z = x.clone(), x.clone()
    for bad in (lambda: Muon([x], [y], [x]), lambda: Muon([x], [x], [y]), lambda: Muon([x], [y], [z[:, :4]]), lambda: Muon([x], [y], [z], weights=[z]),
                lambda: Muon([x[0, 0]], [y[0, 0]], [z[0, 0]]), lambda: Muon([x], [y], [z, z]), lambda: Muon([x], [y], [z], lr=torch.zeros((2,), device=DEV)),
                lambda: Muon([x], [y], [z], coefficients=()), lambda: Muon([x], [y], [z], coefficients=((1.0, 2.0),)),
                lambda: Muon([x.transpose(1, 2)], [y], [z]), lambda: Muon([x.to(torch.bfloat16)], [y], [z]), lambda: Orthogonal(1, 0, 4, device=DEV),
                lambda: Orthogonal(1, 8, 8, out_dtype=torch.float16, device=DEV), lambda: Orthogonal(2, 8, 8, device=DEV).apply(x[:1]),
                lambda: Orthogonal(2, 8, 8, device=DEV).apply(x.cpu())):
        with pytest.raises(AssertionError):
            bad()
    with pytest.raises(TypeError):
        Muon([x], [y.half()], [z])
    # products that leave the range of what is kept
    for c in (((20.0, 0.0, 0.0),), ((3.0, 0.0, 0.0),) * 3, ((float("nan"), 0.0, 0.0),)):
        with pytest.raises(B.MoEError) as e:
            Orthogonal(2, 8, 8, coefficients=c, device=DEV).apply(x)
        assert e.value.status == -2
    out = torch.empty((4, 8, 8), device=DEV)
    with pytest.raises(B.MoEError):
        B.moe_orthogonalize(out[:2], out[1:3], torch.empty((1 << 20,), dtype=torch.uint8, device=DEV))
    with pytest.raises(B.MoEError):
        B.moe_orthogonalize(x, out[:2], torch.empty((1 << 10,), dtype=torch.uint8, device=DEV))
    with pytest.raises(TypeError):
        B._native.moe_orthogonalize(x, 0, 2, 8, 8, 1, x, 0, out[:2], 0, out, 1 << 20)
