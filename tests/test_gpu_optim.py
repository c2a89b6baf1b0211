"""Clipping and the AdamW update against their formulas in 64 bits.

Tolerances: norm and coef are sums in 64 bits rounded once to fp32, coef goes through the rounded product: 2^-23 relative.  Clipped gradients:
the factor's rounding and the product's, 2^-23 relative in fp32, 2^-8 + 2^-23 in bf16 (element by element).  AdamW: m and v three roundings of
2^-24 of the larger of their terms each; p the same plus the update's: 8 roundings of at most |p| + |update|, 2^-21 of that, the update taken with the
larger of m's two terms, which may cancel (no fixed multiple of lr bounds it: where v and g are near 0 it reaches hundreds of lr); weights are p
rounded."""
import math
import random

import pytest
import torch

DEV = "cuda:0"
LISTS = [[1], [5], [4, 3, 0, 7], [0, 0, 1], [4096], [2047, 2049, 1], [100_003, 17, 0, 65_536, 9], [1] * 300, list(range(0, 260)), [3_000_001, 8, 1_500_007]]


def views(sizes, dtype, offset, seed, scale=1.0):
    """Tensors one after another in one buffer from element `offset` on: any alignment."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    buf = (torch.randn((sum(sizes) + offset,), device=DEV, generator=g) * scale).to(dtype)
    return buf, list(buf[offset:].split(sizes))


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", LISTS)
@pytest.mark.parametrize("offset", [0, 1, 3])
@pytest.mark.parametrize("limit", [0.3, 5.0])
def test_clip(sizes, offset, limit):
    from paper_2505_11432_amd.optim import GradClip
    buf, grads = views(sizes, torch.float32, offset, 1)
    buf16, grads16 = views(sizes, torch.bfloat16, offset, 2)
    all_grads = [t for pair in zip(grads, grads16) for t in pair]
    outs = [torch.full_like(t, 7.0) for t in all_grads]
    want = math.sqrt(sum(float(t.double().square().sum()) for t in all_grads))
    max_norm = limit * want
    op = GradClip(all_grads, max_norm, out=outs)
    before = buf.clone(), buf16.clone()
    op.clip()
    coef = min(1.0, max_norm / (want + 1e-6))
    assert abs(float(op.norm) - want) <= 2.0 ** -23 * want
    assert abs(float(op.coef) - coef) <= 2.0 ** -23 * coef
    for g, o in zip(all_grads, outs):
        tol = 2.0 ** -23 if g.dtype == torch.float32 else 2.0 ** -8 + 2.0 ** -23
        assert bool(((o.double() - g.double() * coef).abs() <= tol * (g.double() * coef).abs()).all())
    assert torch.equal(buf, before[0]) and torch.equal(buf16, before[1])
    # the norm and the factor alone, and in place
    alone = GradClip(all_grads, max_norm)
    alone.clip()
    assert torch.equal(alone.norm, op.norm) and torch.equal(alone.coef, op.coef)
    inplace = GradClip(all_grads, max_norm, out=all_grads)
    inplace.clip()
    assert torch.equal(inplace.norm, op.norm)
    for g, o in zip(all_grads, outs):
        assert torch.equal(g, o)
    assert torch.equal(buf[:offset], before[0][:offset])


@pytest.mark.gpu
def test_clip_extremes():
    from paper_2505_11432_amd.optim import GradClip
    big = torch.full((1000,), 2.0 ** 100, device=DEV)
    op = GradClip([big], 1.0)
    op.clip()
    assert abs(float(op.norm) / (2.0 ** 100 * math.sqrt(1000)) - 1) <= 2.0 ** -23
    small = torch.full((1000,), 2.0 ** -120, device=DEV)
    op = GradClip([small], 1.0, out=[torch.empty_like(small)])
    op.clip()
    assert abs(float(op.norm) / (2.0 ** -120 * math.sqrt(1000)) - 1) <= 2.0 ** -23 and float(op.coef) == 1.0
    zero = torch.zeros((77,), device=DEV)
    op = GradClip([zero], 1.0, out=[zero])
    op.clip()
    assert float(op.norm) == 0.0 and float(op.coef) == 1.0
    for bad, coef in ((float("nan"), None), (float("inf"), 0.0)):
        zero[3] = bad
        op.clip()
        assert not math.isfinite(float(op.norm))
        assert math.isnan(float(op.coef)) if coef is None else float(op.coef) == coef
        zero.zero_()
    op = GradClip([], 1.0)
    op.clip()
    assert float(op.norm) == 0.0 and float(op.coef) == 1.0


def adamw_reference(p, g, m, v, t, lr, betas, eps, wd, coef):
    p, g, m, v = p.double(), g.double() * coef, m.double(), v.double()
    m = m * betas[0] + g * (1 - betas[0])
    v = v * betas[1] + g * g * (1 - betas[1])
    p = p * (1 - lr * wd) - lr * (m / (1 - betas[0] ** t)) / ((v / (1 - betas[1] ** t)).sqrt() + eps)
    return p, m, v


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", LISTS)
@pytest.mark.parametrize("grad_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("offsets", [(0, 0, 0, 0, 0), (1, 1, 1, 1, 1), (0, 3, 1, 2, 1)])
def test_adamw(sizes, grad_dtype, offsets):
    from paper_2505_11432_amd.optim import AdamW
    pb, p = views(sizes, torch.float32, offsets[0], 1, 0.02)
    gb, g = views(sizes, grad_dtype, offsets[1], 2, 1e-3)
    mb, m = views(sizes, torch.float32, offsets[2], 3, 3e-4)
    vb, v = views(sizes, torch.float32, offsets[3], 4, 1e-3)
    vb.square_()
    wb, w = views(sizes, torch.bfloat16, offsets[4], 5)
    lr, betas, eps, wd, start = 3e-4, (0.9, 0.95), 1e-8, 0.1, 6
    lr = float(torch.tensor(lr))
    coef = torch.full((1,), 0.625, device=DEV)
    step = torch.full((1,), start, dtype=torch.int32, device=DEV)
    op = AdamW(p, g, m, v, weights=w, lr=lr, betas=betas, eps=eps, weight_decay=wd, step=step)
    for t in (start + 1, start + 2):
        was = [(a.clone(), b.clone(), c.clone()) for a, b, c in zip(p, m, v)]
        op.step(coef=coef)
        assert int(step) == t
        for i in range(len(sizes)):
            rp, rm, rv = adamw_reference(was[i][0], g[i], was[i][1], was[i][2], t, lr, betas, eps, wd, 0.625)
            big_m = torch.maximum(was[i][1].double().abs(), g[i].double().abs())
            big_v = torch.maximum(was[i][2].double(), g[i].double().square())
            assert bool(((m[i].double() - rm).abs() <= 3 * 2.0 ** -24 * big_m).all())
            assert bool(((v[i].double() - rv).abs() <= 4 * 2.0 ** -24 * big_v).all())
            update = lr * big_m / (1 - betas[0] ** t) / ((rv / (1 - betas[1] ** t)).sqrt() + eps)
            assert bool(((p[i].double() - rp).abs() <= 2.0 ** -21 * (was[i][0].double().abs() + update)).all())
            assert torch.equal(w[i], p[i].to(torch.bfloat16))
    for b, o in ((pb, offsets[0]), (mb, offsets[2])):
        ref = views(sizes, torch.float32, o, 1 if b is pb else 3, 0.02 if b is pb else 3e-4)[0]
        assert torch.equal(b[:o], ref[:o])


@pytest.mark.gpu
def test_adamw_first_step_without_weights_and_empty():
    from paper_2505_11432_amd.optim import AdamW
    p = torch.randn((1000,), device=DEV)
    g = torch.randn((1000,), device=DEV)
    m, v = torch.zeros_like(p), torch.zeros_like(p)
    was = p.clone()
    op = AdamW([p], [g], [m], [v], lr=1e-2, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.0)
    op.step()
    # the first update is lr * sign(g), up to eps / |g| and a few roundings
    want = was.double() - float(torch.tensor(1e-2)) * g.double() / (g.double().abs() + 1e-8)
    assert float((p.double() - want).abs().max()) <= 2.0 ** -21 * max(1.0, float(want.abs().max()))
    op = AdamW([], [], [], [])
    op.step()
    assert int(op.step_count) == 1
    op.step()
    assert int(op.step_count) == 2


@pytest.mark.gpu
def test_clip_and_update_in_a_graph():
    """A captured clip and update, replayed with other gradients and learning rates: every replay equals the eager calls."""
    from paper_2505_11432_amd.optim import AdamW, GradClip
    sizes = [5000, 17, 0, 70_001]

    def state():
        p, m, v = (views(sizes, torch.float32, 0, s, 0.02)[1] for s in (1, 2, 3))
        for t in v:
            t.square_()
        g = views(sizes, torch.float32, 0, 4)[1]
        clip = GradClip(g, 10.0)
        lr = torch.full((1,), 1e-3, device=DEV)
        return p, g, m, v, lr, clip, AdamW(p, g, m, v, lr=lr)

    a, b = state(), state()
    a[5].clip(); a[6].step(coef=a[5].coef)
    b[5].clip(); b[6].step(coef=b[5].coef)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a[5].clip()
        a[6].step(coef=a[5].coef)
    for i in range(4):
        for s in (a, b):
            for j, t in enumerate(s[1]):
                t.copy_(views([t.numel()], torch.float32, 0, 50 + 10 * i + j)[1][0])
            s[4].fill_(1e-3 / (i + 1))
        graph.replay()
        torch.cuda.synchronize()
        b[5].clip()
        b[6].step(coef=b[5].coef)
        assert int(a[6].step_count) == int(b[6].step_count) == i + 2
        for x, y in zip(a[0] + a[2] + a[3], b[0] + b[2] + b[3]):
            assert torch.equal(x, y)


@pytest.mark.gpu
def test_refused_lists():
    from paper_2505_11432_amd.optim import AdamW, GradClip
    x = torch.zeros((8, 8), device=DEV)
    for bad in (lambda: GradClip([x.t()[:, :4]], 1.0), lambda: GradClip([x], 1.0, out=[x.to(torch.bfloat16)]), lambda: GradClip([x], 1.0, out=[x[:4]]),
                lambda: GradClip([x], 1.0, out=[x, x]), lambda: AdamW([x], [x[:4]], [x], [x]), lambda: AdamW([x], [x], [x.to(torch.bfloat16)], [x]),
                lambda: AdamW([x], [x], [x], [x], weights=[x]), lambda: AdamW([x, x], [x, x.to(torch.bfloat16)], [x, x], [x, x]),
                lambda: AdamW([x], [x], [x], [x], lr=torch.zeros((2,), device=DEV)), lambda: GradClip([x.cpu()], 1.0)):
        with pytest.raises(AssertionError):
            bad()
    with pytest.raises(TypeError):
        GradClip([x.half()], 1.0)


@pytest.mark.gpu
def test_past_32_bits():
    """One tensor of more than 2^31 elements and a small one behind it: norm, clipped gradients and the update at both ends of the large one."""
    from paper_2505_11432_amd.optim import AdamW, GradClip
    big, small = 2 ** 31 + 5003, 777
    g = [torch.empty((n,), dtype=torch.bfloat16, device=DEV).normal_(0.0, 1e-3) for n in (big, small)]
    p, m, v = ([torch.empty((n,), device=DEV).normal_(0.0, 0.02) for n in (big, small)] for _ in range(3))
    for t in v:
        t.square_()
    want = math.sqrt(sum(float(part.double().square().sum()) for t in g for part in t.split(2 ** 28)))
    out = [torch.empty_like(t) for t in g]
    clip = GradClip(g, 0.5 * want, out=out)
    clip.clip()
    coef = 0.5 * want / (want + 1e-6)
    assert abs(float(clip.norm) - want) <= 2.0 ** -23 * want and abs(float(clip.coef) - coef) <= 2.0 ** -23 * coef
    places = [slice(0, 4099), slice(2 ** 31 - 2048, 2 ** 31 + 2048), slice(big - 5000, big)]
    was = [[t[0][s].clone() for t in (p, m, v)] for s in places] + [[t[1].clone() for t in (p, m, v)]]
    lr = float(torch.tensor(1e-3))
    AdamW(p, g, m, v, lr=lr, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1).step(coef=clip.coef)
    for i, (p0, m0, v0) in enumerate(was):
        pick = (lambda t: t[0][places[i]]) if i < 3 else (lambda t: t[1])
        assert bool(((pick(out).double() - pick(g).double() * coef).abs() <= (2.0 ** -8 + 2.0 ** -23) * (pick(g).double() * coef).abs()).all())
        rp, rm, rv = adamw_reference(p0, pick(g), m0, v0, 1, lr, (0.9, 0.95), 1e-8, 0.1, float(clip.coef))
        gc = pick(g).double().abs()
        big_m = torch.maximum(m0.double().abs(), gc)
        update = lr * big_m / 0.1 / ((rv / (1 - 0.95)).sqrt() + 1e-8)
        assert bool(((pick(m).double() - rm).abs() <= 3 * 2.0 ** -24 * big_m).all())
        assert bool(((pick(p).double() - rp).abs() <= 2.0 ** -21 * (p0.double().abs() + update)).all())
