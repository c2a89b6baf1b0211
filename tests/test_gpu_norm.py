"""Norms around a block against their formulas in 64 bits.

Tolerances.  A mean over a row is a tree of sums in fp32: at most 64 roundings one behind another in the widest row (16 steps in a thread, 8 elements, waves),
so 1 / rms is off by less than 40 * 2^-24 relative and every product of a few factors by less than 2^-18 = 64 * 2^-24 of the sum of its terms' sizes
(`size` below: the formula with absolute values).  Then half a step of the type (bf16 2^-8, fp32 2^-24) of the value.  h is held to the formula on the stream
as it was written.  A weight's gradient sums T terms: T + 64 roundings of 2^-24 of their sizes, on top of the 2^-18 of each."""
import pytest
import torch

DEV = "cuda:0"
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
CALC = 2.0 ** -18
EPS = 1e-6


def near(got, want, size, dtype):
    return bool(((got.double() - want).abs() <= CALC * (1 + HALF[dtype]) * size + HALF[dtype] * want.abs()).all())


def rms(v):
    return torch.sqrt(v.square().mean(1, keepdim=True) + EPS)


def inputs(T, d, dtype, residual, after, gate_rows, before, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    rows = lambda s: (torch.randn((T, d), device=DEV, generator=g) * s).to(dtype)
    vec = lambda *shape: 1.0 + 0.5 * torch.randn(shape, device=DEV, generator=g)
    x, y = rows(2.0), rows(0.7) if residual else None
    if T > 2:
        x[1] = 0                                    # rows of zeros: eps alone
        if residual:
            y[2] = 0
    return dict(x=x, y=y, w_after=vec(d) if after else None, gate=vec(-(-T // gate_rows), d) if gate_rows else None, w_before=vec(d) if before else None,
                d_out=rows(1.0) if residual else None, d_h=rows(1.0) if before else None)


def gate_of(s, T, gate_rows):
    return s["gate"].double().repeat_interleave(gate_rows, 0)[:T] if gate_rows else 1.0


def check_forward(op, s, alpha):
    T, dtype = op.T, op.dtype
    out, h = op.forward(s["x"], s["y"], s["w_after"], s["gate"], s["w_before"])
    x = s["x"].double()
    if op.residual:
        n = s["y"].double()
        if op.after:
            n = n / rms(n) * s["w_after"].double()
        n = n * gate_of(s, T, op.gate_rows)
        assert near(out, alpha * x + n, (alpha * x).abs() + n.abs(), dtype)
    else:
        assert out is s["x"]
    if op.before:
        kept = out.double()
        want = kept / rms(kept) * s["w_before"].double()
        assert near(h, want, want.abs(), dtype)
    return out


def back(v, u, size_u):
    """(u - unit mean(u unit)) / rms and its size, unit, rms."""
    r = rms(v)
    unit = v / r
    return (u - unit * (u * unit).mean(1, keepdim=True)) / r, (size_u + unit.abs() * (size_u * unit.abs()).mean(1, keepdim=True)) / r, unit


def by_gate(t, gate_rows):
    T, d = t.shape
    groups = -(-T // gate_rows)
    return torch.nn.functional.pad(t, (0, 0, 0, groups * gate_rows - T)).view(groups, gate_rows, d).sum(1)


def check_backward(op, s, out, alpha, accumulate):
    T, dtype = op.T, op.dtype
    olds = {}
    for k in ("d_w_after", "d_gate", "d_w_before"):
        if (t := getattr(op, k)) is not None:
            t.copy_(torch.randn_like(t))
            olds[k] = t.double().clone() if accumulate else torch.zeros_like(t, dtype=torch.float64)
    op.workspace.fill_(255)
    op.backward(out, s["y"], s["w_after"], s["gate"], s["w_before"], s["d_out"], s["d_h"], accumulate=accumulate)
    zero = torch.zeros((T, op.d), dtype=torch.float64, device=DEV)
    g = s["d_out"].double() if s["d_out"] is not None else zero
    size = g.abs()

    def weight(name, terms, sizes):
        # (the terms' own errors, the sums', and that of the sum with what was there)
        tol = (CALC + (T + 64) * 2.0 ** -24) * sizes + 2.0 ** -23 * olds[name].abs()
        assert bool(((getattr(op, name).double() - terms - olds[name]).abs() <= tol).all()), name

    if op.before:
        u = s["d_h"].double() * s["w_before"].double()
        b, size_b, unit = back(out.double(), u, u.abs())
        weight("d_w_before", (s["d_h"].double() * unit).sum(0), (s["d_h"].double() * unit).abs().sum(0))
        g, size = g + b, size + size_b
    assert near(op.dx, alpha * g, abs(alpha) * size, dtype)
    if not op.residual:
        assert op.dy is None
        return
    n = size_n = s["y"].double()
    size_n = n.abs()
    if op.after:
        n = n / rms(n) * s["w_after"].double()
        size_n = n.abs()
    gate = gate_of(s, T, op.gate_rows)
    if op.gate_rows:
        weight("d_gate", by_gate(g * n, op.gate_rows), by_gate(size * size_n, op.gate_rows))
    u, size_u = g * gate, size * (gate.abs() if op.gate_rows else 1.0)
    if op.after:
        w = s["w_after"].double()
        b, size_b, unit = back(s["y"].double(), u * w, size_u * w.abs())
        weight("d_w_after", (u * unit).sum(0), (size_u * unit.abs()).sum(0))
        u, size_u = b, size_b
    assert near(op.dy, u, size_u, dtype)


PARTS = [(False, False, 0, True), (True, False, 0, False), (True, False, 0, True), (True, True, 0, False), (True, True, 0, True), (True, False, 1, True),
         (True, True, 1, True), (True, True, 3, True), (True, True, 7, False), (True, True, 10 ** 6, True), (True, False, 10 ** 6, False)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,d", [(1, 16), (5, 4096), (37, 528), (64, 1024), (203, 1040), (33, 2064), (21, 5008), (9, 16384)])
@pytest.mark.parametrize("parts", PARTS)
def test_forward_and_backward(T, d, dtype, parts):
    from paper_2505_11432_amd.norm import BlockNorm
    residual, after, gate_rows, before = parts
    alpha = 0.75 if residual else 1.0
    op = BlockNorm(T, d, dtype=dtype, eps=EPS, alpha=alpha, residual=residual, after=after, gate_rows=gate_rows, before=before, device=DEV)
    s = inputs(T, d, dtype, *parts)
    out = check_forward(op, s, alpha)
    check_backward(op, s, out, alpha, False)
    check_backward(op, s, out, alpha, True)


@pytest.mark.gpu
@pytest.mark.parametrize("T,d", [(9001, 64), (5000, 1040), (2111, 4096), (1301, 8208)])
@pytest.mark.parametrize("gate_rows", [1, 2, 5, 97, 1300, 10 ** 6])
def test_many_rows(T, d, gate_rows):
    """Several rows per team, rows of the gate inside a team, over two and over many."""
    from paper_2505_11432_amd.norm import BlockNorm
    op = BlockNorm(T, d, dtype=torch.bfloat16, eps=EPS, gate_rows=gate_rows, device=DEV)
    s = inputs(T, d, torch.bfloat16, True, True, gate_rows, True)
    out = check_forward(op, s, 1.0)
    check_backward(op, s, out, 1.0, False)
    first = [t.clone() for t in (op.dx, op.dy, op.d_w_after, op.d_gate, op.d_w_before)]
    op.workspace.zero_()
    op.backward(out, s["y"], s["w_after"], s["gate"], s["w_before"], s["d_out"], s["d_h"])
    for a, b in zip(first, (op.dx, op.dy, op.d_w_after, op.d_gate, op.d_w_before)):
        assert torch.equal(a, b)


@pytest.mark.gpu
def test_gradients_against_differences():
    """Directional differences of the 64-bit forward formula against the kernel's gradients in fp32: a step of 1e-4 leaves 1e-8 of curvature, the gradients
    their 2^-18."""
    from paper_2505_11432_amd.norm import BlockNorm
    T, d, gate_rows, alpha = 24, 64, 5, 0.6
    op = BlockNorm(T, d, dtype=torch.float32, eps=EPS, alpha=alpha, gate_rows=gate_rows, device=DEV)
    s = inputs(T, d, torch.float32, True, True, gate_rows, True, seed=3)
    s["x"][1], s["y"][2] = torch.randn((d,), device=DEV), torch.randn((d,), device=DEV)

    def value(x, y, w_after, gate, w_before):
        out = alpha * x + y / rms(y) * w_after * gate.repeat_interleave(gate_rows, 0)[:T]
        return float((out * s["d_out"].double()).sum() + (out / rms(out) * w_before * s["d_h"].double()).sum())

    out, _ = op.forward(s["x"], s["y"], s["w_after"], s["gate"], s["w_before"])
    op.backward(out, s["y"], s["w_after"], s["gate"], s["w_before"], s["d_out"], s["d_h"])
    names, grads = ("x", "y", "w_after", "gate", "w_before"), (op.dx, op.dy, op.d_w_after, op.d_gate, op.d_w_before)
    at = [s[k].double() for k in names]
    for i, grad in enumerate(grads):
        way = torch.randn_like(at[i])
        step = 1e-4
        moved = [[t + sign * step * way if j == i else t for j, t in enumerate(at)] for sign in (1, -1)]
        slope = (value(*moved[0]) - value(*moved[1])) / (2 * step)
        assert abs(slope - float((grad.double() * way).sum())) <= 2.0 ** -16 * float((grad.double() * way).abs().sum()), names[i]


@pytest.mark.gpu
def test_in_place_and_no_stream_gradient():
    from paper_2505_11432_amd import binding as B
    from paper_2505_11432_amd.norm import BlockNorm
    T, d = 50, 528
    op = BlockNorm(T, d, gate_rows=10 ** 6, device=DEV)
    s = inputs(T, d, torch.bfloat16, True, True, 10 ** 6, True)
    out, h = (t.clone() for t in op.forward(s["x"], s["y"], s["w_after"], s["gate"], s["w_before"]))
    for k in ("x", "y"):
        mine = dict(s, **{k: s[k].clone()})
        B.moe_block_norm_fwd(mine["x"], mine["y"], s["w_after"], s["gate"], s["w_before"], 10 ** 6, 1.0, 1e-6, mine[k], op.h)
        assert torch.equal(mine[k], out) and torch.equal(op.h, h)
    dx, dy = (t.clone() for t in op.backward(out, s["y"], s["w_after"], s["gate"], s["w_before"], s["d_out"], s["d_h"]))
    vectors = [t.clone() for t in (op.d_w_after, op.d_gate, op.d_w_before)]
    for a, b in (("d_out", "d_h"), ("d_h", "d_out"), ("d_out", "y")):
        mine = dict(s, **{a: s[a].clone(), b: s[b].clone()})
        B.moe_block_norm_bwd(out, mine["y"], s["w_after"], s["gate"], s["w_before"], mine["d_out"], mine["d_h"], 10 ** 6, 1.0, 1e-6, mine[a], mine[b],
                             op.d_w_after, op.d_gate, op.d_w_before, False, op.workspace)
        assert torch.equal(mine[a], dx) and torch.equal(mine[b], dy)
        for t, v in zip((op.d_w_after, op.d_gate, op.d_w_before), vectors):
            assert torch.equal(t, v)
    # no gradient down the stream is one of zeros
    op.backward(out, s["y"], s["w_after"], s["gate"], s["w_before"], None, s["d_h"])
    dx = op.dx.clone()
    op.backward(out, s["y"], s["w_after"], s["gate"], s["w_before"], torch.zeros_like(s["d_out"]), s["d_h"])
    assert torch.equal(op.dx, dx)


@pytest.mark.gpu
def test_bad_rows_stay_where_they_are():
    from paper_2505_11432_amd.norm import BlockNorm
    T, d = 40, 64
    op = BlockNorm(T, d, gate_rows=1, device=DEV)
    s = inputs(T, d, torch.bfloat16, True, True, 1, True)
    s["y"][7, 3], s["x"][9, 1] = float("nan"), float("inf")
    out, h = op.forward(s["x"], s["y"], s["w_after"], s["gate"], s["w_before"])
    bad = torch.zeros((T,), dtype=torch.bool, device=DEV)
    bad[7] = bad[9] = True
    assert bool(torch.isfinite(out[~bad]).all()) and bool(torch.isfinite(h[~bad]).all())
    assert bool(torch.isnan(out[7]).all()) and bool(torch.isinf(out[9, 1]))
    op.backward(out, s["y"], s["w_after"], s["gate"], s["w_before"], s["d_out"], s["d_h"])
    for t in (op.dx, op.dy, op.d_gate):
        assert bool(torch.isfinite(t[~bad]).all())


@pytest.mark.gpu
def test_empty_and_past_32_bits():
    from paper_2505_11432_amd.norm import BlockNorm
    op = BlockNorm(0, 64, gate_rows=5, device=DEV)
    e = torch.empty((0, 64), dtype=torch.bfloat16, device=DEV)
    w = torch.ones((64,), device=DEV)
    op.forward(e, e, w, torch.empty((0, 64), device=DEV), w)
    op.backward(e, e, w, torch.empty((0, 64), device=DEV), w, e, e)
    assert bool((op.d_w_after == 0).all())
    T, d = 140_003, 16384
    op = BlockNorm(T, d, gate_rows=70_000, device=DEV)
    s = {k: torch.empty((T, d), dtype=torch.bfloat16, device=DEV).normal_() for k in ("x", "y", "d_out", "d_h")}
    w_after, w_before, gate = (1 + 0.1 * torch.randn(shape, device=DEV) for shape in ((d,), (d,), (3, d)))
    out, h = op.forward(s["x"], s["y"], w_after, gate, w_before)
    op.backward(out, s["y"], w_after, gate, w_before, s["d_out"], s["d_h"])
    for t in (0, 65_536, 131_071, T - 1):
        y, o, dh = s["y"][t:t + 1].double(), out[t:t + 1].double(), s["d_h"][t:t + 1].double()
        n, gt = y / rms(y) * w_after.double(), gate[t // 70_000].double()
        x = s["x"][t:t + 1].double()
        assert near(out[t:t + 1], x + gt * n, x.abs() + (gt * n).abs(), torch.bfloat16)
        want = o / rms(o) * w_before.double()
        assert near(h[t:t + 1], want, want.abs(), torch.bfloat16)
        b, size, _ = back(o, dh * w_before.double(), (dh * w_before.double()).abs())
        g = s["d_out"][t:t + 1].double()
        assert near(op.dx[t:t + 1], g + b, g.abs() + size, torch.bfloat16)


@pytest.mark.gpu
def test_captured_twice_and_replayed():
    from paper_2505_11432_amd.norm import BlockNorm
    T, d = 700, 1040
    ops = [BlockNorm(T, d, gate_rows=100, device=DEV) for _ in range(3)]
    states = [inputs(T, d, torch.bfloat16, True, True, 100, True, seed=i) for i in range(2)]

    def both(op, s):
        out, _ = op.forward(s["x"], s["y"], s["w_after"], s["gate"], s["w_before"])
        op.backward(out, s["y"], s["w_after"], s["gate"], s["w_before"], s["d_out"], s["d_h"])

    graphs = []
    for op, s in zip(ops, states):
        both(op, s)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            both(op, s)
        graphs.append(graph)
    for r in range(3):
        for i, s in enumerate(states):
            for k, v in inputs(T, d, torch.bfloat16, True, True, 100, True, seed=10 * r + i).items():
                s[k].copy_(v)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for op, s in zip(ops, states):
            both(ops[2], s)
            for k in ("out", "h", "dx", "dy", "d_w_after", "d_gate", "d_w_before"):
                assert torch.equal(getattr(op, k), getattr(ops[2], k)), k


@pytest.mark.gpu
def test_on_another_stream():
    from paper_2505_11432_amd.norm import BlockNorm
    T, d = 900, 528
    s = inputs(T, d, torch.bfloat16, True, True, 100, True, seed=3)
    op = BlockNorm(T, d, gate_rows=100, device=DEV)
    names = ("out", "h", "dx", "dy", "d_w_after", "d_gate", "d_w_before")

    def both(y):
        out, _ = op.forward(s["x"], y, s["w_after"], s["gate"], s["w_before"])
        op.backward(out, y, s["w_after"], s["gate"], s["w_before"], s["d_out"], s["d_h"])

    both(s["y"])
    want = {k: getattr(op, k).clone() for k in names}
    later = torch.zeros_like(s["y"])
    for k in names:
        getattr(op, k).zero_()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(2_000_000)
        later.copy_(s["y"])
        both(later)
    side.synchronize()
    for k in names:
        assert torch.equal(getattr(op, k), want[k]), k


@pytest.mark.gpu
def test_refused():
    from paper_2505_11432_amd import binding as B
    from paper_2505_11432_amd.norm import BlockNorm
    T, d = 8, 32
    op = BlockNorm(T, d, gate_rows=4, device=DEV)
    s = inputs(T, d, torch.bfloat16, True, True, 4, True)
    args = lambda **k: [dict(s, **k)[n] for n in ("x", "y", "w_after", "gate", "w_before")]
    for bad in (lambda: op.forward(*args(x=s["x"].float())), lambda: op.forward(*args(y=None)), lambda: op.forward(*args(w_after=None)),
                lambda: op.forward(*args(gate=s["gate"][:1])), lambda: op.forward(*args(gate=s["gate"].to(torch.bfloat16))),
                lambda: op.forward(*args(w_before=s["w_before"][:16])), lambda: op.forward(*args(y=s["y"].t().contiguous().t())),
                lambda: op.backward(*args(), s["d_out"], None), lambda: op.backward(*args(), s["d_out"].float(), s["d_h"]),
                lambda: BlockNorm(T, 40, device=DEV), lambda: BlockNorm(T, 16400, device=DEV), lambda: BlockNorm(T, d, residual=False, device=DEV),
                lambda: BlockNorm(T, d, residual=True, before=False, device=DEV, gradients=False).backward(s["x"])):
        with pytest.raises(AssertionError):
            bad()
    for out, h in ((op.out, op.out), (op.out, s["x"]), (s["d_h"][:4], op.h)):
        with pytest.raises((B.MoEError, AssertionError)):
            B.moe_block_norm_fwd(*args(), 4, 1.0, 1e-6, out, h)
    with pytest.raises(B.MoEError):
        B.moe_block_norm_bwd(*args(), s["d_out"], s["d_h"], 4, 1.0, 1e-6, op.dx, op.dx, op.d_w_after, op.d_gate, op.d_w_before, False, op.workspace)
    with pytest.raises(B.MoEError):
        B.moe_block_norm_bwd(*args(), s["d_out"], s["d_h"], 4, 1.0, 1e-6, s["x"], op.dy, op.d_w_after, op.d_gate, op.d_w_before, False, op.workspace)
    with pytest.raises(B.MoEError):
        B.moe_block_norm_bwd(*args(), s["d_out"], s["d_h"], 4, 1.0, 1e-6, op.dx, op.dy, op.d_w_after, op.d_gate, op.d_w_before, False, op.workspace[:256])
