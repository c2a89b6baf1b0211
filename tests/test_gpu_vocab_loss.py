"""The vocabulary loss against its definition in 64 bits (torch on the CPU, from the same bf16 or fp32 inputs).

Tolerances, as relative 2-norms over a tensor (and per row for dx), with u = eps / 2 of the type (bf16 2^-8, fp32 2^-24):
  loss, lse, total   z is a sum of d products in fp32: at most about sqrt(d) u32 |x||w| off; with exp, log and the joins 64 u32 of the largest
                     |z| or loss: 2^-16 of the larger of max |lse| and 1
  dx, d_w in bf16    one rounding of the result, u16, and one of G, u16, none of them larger than that element by element: 2 u16 in norm
  d_w in fp32 from bf16 data   the rounding of G alone: u16
  fp32 data          products of d, V or T terms: 2^-24 sqrt(terms) and the exponentials' 8 u32: 2^-16 in norm
"""
import math

import numpy as np
import pytest
import torch

DEV = "cuda:0"
U16, F32_TOL = 2.0 ** -8, 2.0 ** -16


def reference(x, w, target, token_w=None):
    """In 64 bits on the CPU: total, loss, lse, dx, d_w."""
    x, w, target = x.double().cpu(), w.double().cpu(), target.long().cpu()
    T, V = x.shape[0], w.shape[0]
    keep = (target >= 0) & (target < V)
    loss, lse = torch.zeros(T, dtype=torch.float64), torch.zeros(T, dtype=torch.float64)
    dx, d_w = torch.zeros_like(x), torch.zeros_like(w)
    rows = keep.nonzero().squeeze(1)
    c = token_w.double().cpu()[rows] if token_w is not None else torch.full((len(rows),), 1.0 / max(1, len(rows)), dtype=torch.float64)
    z = x[rows] @ w.t()
    lse[rows] = torch.logsumexp(z, 1)
    loss[rows] = lse[rows] - z[torch.arange(len(rows)), target[rows]]
    g = torch.exp(z - lse[rows][:, None])
    g[torch.arange(len(rows)), target[rows]] -= 1.0
    g *= c[:, None]
    dx[rows] = g @ w
    d_w += g.t() @ x[rows]
    return (c * loss[rows]).sum(), loss, lse, dx, d_w


def inputs(T, d, V, dtype, seed, ignored=0.2, lean=6.0):
    g = torch.Generator().manual_seed(seed)
    w = torch.randn((V, d), generator=g) * (1.28 / math.sqrt(d))
    target = torch.randint(0, V, (T,), generator=g)
    x = torch.randn((T, d), generator=g) + torch.rand((T, 1), generator=g) * lean * w[target]
    out = torch.rand((T,), generator=g) < ignored
    target = torch.where(out, torch.full_like(target, -100), target).to(torch.int32)
    token_w = torch.rand((T,), generator=g) / max(T, 1)
    return x.to(dtype).to(DEV), w.to(dtype).to(DEV), target.to(DEV), token_w.to(DEV)


def rel(got, want):
    got, want = got.double().cpu(), want.double()
    n = want.norm()
    return float((got - want).norm() / n) if n > 0 else float(got.abs().max() if got.numel() else 0.0)


def check(op, x, w, target, token_w, tol_g, tol_w):
    total, loss, lse, dx, d_w = reference(x, w, target, token_w)
    scale = max(1.0, float(lse.abs().max()) if lse.numel() else 1.0)
    assert float((op.loss.double().cpu() - loss).abs().max()) <= F32_TOL * scale
    assert float((op.lse.double().cpu() - lse).abs().max()) <= F32_TOL * scale
    c_sum = float(token_w.sum()) if token_w is not None else 1.0
    assert abs(float(op.total) - float(total)) <= F32_TOL * scale * max(c_sum, 1e-30)
    assert rel(op.dx, dx) <= tol_g
    assert rel(op.d_w, d_w) <= tol_w
    # row by row: no row is lost in the norm of the others
    far = (op.dx.double().cpu() - dx).norm(dim=1)
    assert bool((far <= 2 * tol_g * dx.norm(dim=1) + 1e-30).all())
    out = (target.cpu() < 0) | (target.cpu() >= w.shape[0])
    assert not bool(op.dx.float().cpu()[out].any()) and not bool(op.loss.cpu()[out].any()) and not bool(op.lse.cpu()[out].any())


def make(T, d, V, dtype, **kw):
    from paper_2505_11432_amd.head import VocabLoss
    return VocabLoss(T, d, V, dtype=dtype, **kw)


SIZES = [(1, 16, 1), (1, 128, 7), (2, 32, 65), (3, 48, 1000), (17, 256, 129), (64, 64, 500), (129, 144, 2049), (257, 80, 4099), (300, 1040, 5003),
         (513, 512, 128), (700, 16, 9001), (1025, 272, 1537)]


@pytest.mark.gpu
@pytest.mark.parametrize("T,d,V", SIZES)
@pytest.mark.parametrize("weights", [0, 1])
def test_bf16_step(T, d, V, weights):
    x, w, target, token_w = inputs(T, d, V, torch.bfloat16, seed=T * 7 + V)
    tw = token_w if weights else None
    for grad_dtype, tol_w in ((torch.bfloat16, 2 * U16), (torch.float32, U16)):
        op = make(T, d, V, torch.bfloat16, grad_dtype=grad_dtype)
        op.step(x, w, target, token_w=tw)
        check(op, x, w, target, tw, 2 * U16, tol_w)


@pytest.mark.gpu
@pytest.mark.parametrize("T,d,V", SIZES)
@pytest.mark.parametrize("weights", [0, 1])
def test_f32_step(T, d, V, weights):
    x, w, target, token_w = inputs(T, d, V, torch.float32, seed=T * 5 + V)
    tw = token_w if weights else None
    op = make(T, d, V, torch.float32)
    op.step(x, w, target, token_w=tw)
    check(op, x, w, target, tw, F32_TOL, F32_TOL)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,d,V", SIZES + [(256, 64, 700), (33, 128, 30011)])
def test_score(T, d, V, dtype):
    x, w, target, _ = inputs(T, d, V, dtype, seed=T + V)
    op = make(T, d, V, dtype, gradients=False)
    loss, lse = op.score(x, w, target)
    _, want_loss, want_lse, _, _ = reference(x, w, target)
    scale = max(1.0, float(want_lse.abs().max()))
    assert float((loss.double().cpu() - want_loss).abs().max()) <= F32_TOL * scale
    assert float((lse.double().cpu() - want_lse).abs().max()) <= F32_TOL * scale


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,tol", [(torch.bfloat16, 2 * U16), (torch.float32, F32_TOL)])
@pytest.mark.parametrize("grad", [0, 1])
def test_pieces(dtype, tol, grad):
    """Several pieces, the last one short, some empty: the same results as one piece within the rounding."""
    T, d, V = 1500, 96, 1111
    for ignored in (0.0, 0.5, 0.95):
        x, w, target, token_w = inputs(T, d, V, dtype, seed=3, ignored=ignored)
        gdt = dtype if grad else torch.float32
        op = make(T, d, V, dtype, grad_dtype=gdt, piece_bytes=256 * 1152 * (2 if dtype == torch.bfloat16 else 4))
        assert op.piece_rows == 256
        for _ in range(2):
            op.step(x, w, target, token_w=token_w)
            check(op, x, w, target, token_w, tol, tol)
        loss, lse = op.score(x, w, target)
        _, want, _, _, _ = reference(x, w, target)
        assert float((loss.double().cpu() - want).abs().max()) <= F32_TOL * 64


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T", [5, 300])
def test_nothing_counts(dtype, T):
    d, V = 64, 333
    x, w, target, token_w = inputs(T, d, V, dtype, seed=1)
    target.fill_(-100)
    target[0] = V                                       # out of range on the other side
    x.fill_(float("nan"))
    op = make(T, d, V, dtype)
    op.dx.fill_(7.0)
    op.d_w.fill_(7.0)
    op.step(x, w, target)
    assert float(op.total) == 0.0
    assert not bool(op.dx.any()) and not bool(op.d_w.any()) and not bool(op.loss.any()) and not bool(op.lse.any())
    op.score(x, w, target)
    assert not bool(op.loss.any()) and not bool(op.lse.any())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,tol", [(torch.bfloat16, 2 * U16), (torch.float32, F32_TOL)])
@pytest.mark.parametrize("T", [40, 400])
def test_left_out_rows_hold_anything(dtype, tol, T):
    """NaN and infinities in rows that are left out reach no result."""
    d, V = 96, 777
    x, w, target, _ = inputs(T, d, V, dtype, seed=2, ignored=0.4)
    clean = x.clone()
    out = target < 0
    x[out] = float("nan")
    x[out.nonzero()[::2].squeeze(1)] = float("inf")
    op = make(T, d, V, dtype)
    op.step(x, w, target)
    clean[out] = 0
    check(op, clean, w, target, None, tol, tol)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_nan_row_that_counts_shows(dtype):
    T, d, V = 300, 64, 500
    x, w, target, _ = inputs(T, d, V, dtype, seed=9, ignored=0.0)
    x[5] = float("nan")
    op = make(T, d, V, dtype)
    op.step(x, w, target)
    assert math.isnan(float(op.loss[5])) and math.isnan(float(op.total))
    assert not bool(op.loss[:5].isnan().any()) and not bool(op.loss[6:].isnan().any())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,tol", [(torch.bfloat16, 2 * U16), (torch.float32, F32_TOL)])
def test_large_logits(dtype, tol):
    """Logits in the hundreds, of both signs: the maximum is taken off before exp; certain tokens have a loss and gradients near 0."""
    T, d, V = 270, 128, 900
    x, w, target, _ = inputs(T, d, V, dtype, seed=4, ignored=0.1, lean=200.0)
    op = make(T, d, V, dtype)
    op.step(x, w, target)
    total, loss, lse, dx, d_w = reference(x, w, target)
    assert float(lse.abs().max()) > 150
    scale = float(lse.abs().max())
    assert float((op.lse.double().cpu() - lse).abs().max()) <= F32_TOL * scale
    assert float((op.loss.double().cpu() - loss).abs().max()) <= F32_TOL * scale
    # exp of a logit that is F32_TOL * scale off is off by as much
    assert rel(op.dx, dx) <= tol + F32_TOL * scale and rel(op.d_w, d_w) <= tol + F32_TOL * scale


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,grad", [(torch.bfloat16, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.float32, torch.float32)])
@pytest.mark.parametrize("pieces", [1, 3])
def test_accumulate(dtype, grad, pieces):
    T, d, V = 600, 64, 515
    es = 2 if dtype == torch.bfloat16 else 4
    x, w, target, _ = inputs(T, d, V, dtype, seed=6)
    op = make(T, d, V, dtype, grad_dtype=grad, piece_bytes=(1 << 30) if pieces == 1 else 256 * 576 * es)
    op.step(x, w, target)
    op.step(x, w, target, accumulate=True)
    _, _, _, _, d_w = reference(x, w, target)
    tol = F32_TOL if dtype == torch.float32 else U16 if grad == torch.float32 else 3 * U16
    assert rel(op.d_w, 2 * d_w) <= tol


@pytest.mark.gpu
def test_gradients_by_differences():
    """total(x + h e) - total(x - h e) over 2 h, fp32 data, directions drawn at random: the difference of two fp32 totals of size L is
    L 2^-24 * 8 / h off, the third-order term h^2."""
    T, d, V = 50, 32, 211
    x, w, target, _ = inputs(T, d, V, torch.float32, seed=8)
    op = make(T, d, V, torch.float32)
    op.step(x, w, target)
    dx, d_w = op.dx.clone(), op.d_w.clone()
    g = torch.Generator(device=DEV).manual_seed(0)
    h = 2.0 ** -5
    for which in ("x", "w"):
        t, grad = (x, dx) if which == "x" else (w, d_w)
        e = torch.randn(t.shape, device=DEV, generator=g)
        e /= e.norm()
        up = float(op.step(x + h * e, w, target) if which == "x" else op.step(x, w + h * e, target))
        down = float(op.step(x - h * e, w, target) if which == "x" else op.step(x, w - h * e, target))
        want = float((grad.double() * e.double()).sum())
        assert abs((up - down) / (2 * h) - want) <= 16 * 2.0 ** -24 * abs(up) / h + h * h


@pytest.mark.gpu
@pytest.mark.parametrize("T,d,V", [(1, 128, 3000), (300, 256, 4099), (1100, 64, 700)])
def test_same_bits_every_time(T, d, V):
    x, w, target, _ = inputs(T, d, V, torch.bfloat16, seed=11)
    op = make(T, d, V, torch.bfloat16)
    op.step(x, w, target)
    first = [t.clone() for t in (op.total, op.loss, op.lse, op.dx, op.d_w)]
    op.workspace.fill_(255)                             # NaN patterns in whatever is not written
    op.step(x, w, target)
    for a, b in zip(first, (op.total, op.loss, op.lse, op.dx, op.d_w)):
        assert torch.equal(a, b)


@pytest.mark.gpu
def test_on_another_stream_and_in_a_graph():
    from paper_2505_11432_amd import binding as B
    T, d, V = 300, 128, 2000
    x, w, target, _ = inputs(T, d, V, torch.bfloat16, seed=12)
    op = make(T, d, V, torch.bfloat16)
    op.step(x, w, target)
    want = [t.clone() for t in (op.total, op.loss, op.dx, op.d_w)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        op.dx.zero_()
        op.step(x, w, target)
        got = [t.clone() for t in (op.total, op.loss, op.dx, op.d_w)]
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    B.moe_init()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        op.step(x, w, target)
    for i in range(3):
        x2, _, t2, _ = inputs(T, d, V, torch.bfloat16, seed=20 + i)
        x.copy_(x2)
        target.copy_(t2)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (op.total, op.loss, op.dx, op.d_w)]
        op.step(x, w, target)
        assert all(torch.equal(a, b) for a, b in zip((op.total, op.loss, op.dx, op.d_w), got))


@pytest.mark.gpu
def test_empty_batch():
    op = make(0, 64, 100, torch.bfloat16)
    x = torch.empty((0, 64), dtype=torch.bfloat16, device=DEV)
    w = torch.randn((100, 64), device=DEV).to(torch.bfloat16)
    target = torch.empty((0,), dtype=torch.int32, device=DEV)
    op.d_w.fill_(3.0)
    assert float(op.step(x, w, target)) == 0.0 and not bool(op.d_w.any())
    loss, lse = op.score(x, w, target)
    assert loss.numel() == 0 and lse.numel() == 0


@pytest.mark.gpu
def test_refused_tensors():
    T, d, V = 8, 64, 100
    x, w, target, token_w = inputs(T, d, V, torch.bfloat16, seed=1)
    op = make(T, d, V, torch.bfloat16)
    for bad in (lambda: op.step(x.t().contiguous().t(), w, target), lambda: op.step(x, w[:, :32], target), lambda: op.step(x, w, target.long()),
                lambda: op.step(x[:4], w, target), lambda: op.step(x, w, target, token_w=token_w.double()), lambda: op.step(x.float(), w, target),
                lambda: op.step(x, w.float(), target), lambda: op.step(x.cpu(), w, target)):
        with pytest.raises(AssertionError):
            bad()
    with pytest.raises(AssertionError):
        make(T, d, V, torch.bfloat16, gradients=False).step(x, w, target)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,tol", [(torch.bfloat16, 2 * U16), (torch.float32, F32_TOL)])
@pytest.mark.parametrize("T,d,V", [(2048, 32, 300), (2049, 32, 300), (9001, 48, 130), (65536, 16, 70), (66001, 16, 70)])
def test_many_tokens(dtype, tol, T, d, V):
    """Sizes around those at which the rows that count are found in another way."""
    x, w, target, token_w = inputs(T, d, V, dtype, seed=T, ignored=0.3)
    op = make(T, d, V, dtype)
    op.step(x, w, target, token_w=token_w)
    check(op, x, w, target, token_w, tol, tol)
    op.loss.fill_(-1.0)
    loss, _ = op.score(x, w, target)
    _, want, _, _, _ = reference(x, w, target)
    assert float((loss.double().cpu() - want).abs().max()) <= F32_TOL * 64


@pytest.mark.gpu
@pytest.mark.parametrize("T", [60, 128, 150, 192, 260, 320, 400, 640])
@pytest.mark.parametrize("V", [2000, 30000])
def test_row_tiles(T, V):
    """Numbers of rows around the tiles', words that fill no tile, most rows counting."""
    d = 208
    x, w, target, _ = inputs(T, d, V + 13, torch.bfloat16, seed=T + V, ignored=0.05)
    op = make(T, d, V + 13, torch.bfloat16)
    op.step(x, w, target)
    check(op, x, w, target, None, 2 * U16, U16)
    want = op.loss.clone(), op.lse.clone()
    op.score(x, w, target)
    for a, b in zip(want, (op.loss, op.lse)):
        assert float((a - b).abs().max()) <= 2 * F32_TOL * max(1.0, float(op.lse.abs().max()))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,tol", [(torch.bfloat16, 2 * U16), (torch.float32, F32_TOL)])
@pytest.mark.parametrize("T,d,V", [(2049, 48, 300), (4500, 32, 1500), (6000, 16, 5000)])
def test_every_token_counts(dtype, tol, T, d, V):
    """Nothing is left out, then one token is, with the same buffers: rows are read in place or gathered."""
    x, w, target, token_w = inputs(T, d, V, dtype, seed=T, ignored=0.0)
    op = make(T, d, V, dtype)
    for _ in range(2):
        op.step(x, w, target)
        check(op, x, w, target, None, tol, tol)
        loss, _ = op.score(x, w, target)
        _, want, _, _, _ = reference(x, w, target)
        assert float((loss.double().cpu() - want).abs().max()) <= F32_TOL * 64
        target[T // 2] = -1
        x[T // 2] = float("nan")
        w = w.clone()
        clean = x.clone()
        clean[T // 2] = 0
        op.step(x, w, target)
        check(op, clean, w, target, None, tol, tol)
        x, target = clean, torch.where(target < 0, torch.zeros_like(target), target)


@pytest.mark.gpu
def test_past_32_bits():
    """A vocabulary matrix of more than 2^31 elements (4.4 GB), targets at both ends of it.  The reference is fp32 on the GPU, in chunks of words:
    its own error is far below the tolerances."""
    T, d, V, step = 24, 4096, 530_000, 53_000
    g = torch.Generator(device=DEV).manual_seed(5)
    w = torch.empty((V, d), dtype=torch.bfloat16, device=DEV)
    for part in w.split(step):
        part.copy_(torch.randn(part.shape, device=DEV, generator=g) * (1.28 / math.sqrt(d)))
    target = torch.randint(0, V, (T,), device=DEV, generator=g)
    target[:3], target[3:6] = torch.tensor([V - 1, V - 2, V - 300]), torch.tensor([0, 1, 255])
    target[6] = -100
    kept = (target >= 0).nonzero().squeeze(1)
    x = torch.randn((T, d), device=DEV, generator=g) + 5.0 * w[target.clamp(min=0)].float()
    x = x.to(torch.bfloat16)
    op = make(T, d, V, torch.bfloat16, grad_dtype=torch.bfloat16)
    op.step(x, w, target.to(torch.int32))
    xf = x.float()[kept]
    z = torch.cat([xf @ part.float().t() for part in w.split(step)], 1)
    lse = torch.logsumexp(z.double(), 1)
    at, tg = torch.arange(len(kept), device=DEV), target[kept]
    loss = lse - z[at, tg].double()
    assert float((op.loss.double()[kept] - loss).abs().max()) <= F32_TOL * float(lse.abs().max())
    p = torch.exp(z - lse.float()[:, None])
    p[at, tg] -= 1.0
    p /= len(kept)
    dx = torch.zeros((len(kept), d), device=DEV)
    for i, part in enumerate(w.split(step)):
        dx += p[:, i * step:i * step + len(part)] @ part.float()
        d_w = p[:, i * step:i * step + len(part)].t() @ xf
        got = op.d_w[i * step:i * step + len(part)].float()
        assert float((got - d_w).norm()) <= 2 * U16 * float(d_w.norm()), i
    assert float((op.dx.float()[kept] - dx).norm()) <= 2 * U16 * float(dx.norm())
    assert not bool(op.dx[6].any())
