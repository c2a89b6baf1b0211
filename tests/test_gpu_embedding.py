"""Embedding rows and their gradient against their formulas in 64 bits.

Tolerances: a row is one product with the scale (itself rounded to fp32) and one rounding to the type: 2 * 2^-24 and half a step of it (bf16 2^-8).
A gradient element is a sum of n terms in fp32, in any order: n roundings of at most 2^-24 of the sum of their sizes, three more for the scale, its product
and the sum with what was there, then the rounding to the gradient's type."""
import math

import pytest
import torch

DEV = "cuda:0"
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def make_tokens(T, V, kind, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    if kind == "uniform":
        t = torch.randint(0, V, (T,), device=DEV, generator=g)
    elif kind == "zipf":
        t = (torch.exp(torch.rand((T,), device=DEV, generator=g, dtype=torch.float64) * math.log(V + 1)).long() - 1).clamp(0, V - 1)
    elif kind == "one":
        t = torch.full((T,), V - 1, device=DEV)
    elif kind == "sorted":
        t = torch.arange(T, device=DEV) * V // max(T, 1)
    elif kind == "down":
        t = (T - 1 - torch.arange(T, device=DEV)) % V
    elif kind == "padding":
        t = torch.full((T,), -1, device=DEV)
    else:                       # everything that is no word beside words
        t = torch.randint(0, V, (T,), device=DEV, generator=g)
        bad = torch.tensor([-1, -100, V, V + 1, 2 ** 31 - 1, -2 ** 31], device=DEV)
        pick = torch.randint(0, 12, (T,), device=DEV, generator=g)
        t = torch.where(pick < 6, bad[pick.clamp(max=5)], t)
    return t.to(torch.int32)


def counted(tokens, V):
    return (tokens >= 0) & (tokens < V)


def sums(tokens, rows, V):
    """Sums of rows by word in 64 bits."""
    keep = counted(tokens, V)
    out = torch.zeros((V, rows.shape[1]), dtype=torch.float64, device=DEV)
    return out.index_add_(0, tokens[keep].long(), rows[keep].double())


KINDS = ["uniform", "zipf", "one", "sorted", "down", "padding", "mixed"]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,d,V", [(1, 16, 1), (1, 4096, 32000), (3, 48, 2), (257, 1040, 5003), (1000, 64, 131), (4099, 512, 70000)])
@pytest.mark.parametrize("scale", [1.0, 45.25, -0.3])
def test_lookup(T, d, V, dtype, scale):
    from paper_2505_11432_amd.embedding import Embedding
    g = torch.Generator(device=DEV).manual_seed(1)
    table = torch.randn((V, d), device=DEV, generator=g).to(dtype)
    op = Embedding(T, d, V, dtype=dtype, scale=scale, gradients=False, device=DEV)
    for kind in ("uniform", "mixed"):
        tokens = make_tokens(T, V, kind)
        out = op.lookup(table, tokens)
        keep = counted(tokens, V)
        want = torch.where(keep[:, None], table[tokens.clamp(0, V - 1).long()].double() * scale, torch.zeros((), dtype=torch.float64, device=DEV))
        assert bool(((out.double() - want).abs() <= (HALF[dtype] + 2.0 ** -23) * want.abs()).all())
        assert bool((out[~keep] == 0).all())
        if scale == 1.0:
            assert torch.equal(out[keep], table[tokens[keep].long()])


def check_gradient(T, d, V, dtype, grad_dtype, kind, scale, accumulate, seed=0):
    from paper_2505_11432_amd.embedding import Embedding
    g = torch.Generator(device=DEV).manual_seed(seed + 7)
    tokens = make_tokens(T, V, kind, seed)
    dy = torch.randn((T, d), device=DEV, generator=g).to(dtype)
    # the gradient lies inside a larger buffer, whose other rows have to stay as they are
    around = torch.randn((V + 2, d), device=DEV, generator=g).to(grad_dtype)
    was = around.clone()
    d_table = around[1:V + 1]
    op = Embedding(T, d, V, dtype=dtype, scale=scale, d_table=d_table, device=DEV)
    op.workspace.fill_(255)
    got = op.backward(tokens, dy, accumulate=accumulate).clone()
    old = was[1:V + 1].double() if accumulate else torch.zeros((V, d), dtype=torch.float64, device=DEV)
    want = sums(tokens, dy, V) * scale + old
    size = sums(tokens, dy.abs(), V) * abs(scale) + old.abs()
    n = torch.bincount(tokens[counted(tokens, V)].long(), minlength=V)[:, None].double()
    tol = (n + 3) * 2.0 ** -24 * size
    if grad_dtype == torch.bfloat16:
        tol = tol * (1 + HALF[grad_dtype]) + HALF[grad_dtype] * want.abs()
    assert bool(((got.double() - want).abs() <= tol).all())
    untouched = (n == 0).squeeze(1)
    assert torch.equal(got[untouched], was[1:V + 1][untouched] if accumulate else torch.zeros_like(got[untouched]))
    assert torch.equal(around[0], was[0]) and torch.equal(around[-1], was[-1])
    # the same bits whatever lay in the workspace and ran before
    around.copy_(was)
    op.workspace.zero_()
    assert torch.equal(op.backward(tokens, dy, accumulate=accumulate), got)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype,grad_dtype", [(torch.bfloat16, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.float32, torch.float32)])
@pytest.mark.parametrize("T,d,V", [(1, 16, 1), (2, 4096, 3), (63, 528, 40), (64, 512, 64), (65, 496, 1), (1009, 1040, 503), (4097, 64, 3000)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_gradient(T, d, V, dtype, grad_dtype, kind, accumulate):
    check_gradient(T, d, V, dtype, grad_dtype, kind, 0.7, accumulate)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T,d,V", [(8191, 32, 511), (8192, 32, 512), (8193, 32, 513), (20000, 48, 262143), (20000, 48, 262144), (100_001, 16, 32000), (12289, 2048, 700),
                                   (2049, 528, 9000), (2048, 2048, 300), (2048, 2064, 300), (1500, 8192, 700), (3000, 16, 600_000), (8192, 16, 524_287), (8192, 16, 524_288), (7000, 1040, 3000)])
def test_gradient_of_many_tokens(T, d, V, kind):
    """One workgroup sorts up to 8192 tokens of words of up to 19 bits, tiles of 4096 more; 9, 18, 19 and 20 bits of words.  Few tokens are not sorted where
    their squared number times the slabs of 512 columns is at most 2^24."""
    check_gradient(T, d, V, torch.bfloat16, torch.float32, kind, 1.0, False)


@pytest.mark.gpu
def test_empty_batch():
    from paper_2505_11432_amd.embedding import Embedding
    op = Embedding(0, 32, 50, device=DEV)
    tokens, dy = torch.empty((0,), dtype=torch.int32, device=DEV), torch.empty((0, 32), dtype=torch.bfloat16, device=DEV)
    op.d_table.fill_(3.0)
    op.backward(tokens, dy, accumulate=True)
    assert bool((op.d_table == 3).all())
    op.backward(tokens, dy)
    assert bool((op.d_table == 0).all())
    assert tuple(op.lookup(torch.zeros((50, 32), dtype=torch.bfloat16, device=DEV), tokens).shape) == (0, 32)


@pytest.mark.gpu
def test_non_finite_rows_stay_in_their_words():
    from paper_2505_11432_amd.embedding import Embedding
    T, d, V = 300, 32, 100
    tokens = make_tokens(T, V - 2, "zipf")
    tokens[5], tokens[6], tokens[7] = V - 1, -1, V - 2
    dy = torch.ones((T, d), dtype=torch.bfloat16, device=DEV)
    dy[5], dy[6], dy[7] = float("inf"), float("nan"), float("nan")
    got = Embedding(T, d, V, device=DEV).backward(tokens, dy)
    assert bool(torch.isinf(got[V - 1]).all()) and bool(torch.isnan(got[V - 2]).all())
    assert bool(torch.isfinite(got[:V - 2]).all())


@pytest.mark.gpu
def test_past_32_bits():
    """A table, its gradient and a batch whose offsets pass 2^32 bytes."""
    from paper_2505_11432_amd.embedding import Embedding
    T, d, V = 70_001, 16384, 140_003
    g = torch.Generator(device=DEV).manual_seed(3)
    table = torch.empty((V, d), dtype=torch.bfloat16, device=DEV).normal_(0.0, 1.0, generator=g)
    tokens = make_tokens(T, V, "uniform")
    tokens[-1], tokens[-2], tokens[0] = V - 1, V - 1, V - 2
    op = Embedding(T, d, V, grad_dtype=torch.bfloat16, device=DEV)
    out = op.lookup(table, tokens)
    for t in (0, 1, T // 2, T - 2, T - 1):
        assert torch.equal(out[t], table[int(tokens[t])])
    got = op.backward(tokens, out)
    for v in (V - 1, V - 2, 0, int(tokens[T // 2])):
        rows = (tokens == v).nonzero().squeeze(1)
        want = out[rows].double().sum(0) if len(rows) else torch.zeros((d,), dtype=torch.float64, device=DEV)
        assert bool(((got[v].double() - want).abs() <= (2.0 ** -8 + (len(rows) + 3) * 2.0 ** -24) * out[rows].double().abs().sum(0)).all())


@pytest.mark.gpu
def test_captured_twice_and_replayed():
    """Two captured gradients with handles of their own, replayed in turn with other tokens between eager work; every replay equals the eager call."""
    from paper_2505_11432_amd.embedding import Embedding
    T, d, V = 9000, 64, 1000
    table = torch.randn((V, d), device=DEV).to(torch.bfloat16)
    ops = [Embedding(T, d, V, scale=2.0, device=DEV) for _ in range(3)]
    tokens = [make_tokens(T, V, "zipf", s) for s in range(2)]
    dys = [torch.randn((T, d), device=DEV).to(torch.bfloat16) for _ in range(2)]
    graphs = []
    for i in range(2):
        ops[i].lookup(table, tokens[i])
        ops[i].backward(tokens[i], dys[i])
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            ops[i].lookup(table, tokens[i])
            ops[i].backward(tokens[i], dys[i])
        graphs.append(graph)
    for r in range(3):
        for i in range(2):
            tokens[i].copy_(make_tokens(T, V, "mixed", 10 * r + i))
            dys[i].normal_()
        for i in range(2):
            graphs[i].replay()
        torch.cuda.synchronize()
        for i in range(2):
            assert torch.equal(ops[2].lookup(table, tokens[i]), ops[i].out)
            assert torch.equal(ops[2].backward(tokens[i], dys[i]), ops[i].d_table)


@pytest.mark.gpu
def test_on_another_stream():
    from paper_2505_11432_amd.embedding import Embedding
    T, d, V = 3000, 128, 500
    tokens = make_tokens(T, V, "zipf")
    dy = torch.randn((T, d), device=DEV).to(torch.bfloat16)
    op = Embedding(T, d, V, device=DEV)
    want = op.backward(tokens, dy).clone()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        later = torch.zeros_like(dy)
        torch.cuda._sleep(2_000_000)
        later.copy_(dy)
        op.backward(tokens, later)
    side.synchronize()
    assert torch.equal(op.d_table, want)


@pytest.mark.gpu
def test_refused():
    from paper_2505_11432_amd import binding as B
    from paper_2505_11432_amd.embedding import Embedding
    op = Embedding(8, 32, 10, device=DEV)
    tokens, dy = make_tokens(8, 10, "uniform"), torch.zeros((8, 32), dtype=torch.bfloat16, device=DEV)
    table = torch.zeros((10, 32), dtype=torch.bfloat16, device=DEV)
    for bad in (lambda: op.lookup(table.float(), tokens), lambda: op.lookup(table[:9], tokens), lambda: op.lookup(table, tokens.long()),
                lambda: op.lookup(table, tokens[:4]), lambda: op.backward(tokens, dy.float()), lambda: op.backward(tokens, dy[:, :16]),
                lambda: op.backward(tokens[::2], dy), lambda: op.backward(tokens.cpu(), dy), lambda: Embedding(8, 40, 10, device=DEV),
                lambda: Embedding(8, 32, 10, dtype=torch.float32, grad_dtype=torch.bfloat16, device=DEV), lambda: Embedding(8, 32, 0, device=DEV),
                lambda: Embedding(8, 32, 10, device=DEV, gradients=False).backward(tokens, dy), lambda: Embedding(8, 32, 11, device=DEV, d_table=op.d_table)):
        with pytest.raises(AssertionError):
            bad()
    same = torch.zeros((64, 32), dtype=torch.bfloat16, device=DEV)
    with pytest.raises(B.MoEError):
        B.moe_embedding_fwd(same[:10], tokens, 1.0, same[8:16])
    with pytest.raises(B.MoEError):
        B.moe_embedding_bwd(tokens, same[:8], 1.0, same[4:14], False, op.workspace)
    with pytest.raises(B.MoEError):
        B.moe_embedding_bwd(tokens, dy, 1.0, op.d_table, False, op.workspace[:16])
