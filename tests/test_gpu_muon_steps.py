"""Lists of steps and matrices of low rank: the error of an orthogonalised matrix within a model of the roundings, and within what moe.h promises.

Above a side of 64: `rounded` of test_gpu_muon, twice of which is allowed.  With a side of at most 64 all is in 64 bits but X (24 bits: its single precision) and the
last product, whose operands have 22 bits and whose sums of 64 terms are made in fp32, here one term after another, each sum rounded by up to 2^-24 of it (the matrix
instructions take many at a time): `small_rounded`, twice of which is allowed too."""
import math

import pytest
import torch

from test_gpu_muon import DEV, formula, in_pairs, rounded

USUAL, SLOW, CUBIC = (3.4445, -4.7750, 2.0315), (2.0, -1.5, 0.5), (1.5, -0.5, 0.0)
LISTS = {"3": (USUAL,) * 3, "5": (USUAL,) * 5, "6": (USUAL,) * 6, "7": (USUAL,) * 7, "10": (USUAL,) * 10, "slow": (SLOW,) * 5, "13 slow": (SLOW,) * 13,
         "cubic": (CUBIC,) * 16, "usual first": (USUAL,) * 2 + (SLOW,) * 3, "usual last": (SLOW,) * 3 + (USUAL,) * 3, "one": (SLOW,),
         "falling": ((4.0, -6.0, 2.5), (3.8, -5.5, 2.2), (3.2, -4.0, 1.4), (2.6, -2.6, 0.9), (2.0, -1.5, 0.5), (1.9, -1.3, 0.4))}


def gain(steps):
    run = most = 1.0
    for a, _, _ in steps:
        run = max(run, 1.0) * abs(a)
        most = max(most, run)
    return most


def small_rounded(x, steps, seed=5):
    g = torch.Generator(device=DEV).manual_seed(seed)

    def off(t, bits):
        return t * (1.0 + (2.0 * torch.rand(t.shape, dtype=torch.float64, device=DEV, generator=g) - 1.0) * 2.0 ** -bits)

    x = off(x, 24)
    one = torch.eye(x.shape[0], dtype=torch.float64, device=DEV)
    gram, q = x @ x.t(), one
    for a, b, c in steps:
        p = a * one + b * gram + c * gram @ gram
        q, gram = p @ q, p @ gram @ p
    q, x = off(q, 22), off(x, 22)
    total = torch.zeros_like(x)
    for k in range(x.shape[0]):
        total = off(total + q[:, k:k + 1] * x[k:k + 1], 24)
    return total


def of_rank(rows, cols, rank, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    rank = min(rank, rows, cols)
    return (torch.randn((rows, rank), device=DEV, generator=g, dtype=torch.float64) @ torch.randn((rank, cols), device=DEV, generator=g, dtype=torch.float64)).float()


def check(rows, cols, rank, steps, promised):
    from paper_2505_11432_amd.optim import Orthogonal
    u = of_rank(rows, cols, rank)
    out = Orthogonal(1, rows, cols, out_dtype=torch.float32, coefficients=steps, device=DEV).apply(u[None])[0].double()
    flip = rows > cols
    x = u.double().t().contiguous() if flip else u.double()
    x = x / x.norm()
    want = formula(x, steps)
    model = small_rounded(x, steps) if min(rows, cols) <= 64 else rounded(x, steps, in_pairs(1, rows, cols))
    size = float(want.norm())
    error = float(((out.t() if flip else out) - want).norm())
    assert error <= 2.0 * float((model - want).norm()) + 2.0 ** -22 * math.sqrt(max(x.shape)) * size
    assert error <= promised * size


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(LISTS))
@pytest.mark.parametrize("rows,cols", [(64, 512), (16, 16), (32, 4096), (700, 50), (1, 64)])
@pytest.mark.parametrize("rank", [1, 2, 8, 64])
def test_a_side_of_at_most_64(rows, cols, rank, name):
    """2e-4 for the default steps (2e-5 of full rank: a tenth of the rows' number or more singular values alike), 4e-7 of the gain for others, 1e-5 at least."""
    steps = LISTS[name]
    check(rows, cols, rank, steps, max(1e-5, 4e-7 * gain(steps)))


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols", [(64, 512), (64, 2048), (2048, 64), (50, 300), (64, 64)])
def test_full_rank_with_a_side_of_at_most_64(rows, cols):
    check(rows, cols, 64, LISTS["5"], 2e-5)


@pytest.mark.gpu
@pytest.mark.parametrize("name", [n for n in LISTS if n != "10"])
@pytest.mark.parametrize("rows,cols", [(65, 512), (128, 300), (300, 128), (300, 1000), (512, 512)])
@pytest.mark.parametrize("rank", [1, 2, 16, 512])
def test_larger_sides(rows, cols, rank, name):
    steps = LISTS[name]
    full = rank >= min(rows, cols)
    check(rows, cols, rank, steps, (2e-3 if full else 3e-3) if name == "5" else 4e-3 + 3.5e-5 * gain(steps))


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols", [(1500, 7100), (7100, 1500)])
@pytest.mark.parametrize("rank", [1, 2, 190, 1500])
def test_default_steps_in_pairs(rows, cols, rank):
    check(rows, cols, rank, LISTS["5"], 3e-3 if rank == 1500 else 7e-3)
