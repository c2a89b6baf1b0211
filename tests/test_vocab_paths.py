"""The tiles and cuts of the bf16 vocabulary products that large steps take, each at the smallest sizes that take it: 256 x 256 and 128 x 128 tiles,
whole and cut along the contraction, written and added to, in one piece and in several.  A host test pins which sizes take what (row_plan.h), a GPU test
compares with 64 bits.

Tolerances, u16 = 2^-8: dx two roundings (G and the result), d_w in fp32 one (G), in bf16 two, and one more of the sum where it is added to.  They hold for
the norm of the whole and for every block of 128 x 128, which a lost tile or part would miss; for a block of the share of the whole's norm as well, as a
block may be small by cancellation."""
import math
import os
import subprocess

import pytest
import torch

DEV, U16 = "cuda:0", 2.0 ** -8
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2505_11432_amd", "csrc")

# T, d, V, rows of a piece (0: all) -> of a piece: dx tile, dx cut, dx has whole tiles; d_w tile, d_w cut, d_w has whole tiles
CASES = {
    (1100, 64, 700, 0): (128, 1, 0, 128, 1, 0),
    (1025, 272, 1537, 0): (128, 1, 0, 128, 1, 0),
    (8200, 160, 5000, 0): (256, 1, 0, 128, 1, 0),
    (4100, 4096, 515, 0): (256, 1, 1, 128, 1, 0),
    (8200, 160, 20000, 0): (256, 1, 0, 256, 1, 0),
    (1500, 3584, 5000, 0): (256, 1, 0, 256, 1, 1),
    (4500, 64, 700, 2048): (128, 1, 0, 128, 1, 0),
    (12000, 160, 20000, 8192): (256, 1, 0, 256, 1, 0),
}

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include "row_plan.h"
using namespace moe;
static long up(long a, long b) { return (a + b - 1) / b; }
static void product(int tile, long tiles, int groups, int steps, CutCost c) {
  const int rem = (int)(tiles % groups);
  std::printf("%d %d %d ", tile, rem && cut_parts(rem, groups, steps, c) > 1, tiles >= groups);
}
int main(int, char** a) {
  const int R = std::atoi(a[1]), d = std::atoi(a[2]), V = std::atoi(a[3]), dx = vocab_dx_tile(R, V, d), dw = vocab_dw_pairs(R, V, d) ? 128 : 256;
  product(dx, up(R, dx) * up(d, dx), kPlanGroups, (int)up(V, 64), dx == 256 ? kDxFull : kDxMid);
  product(dw, up(V, dw) * up(d, dw), dw == 128 ? 2 * kPlanGroups : kPlanGroups, (int)up(R, 64), dw == 128 ? kDwPair : kDwFull);
}
"""


def test_the_sizes_take_these_paths(tmp_path):
    src, exe = tmp_path / "p.cpp", tmp_path / "p"
    src.write_text(PROGRAM)
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-O2", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    got = {}
    for T, d, V, piece in CASES:
        out = subprocess.run([str(exe), str(piece or T), str(d), str(V)], capture_output=True, text=True, check=True).stdout
        got[T, d, V, piece] = tuple(int(x) for x in out.split())
    assert got == CASES


def close(got, want, tol, add=0.0):
    """|got - want| within tol of want's norm, plus `add`, for the whole and by blocks."""
    far, size = (got.double() - want), want
    assert float(far.norm()) <= tol * float(size.norm()) + add
    pad = lambda t: torch.nn.functional.pad(t, (0, -t.shape[1] % 128, 0, -t.shape[0] % 128)).unfold(0, 128, 128).unfold(1, 128, 128)
    far, size = pad(far).flatten(2).norm(dim=2), pad(size).flatten(2).norm(dim=2)
    share = float(size.norm()) / math.sqrt(size.numel())
    assert bool((far <= tol * (size + share) + add).all())


@pytest.mark.gpu
@pytest.mark.parametrize("T,d,V,piece", CASES)
@pytest.mark.parametrize("grad", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("ignored", [0.0, 0.4])
def test_against_64_bits(T, d, V, piece, grad, ignored):
    from paper_2505_11432_amd.head import VocabLoss
    g = torch.Generator(device=DEV).manual_seed(T + V)
    w = (torch.randn((V, d), device=DEV, generator=g) * (1.28 / math.sqrt(d))).to(torch.bfloat16)
    target = torch.randint(0, V, (T,), device=DEV, generator=g)
    x = (torch.randn((T, d), device=DEV, generator=g) + 6.0 * torch.rand((T, 1), device=DEV, generator=g) * w[target].float()).to(torch.bfloat16)
    keep = torch.rand((T,), device=DEV, generator=g) >= ignored
    token_w = torch.rand((T,), device=DEV, generator=g) / T
    for weights in (None, token_w):
        op = VocabLoss(T, d, V, grad_dtype=grad, piece_bytes=(1 << 40) if piece == 0 else piece * ((V + 63) // 64 * 64) * 2)
        assert op.piece_rows == piece
        tg = torch.where(keep, target, torch.full_like(target, -100)).to(torch.int32)
        op.step(x, w, tg, token_w=weights)
        xd, wd = x.double(), w.double()
        p = xd @ wd.t()
        p -= torch.logsumexp(p, 1, keepdim=True)
        p.exp_()
        p.scatter_add_(1, target[:, None], torch.full((T, 1), -1.0, dtype=torch.float64, device=DEV))
        p *= (keep * (weights.double() if weights is not None else 1.0 / int(keep.sum())))[:, None]
        dx, d_w = p @ wd, p.t() @ xd
        del p
        close(op.dx, dx, 2 * U16)
        close(op.d_w, d_w, U16 if grad == torch.float32 else 2 * U16)
        # added to what is there, of the same size
        op.d_w.normal_(0.0, float(d_w.norm()) / math.sqrt(d_w.numel()), generator=g)
        was = op.d_w.double()
        op.step(x, w, tg, token_w=weights, accumulate=True)
        close(op.d_w, was + d_w, U16 if grad == torch.float32 else 2 * U16)
