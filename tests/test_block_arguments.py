"""Host-only checks of arguments of the calls around the layer, beside those of test_block_abi.  Nothing here reaches a stream."""
import ctypes
import os
import subprocess

import pytest

P, I, Z, D = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t, ctypes.c_double
NULL = P(0)
F32, BF16 = 0, 1
MB = 1 << 20


@pytest.fixture(scope="module")
def lib():
    from paper_2505_11432_amd.build import LIB_PATH, ensure_built
    ensure_built()
    lib = ctypes.CDLL(LIB_PATH)
    lib.moe_embedding_workspace_bytes.restype = lib.moe_block_norm_workspace_bytes.restype = lib.moe_orthogonal_workspace_bytes.restype = Z
    lib.moe_muon_eps.argtypes = [P, P, I, P, P, I, I, I, P, P, D, I, D, D, D, I, P, I, P, Z, P]
    return lib


def test_muon_eps(lib):
    need = lib.moe_orthogonal_workspace_bytes(2, 8, 8, 0)

    def muon(eps, batch=2, p=P(MB), steps=5, n=need):
        return lib.moe_muon_eps(p, P(2 * MB), F32, P(3 * MB), NULL, batch, 8, 8, P(5 * MB), NULL, 0.9, 1, 0.1, 1.0, eps, steps, NULL, 0, P(6 * MB), n, None)

    assert muon(-1e-9) == muon(float("nan")) == muon(1e-7, p=NULL) == muon(1e-7, steps=0) == -1
    assert muon(1e-7, n=need - 1) == muon(0.0, n=need - 1) == -3
    assert muon(1e-7, batch=0) == muon(0.0, batch=0) == 0


def test_gain_of_the_steps(lib):
    """Lists whose small singular values, and roundings with them, are multiplied by more than 8192, or 262144 with a side of at most 64, are refused: -2.  Others
    go on to the workspace, which is too small here: -3."""
    lib.moe_orthogonalize.argtypes = [P, I, I, I, I, I, P, I, P, I, P, Z, P]
    lib.moe_muon.argtypes = [P, P, I, P, P, I, I, I, P, P, D, I, D, D, I, P, I, P, Z, P]

    def both(rows, cols, steps, c=None):
        c = NULL if c is None else ctypes.cast((D * (3 * steps))(*[v for row in c for v in row]), P)
        a = lib.moe_orthogonalize(P(64 * MB), F32, 1, rows, cols, steps, c, 0, P(128 * MB), F32, P(256 * MB), 16, None)
        b = lib.moe_muon(P(64 * MB), P(128 * MB), F32, P(192 * MB), NULL, 1, rows, cols, P(MB), NULL, 0.9, 1, 0.1, 1.0, steps, c, 0, P(256 * MB), 16, None)
        assert a == b
        return a

    for rows, cols in ((65, 65), (65, 4000), (4000, 65)):
        assert both(rows, cols, 7) == -3 and both(rows, cols, 8) == both(rows, cols, 16) == -2
    for rows, cols in ((64, 64), (64, 4000), (4000, 64), (1, 1)):
        assert both(rows, cols, 10) == -3 and both(rows, cols, 11) == both(rows, cols, 16) == -2
    slow, still = (2.0, -1.5, 0.5), (0.5, 0.0, 0.0)
    assert both(100, 100, 13, [slow] * 13) == -3 and both(100, 100, 14, [slow] * 14) == -2
    assert both(60, 100, 14, [slow] * 14) == -3 and both(60, 100, 16, [slow] * 16) == -3
    # (what a later step makes smaller again was large on the way; what an earlier one made smaller is no gain)
    assert both(100, 100, 15, [slow] * 14 + [still]) == -2
    assert both(100, 100, 14, [still] + [slow] * 13) == -3 and both(100, 100, 15, [still] + [slow] * 14) == -2
    assert both(100, 100, 16, [(1.5, -0.5, 0.0)] * 16) == -3


def test_orthogonal_workspace(lib):
    """What is asked for beside the matrices: nothing for parts of tiles where no tile is cut; more matrices never need less."""
    size = lib.moe_orthogonal_workspace_bytes
    assert size(1, 65, 65, 0) < MB and size(1, 300, 1000, 0) < 8 * MB and size(1, 1, 1, 0) < MB
    for rows, cols in ((65, 65), (300, 1000), (520, 9000), (2000, 2000), (128, 16384), (1500, 7100)):
        sizes = [size(n, rows, cols, 0) for n in range(1, 40)]
        assert sizes == sorted(sizes)
        x, gram = 2 * (-(-rows // 128) * 128) * (-(-cols // 128) * 128), 2 * (-(-min(rows, cols) // 128) * 128) ** 2
        for n, s in enumerate(sizes, 1):
            assert n * (4 * x + 2 * gram) < s <= n * (4 * x + 4 * gram) + 128 * MB + 64 * 1024


def test_matrices_at_a_time():
    from paper_2505_11432_amd import binding as B
    from paper_2505_11432_amd.optim import _piece
    assert _piece(4096, 100, 100, 64 * MB) > 300 and _piece(100, 300, 1000, 64 * MB) > 4
    assert _piece(0, 100, 100, MB) == _piece(1, 100, 100, 1) == _piece(9, 100, 100, 1) == 1
    for batch, rows, cols, most in ((64, 2048, 1408, 8 << 30), (64, 2048, 1408, 1 << 30), (50000, 16, 16, 1 << 30), (7, 4096, 14336, 2 << 30)):
        piece = _piece(batch, rows, cols, most)
        assert 1 <= piece <= min(batch, 32768) and 0 < B.moe_orthogonal_workspace_bytes(batch, rows, cols, piece)
        assert piece == 1 or B.moe_orthogonal_workspace_bytes(batch, rows, cols, piece) <= most
    with pytest.raises(AssertionError):
        _piece(1, (1 << 20) + 1, 8, MB)


PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include "orth_tiles.h"
using namespace moe;
int main() {
  std::srand(3);
  long bad = 0, cut = 0;
  for (int i = 0; i < 3000; ++i) {
    const bool symmetric = i & 1;
    const int M = 128 * (1 + std::rand() % (i % 3 ? 12 : 60)), N = symmetric ? M : 128 * (1 + std::rand() % (i % 3 ? 12 : 60)), K = 128 * (1 + std::rand() % (i % 5 ? 20 : 130));
    const OrthTiles t = orth_tiles(symmetric, M, N);
    long before = 0;
    for (int n = 1; n <= 300; ++n) {
      const long bound = orth_most_parts(symmetric, M, N, K, n);
      bad += bound < before || bound > kMostParts;
      before = bound;
      const Cut c = cut_of(t.large * n, K / kOrthStep);
      const long parts = small_tiles_time(t.small * n, K / kOrthStep) < c.time || c.split == 1 ? 0 : (t.large * n - c.full) * c.split;
      cut += parts > 0;
      if (parts > bound && bad++ < 10) std::printf("%d x %d x %d, %d: %ld parts, bound %ld\n", M, N, K, n, parts, bound);
    }
  }
  std::printf("bad %ld, cut %ld\n", bad, cut);
  return bad != 0 || cut < 1000;
}
"""


def test_parts_fit(tmp_path):
    """The parts of cut tiles, for the chosen tiles of every number of matrices, lie within what the workspace holds (orth_tiles.h is host code without HIP)."""
    src, exe = tmp_path / "p.cpp", tmp_path / "p"
    src.write_text(PROGRAM)
    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2505_11432_amd", "csrc")
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-O2", "-I", csrc, str(src), "-o", str(exe)], check=True)
    res = subprocess.run([str(exe)], capture_output=True, text=True)
    assert res.returncode == 0, res.stdout


def test_norm_gradients_in_place(lib):
    """dx may be d_out or d_h, dy y or the other of them: what is allowed goes on to the workspace, which is too small here (-3), y for dx is not."""
    lib.moe_block_norm_bwd.argtypes = [P] * 7 + [I, I, I, I, D, D] + [P] * 5 + [I, P, Z, P]
    need = lib.moe_block_norm_workspace_bytes(8, 64, BF16, 1, 1, 1)

    def bwd(dx, dy, y=P(2 * MB), n=need):
        return lib.moe_block_norm_bwd(P(MB), y, P(3 * MB), P(4 * MB), P(5 * MB), P(6 * MB), P(7 * MB), BF16, 8, 64, 4, 1.0, 1e-6, dx, dy, P(10 * MB), P(11 * MB),
                                      P(12 * MB), 0, P(13 * MB), n, None)

    y, d_out, d_h = P(2 * MB), P(6 * MB), P(7 * MB)
    for dy in (P(9 * MB), d_out, d_h):
        assert bwd(y, dy) == -1
    assert bwd(d_out, d_out) == bwd(d_h, d_h) == -1
    for dx in (P(8 * MB), d_out, d_h):
        assert bwd(dx, y, n=need - 1) == bwd(dx, P(9 * MB), n=need - 1) == -3


def test_embedding_scale(lib):
    """A scale that is no finite number in fp32 would make NaN of padding's rows of zeros: -1.  (A batch of none does nothing; a workspace of none is refused.)"""
    lib.moe_embedding_fwd.argtypes = [P, P, I, I, I, I, D, P, P]
    lib.moe_embedding_bwd.argtypes = [P, P, I, I, I, I, D, P, I, I, P, Z, P]
    for scale in (float("nan"), float("inf"), -float("inf"), 1e39):
        assert lib.moe_embedding_fwd(P(MB), P(2 * MB), BF16, 8, 64, 100, scale, P(3 * MB), None) == -1
        assert lib.moe_embedding_bwd(P(2 * MB), P(MB), BF16, 8, 64, 100, scale, P(3 * MB), F32, 0, P(4 * MB), MB, None) == -1
    for scale in (0.0, -0.5, 3e38):
        assert lib.moe_embedding_fwd(NULL, NULL, BF16, 0, 64, 100, scale, NULL, None) == 0
        assert lib.moe_embedding_bwd(P(2 * MB), P(MB), BF16, 8, 64, 100, scale, P(3 * MB), F32, 0, NULL, 0, None) == -3


def test_norm_rows(lib):
    """A team's share of the rows ends within 31 bits."""
    lib.moe_block_norm_fwd.argtypes = [P, P, P, P, P, I, I, I, I, D, D, P, P, P]
    lib.moe_block_norm_bwd.argtypes = [P] * 7 + [I, I, I, I, D, D] + [P] * 5 + [I, P, Z, P]
    most = 0x7f000000
    for T in (most + 1, 2 ** 31 - 2048, 2 ** 31 - 1):
        assert lib.moe_block_norm_workspace_bytes(T, 16, BF16, 0, 0, 1) == 0
        assert lib.moe_block_norm_fwd(P(MB), NULL, NULL, NULL, P(5 * MB), BF16, T, 16, 1, 1.0, 1e-6, NULL, P(7 * MB), None) == -2
        assert lib.moe_block_norm_bwd(P(MB), NULL, NULL, NULL, P(5 * MB), NULL, P(7 * MB), BF16, T, 16, 1, 1.0, 1e-6, P(8 * MB), NULL, NULL, NULL, P(12 * MB), 0, P(13 * MB),
                                      Z(1 << 40), None) == -2
    # one list of sums for each of at most 2048 teams
    assert 0 < lib.moe_block_norm_workspace_bytes(most, 16, BF16, 0, 0, 1) <= 2048 * 16 * 4 + 256


def test_coefficients():
    """Steps that are made into bytes once are used as they are; a number of steps beyond their bytes, which would be read past their end, is none."""
    import torch

    from paper_2505_11432_amd import binding as B
    steps, packed = made = B._coefficients(B.COEFFICIENTS)
    assert steps == 5 and len(packed) == 120 and B._coefficients(made) == made
    x = torch.zeros((1, 8, 8))
    w = torch.zeros((16,), dtype=torch.uint8)
    for bad in ((), ((1.0, 2.0),), ((1.0, 0.0, 0.0),) * 17, (16, packed), (5, packed[:-8]), (0, b"")):
        with pytest.raises(AssertionError, match="coefficients"):
            B.moe_orthogonalize(x, x, w, coefficients=bad)
        with pytest.raises(AssertionError, match="coefficients"):
            B.moe_muon(x, x, x, None, w, None, 0.9, True, 0.0, 1.0, w, coefficients=bad)
