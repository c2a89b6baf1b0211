"""Host-only checks of the range of sizes that the vocabulary loss takes: what the entry points accept, every kernel behind them takes."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2505_11432_amd", "csrc")
F32, BF16 = 0, 1
MOST = 1 << 24

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include <initializer_list>
#include "row_plan.h"
using namespace moe;
static int bad = 0;
#define CHECK(c, ...) do { if (!(c)) { ++bad; if (bad < 20) { std::printf("%s: ", #c); std::printf(__VA_ARGS__); std::printf("\n"); } } } while (0)
int main() {
  // dx in bf16: the rows of G in a tile span less than 4 GiB
  std::srand(1);
  for (int i = 0; i < 200000; ++i) {
    const int V = (1 << 24) - 64 - (std::rand() % (1 << (1 + i % 24))), R = 1 + std::rand() % (1 << (1 + i % 13)), d = 16 * (1 + std::rand() % 400);
    const long ld = (V + 63L) / 64 * 64;
    CHECK(vocab_dx_takes(vocab_dx_tile(R, V, d), ld), "%d rows, %d words, %d wide", R, V, d);
    CHECK(vocab_dx_takes(vocab_dx_tile(R, V, d), ld) == (vocab_dx_tile(R, V, d) * ld * 2 < 4294967296L), "span");
  }
  CHECK(vocab_dx_tile(640, 1 << 23, 256) == 128, "tile");
  CHECK(vocab_dx_tile(256, 8400000, 1024) == 128, "tile");
  CHECK(vocab_dx_tile(8192, 32000, 4096) == 256, "tile");
  // fp32: threads of the launches of a piece
  for (int i = 0; i < 200000; ++i) {
    const int T = 1 + std::rand() % (1 << (1 + i % 24)), V = 1 + std::rand() % (1 << (1 + i / 24 % 24)), d = 16 * (1 + std::rand() % (1 << (1 + i % 16)));
    const int R = vocab_f32_rows(T, V, d);
    CHECK(R >= 1 && R <= T, "%d of %d rows", R, T);
    CHECK(R * 256L < 1L << 32, "%d rows", R);
    for (int columns : {V, d}) CHECK((columns + 63L) / 64 * ((R + 63L) / 64 + 1) * 256 < 1L << 31, "%d rows, %d columns", R, columns);
  }
  CHECK(vocab_f32_rows(1 << 24, 16, 16) == 1 << 23 && vocab_f32_rows(16384, 131072, 4096) == 16384, "rows");
  std::printf("bad %d\n", bad);
  return bad != 0;
}
"""


def test_choices_are_taken(tmp_path):
    src, exe = tmp_path / "p.cpp", tmp_path / "p"
    src.write_text(PROGRAM)
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-O2", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    res = subprocess.run([str(exe)], capture_output=True, text=True)
    assert res.returncode == 0, res.stdout


@pytest.fixture(scope="module")
def lib():
    from paper_2505_11432_amd.build import LIB_PATH, ensure_built
    ensure_built()
    lib = ctypes.CDLL(LIB_PATH)
    P, I, Z = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
    lib.moe_vocab_workspace_bytes.restype = Z
    lib.moe_vocab_loss.argtypes = [P, P, P, P, I, I, I, I, I, P, P, P, P, P, I, I, P, Z, P]
    return lib


def test_most_words(lib):
    size = lib.moe_vocab_workspace_bytes
    for T in (1, 8, 300):
        assert size(T, 16, MOST, BF16, BF16, 0, 1) == size(T, 16, MOST - 63, BF16, F32, 0, 1) == 0
        assert size(T, 16, MOST - 64, BF16, BF16, 0, 1) > 0
        assert size(T, 16, MOST, BF16, BF16, 0, 0) > 0          # a score has no such product
        assert size(T, 16, MOST, F32, F32, 0, 1) > 0
    at = [ctypes.c_void_p(i << 40) for i in range(1, 9)]
    # refused ahead of any launch
    assert lib.moe_vocab_loss(at[0], at[1], at[2], None, BF16, 8, 16, MOST - 63, 0, at[3], at[4], at[5], at[6], at[7], F32, 0, at[0], 1 << 50, None) == -2


def test_most_rows(lib):
    """fp32: not all of 2^24 rows in one piece, whose pass would have 2^32 threads."""
    for gradients in (0, 1):
        assert 0 < lib.moe_vocab_workspace_bytes(MOST, 16, 16, F32, F32, 0, gradients) < MOST * 64 * 4


def test_no_tokens_leave_the_outputs(lib):
    """T = 0 returns without a launch: total, d_w and the rest stay as they were (host memory here, which no kernel could write)."""
    out = (ctypes.c_float * 64)(*([7.0] * 64))
    at = ctypes.cast(out, ctypes.c_void_p)
    ws = ctypes.c_void_p(4096)
    assert lib.moe_vocab_workspace_bytes(0, 16, 4, BF16, F32, 0, 1) > 0
    assert lib.moe_vocab_loss(None, None, None, None, BF16, 0, 16, 4, 0, at, at, at, at, at, F32, 0, ws, 256, None) == 0
    assert list(out) == [7.0] * 64
