"""Host-only checks of the choices for the vocabulary products (row_plan.h is host code without HIP): what fits the scratch that is asked for, and
that a choice is one that its kernels can take."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2505_11432_amd", "csrc")

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include <initializer_list>
#include "row_plan.h"
using namespace moe;
static int bad = 0;
#define CHECK(c, ...) do { if (!(c)) { ++bad; if (bad < 20) { std::printf("%s: ", #c); std::printf(__VA_ARGS__); std::printf("\n"); } } } while (0)
static long up(long a, long b) { return (a + b - 1) / b; }
int main() {
  const CutCost costs[] = {{13000, 1500, 105, 0}, {6000, 660, 26, 0}, {13000, 1500, 105, 4000}, {11000, 750, 26, 4000}};
  std::srand(1);
  for (int i = 0; i < 200000; ++i) {
    const CutCost c = costs[i % 4];
    const int groups = i % 4 == 3 ? 512 : 256, bound_steps = 1 + std::rand() % 3000;
    const long bound_tiles = 1 + std::rand() % 3000;
    // the device knows fewer rows than the bound: fewer tiles, or fewer steps
    const long tiles = 1 + std::rand() % bound_tiles;
    const int steps = 1 + std::rand() % bound_steps, rem = (int)(tiles % groups);
    if (!rem) continue;
    const int parts = cut_parts(rem, groups, steps, c);
    CHECK(parts >= 1 && parts <= kCutMost, "%d", parts);
    CHECK(parts == 1 || parts * 4 <= steps, "%d parts of %d steps", parts, steps);
    CHECK(parts == 1 || (long)rem * parts <= cut_items(bound_tiles, groups, bound_steps), "%d x %d items, bound %ld", rem, parts,
          cut_items(bound_tiles, groups, bound_steps));
    CHECK(cut_ns(parts, rem, groups, steps, c) <= cut_ns(1, rem, groups, steps, c), "slower than whole");
  }
  // one tile more than a round is cut, a full round is not
  CHECK(cut_parts(1, 256, 1600, costs[0]) >= 32, "%d", cut_parts(1, 256, 1600, costs[0]));
  CHECK(cut_parts(255, 256, 1600, costs[0]) == 1, "%d", cut_parts(255, 256, 1600, costs[0]));
  for (int R = 1; R <= 3000; R += 7)
    for (int V : {100, 5003, 32000, 131072})
      for (int d : {16, 1024, 4096}) {
        CHECK(vocab_tile(R, V, d, true) != VocabTile::ROWS320, "%d %d %d", R, V, d);
        if (R <= 64 && (long)up(V, 128) <= 256) CHECK(vocab_tile(R, V, d, false) == VocabTile::ROWS64 || d < 64, "%d %d %d", R, V, d);
      }
  for (int i = 0; i < 100000; ++i) {
    const bool rows = i & 1;
    const F32Product p{rows, 1 + std::rand() % 20000, 16 * (1 + std::rand() % 300), 1 + std::rand() % 40000, 1};
    const long room = std::rand() % 40;
    const F32Plan q = f32_parts(p, room), z = f32_logit_parts(p, room);
    const int steps = f32_steps(p);
    CHECK(q.parts >= 1 && (q.parts == 1 || (q.parts <= room && q.parts <= 32 && steps / q.parts >= 4)), "%d parts, room %ld, %d steps", q.parts, room, steps);
    CHECK(z.parts == 1 || (z.parts == 2 && room >= 2 && steps >= 24), "%d", z.parts);
    CHECK(q.tile != F32_128_EIGHT && z.tile == F32_64, "tile");
  }
  std::printf("bad %d\n", bad);
  return bad != 0;
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    src, exe = d / "p.cpp", d / "p"
    src.write_text(PROGRAM)
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-O2", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    return str(exe)


def test_choices_fit(program):
    res = subprocess.run([program], capture_output=True, text=True)
    assert res.returncode == 0, res.stdout
