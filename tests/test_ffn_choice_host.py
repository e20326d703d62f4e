"""Which kernel and tiles the feed-forward products take (csrc/mosaic_ffn_choice.h), on the CPU: whatever sizes in the range
of the measured cases take is run by test_gpu_layer_ffn_tiles.py, and no size leads outside the limits that the kernels
and the workspace assume."""
import math
import os
import random
import shutil
import subprocess

import pytest

import test_gpu_layer_ffn_tiles as gpu
from paper_2601_06562_amd import binding as b

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="no g++")

PROGRAM = r"""
#include <stdio.h>
#include "mosaic_ffn_choice.h"
using namespace mosaic::ffn;
static void product(const char* name, int mode, int64_t rows_p, int64_t rows_q, int64_t steps, int64_t splits) {
  const int t = choose_tile(mode, rows_p, rows_q, steps, splits).tile;
  const TileGrid g = tile_grid(mode, t, rows_p, rows_q, splits);
  printf(" %s %d %d %d %lld %d", name, t, kTiles[t].p, kTiles[t].q, (long long)g.n, g.blocks);
}
int main() {
  long long T, d, F;
  while (scanf("%lld %lld %lld", &T, &d, &F) == 3) {
    const int64_t rows = T < kLaunchRows ? T : kLaunchRows;
    const GradientPlan plan = plan_gradients(T, (int32_t)d, (int32_t)F);
    printf("few %d parts %d together %d", few_rows(T, (int32_t)F) ? (int)tiles(T, 16) : 0, plan.splits, plan.tile);
    product("forward", kForward, F, rows, tiles(d, kStepK), 1);
    product("recompute", kRecompute, F, rows, tiles(d, kStepK), 1);
    product("dx", kDx, d, rows, 2 * tiles(F, kStepK), plan.splits);
    product("dw", kDw, d, 2 * F, tiles(T, kStepK), 1);
    if (plan.tile >= 0) printf(" joint %lld", (long long)(tile_grid(kDx, plan.tile, d, rows, plan.splits).n + tile_grid(kDw, plan.tile, d, 2 * F, 1).n));
    printf("\n");
  }
}
"""


@pytest.fixture(scope="module")
def choose(tmp_path_factory):
    at = tmp_path_factory.mktemp("choice")
    (at / "choice.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror", "-I" + os.path.join(ROOT, "include"),
                    "-I" + os.path.join(ROOT, "paper_2601_06562_amd", "csrc"), "-o", str(at / "choice"), str(at / "choice.cpp")],
                   check=True)

    def ask(sizes):
        lines = subprocess.run([str(at / "choice")], input="\n".join("%d %d %d" % s for s in sizes), text=True, check=True,
                               stdout=subprocess.PIPE).stdout.splitlines()
        assert len(lines) == len(sizes)
        found = []
        for line in lines:
            w = line.split()
            c = {"few": int(w[1]), "parts": int(w[3]), "together": int(w[5])}
            for i in range(6, 30, 6):
                c[w[i]] = tuple(int(v) for v in w[i + 1:i + 6])                 # tile, P, Q, tiles there are, blocks
            c["joint"] = int(w[31]) if len(w) > 30 else 0
            found.append(c)
        return found
    return ask


def ways(c):
    """What a size runs: (product, tile, several tiles a block), in parts or whole, the gradients in one launch or two."""
    several = {p: c[p][3] > c[p][4] for p in ("forward", "recompute", "dx", "dw")}
    found = {("few", c["few"])} if c["few"] else {("forward", c["forward"][0], several["forward"])}
    return found | {(p, c[p][0], several[p]) for p in ("recompute", "dx", "dw")} | {
        ("parts", c["dx"][0], c["parts"] > 1), ("together", c["together"], c["parts"] > 1)}


def sweep(n, seed):
    rng = random.Random(seed)

    def log(lo, hi):
        return int(math.exp(rng.uniform(math.log(lo), math.log(hi))))
    return [(log(1, 20000), 8 * log(1, 1024), 8 * log(1, 3584)) for _ in range(n)]


def test_the_gpu_tests_run_all_that_sizes_take(choose):
    tested = set().union(*(ways(c) for c in choose(gpu.SIZES)))
    taken = {}
    for size, c in zip(sweep(30000, 1), choose(sweep(30000, 1))):
        for w in ways(c):
            taken.setdefault(w, size)
    missing = {w: size for w, size in taken.items() if w not in tested}
    assert not missing
    for product, tiles in (("forward", 10), ("recompute", 10), ("dx", 7), ("dw", 7)):
        assert {w[1] for w in tested if w[0] == product} == set(range(tiles))
        assert any(w[0] == product and w[2] is True for w in tested)


def test_the_sizes_are_ragged():
    assert all(T % 16 and d % 64 and F % 64 for T, d, F in gpu.SIZES if T != 9248 and T != 8200)
    assert any(d % 64 and -(-d // 64) >= 16 for _, d, _ in gpu.SIZES)


def test_limits(choose):
    edge = [(T, d, F) for T in (0, 1, 64, 65, 4096, 4097, 131071, 131072, 131073, (1 << 31) - 1)
            for d in (8, 16384, 1 << 17) for F in (8, 4096, 4104, 1 << 17)]
    sizes = edge + sweep(20000, 2)
    for (T, d, F), c in zip(sizes, choose(sizes)):
        for p in ("forward", "recompute", "dx", "dw"):
            tile, tp, _, n, blocks = c[p]
            assert 0 <= n < 1 << 31 and blocks <= min(n, 512) and (blocks > 0) == (n > 0)
            assert tp & (tp - 1) == 0 or p in ("forward", "recompute")           # across K rows are a power of two
        assert c["joint"] <= 2048 and (T <= 131072 or (c["together"] == -1 and c["parts"] == 1))
        assert c["few"] <= 4 and (not c["few"] or T <= 64)
        # the sums of dx lie behind dg | du in the workspace
        if c["parts"] > 1:
            assert 4 * T * F + 4 * c["parts"] * T * d <= b.mosaic_gated_ffn_backward_workspace_bytes(T, d, F)
