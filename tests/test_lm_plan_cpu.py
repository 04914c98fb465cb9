"""The planners of the grouped products, compiled for the host: the shapes of their GPU
tests reach every tile that is built, with whole and with partial stages, and the split
reduction; split sums are what the workspace query answers."""
import os
import random
import shutil
import subprocess

import pytest

import paper_2112_10769_amd as luq

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PLAN = r"""
#include <stdio.h>
#include "grouped_plan.hpp"
int main() {
  char kind;
  long T, a, b, experts;
  while (scanf(" %c %ld %ld %ld %ld", &kind, &T, &a, &b, &experts) == 5) {
    if (kind == 'r') printf("%d 1\n", (int)luq::plan_rows(T, a, b, experts));
    else {
      const luq::DepthPlan p = luq::plan_depth(T, a, b, experts);
      printf("%d %d\n", (int)p.tile, p.splits);
    }
  }
}
"""
TILES = ["256x256", "128x256", "128x128", "64x128", "64x64", "32x64", "32x32", "64x64k1"]
DEPTH = dict(zip(TILES, (128, 128, 128, 256, 512, 512, 1024, 128)))


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("no hipcc")
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.hip").write_text(PLAN)
    pkg = os.path.join(ROOT, "paper_2112_10769_amd", "csrc")
    subprocess.run([hipcc, "--cuda-host-only", "-std=c++17", "-O1", "-I", pkg, "-I", os.path.join(ROOT, "include"),
                    str(d / "plan.hip"), "-o", str(d / "plan")], check=True, capture_output=True)

    def ask(shapes):
        text = "\n".join(" ".join(str(v) for v in s) for s in shapes)
        out = subprocess.run([str(d / "plan")], input=text, check=True, capture_output=True, text=True).stdout
        return [(TILES[int(t)], int(s)) for t, s in (line.split() for line in out.splitlines())]
    return ask


def test_rows_shapes_reach_every_tile(plans):
    from test_gpu_grouped import LARGE_ROWS, rows_shapes
    shapes = [("r", T, N, K, E) for E, T, N, K in rows_shapes()]
    got = {(t, s[3] % DEPTH[t] == 0) for s, (t, _) in zip(shapes, plans(shapes))}
    tiles = ("256x256", "128x128", "64x128", "32x64", "32x32", "64x64k1")
    assert not {(t, w) for t in tiles for w in (True, False)} - got
    assert {t for t, _ in got} <= set(tiles)
    assert LARGE_ROWS


def test_depth_shapes_reach_every_tile(plans):
    from test_gpu_grouped import depth_shapes
    got = plans([("d", T, M, N, E) for E, T, M, N in depth_shapes()])
    assert {t for t, _ in got} == {"256x256", "128x256", "128x128", "64x128", "32x64", "64x64k1"}
    assert any(s > 1 for _, s in got) and any(s == 1 for _, s in got)


def test_long_batches_are_split(plans):
    """A chunk of the stages of a group that has the whole batch is int32-exact."""
    rng = random.Random(4)
    shapes = [(T, rng.randint(1, 3000), rng.randint(1, 3000), rng.randint(1, 40))
              for T in ((1 << 18) + 128, 1 << 19, (1 << 19) + 128, (1 << 21) - 128, 1 << 22)
              for _ in range(20)]
    for (T, M, N, E), (tile, splits) in zip(shapes, plans([("d", *s) for s in shapes])):
        stages = -(-T // DEPTH[tile])
        assert -(-stages // splits) * DEPTH[tile] <= 1 << 18, (T, M, N, E, tile, splits)
        assert luq.grouped_wgrad_workspace(T, M, N, E) == 4 * splits * E * M * N
    assert luq.grouped_wgrad_workspace((1 << 22) + 128, 1, 1, 1) == 0


def test_grids_of_large_outputs(plans):
    """Up to 2^36 outputs; a tile is only taken where its grid has below 2^32 threads."""
    rng = random.Random(5)
    rows, depths = [(1 << 18, 1 << 15, 32, 8), (1 << 17, 1 << 16, 4096, 64), (1 << 30, 33, 32, 1), (1 << 30, 64, 64, 4096),
                    (1, 1 << 29, 32, 1), (1 << 20, 1 << 16, 64, 2)], [(64, 1 << 14, 1 << 13, 128), (64, 1 << 18, 1 << 18, 1)]
    rows += [(2 ** rng.randint(13, 18), 2 ** rng.randint(12, 18), 2 ** rng.randint(5, 12), 2 ** rng.randint(0, 12))
             for _ in range(200)]
    for (T, N, K, E), (tile, _) in zip(rows, plans([("r", *s) for s in rows])):
        m, n = (64, 64) if tile == "64x64k1" else map(int, tile.split("x"))
        assert (T // m + min(E, T) + 1) * -(-N // n) < 1 << 23, (T, N, K, E, tile)
    for (T, M, N, E), (tile, _) in zip(depths, plans([("d", *s) for s in depths])):
        m, n = (64, 64) if tile == "64x64k1" else map(int, tile.split("x"))
        assert -(-(-(-M // m) * -(-N // n)) // 8) * 8 * E < 1 << 23, (T, M, N, E, tile)


def test_workspace_is_the_plans(plans):
    rng = random.Random(3)
    shapes = [(32 * rng.randint(1, 1 << rng.randint(0, 13)), rng.randint(1, 3000), rng.randint(1, 3000), rng.randint(1, 40))
              for _ in range(300)]
    for (T, M, N, E), (_, splits) in zip(shapes, plans([("d", *s) for s in shapes])):
        assert luq.grouped_wgrad_workspace(T, M, N, E) == (4 * splits * E * M * N if splits > 1 else 0)
        assert 1 <= splits <= 16
