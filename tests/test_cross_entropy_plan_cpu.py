"""The planner of the cross entropy, compiled for the host: the shapes of its GPU tests reach every kernel that is
launched, so that a rule that chooses others cannot leave one untested; the workspace queries answer what it needs."""
import os
import random
import shutil
import subprocess

import pytest

torch = pytest.importorskip("torch")
luq = pytest.importorskip("paper_2112_10769_amd")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PLAN = r"""
#include <stdio.h>
#include "cross_entropy_plan.hpp"
int main() {
  long T, V, D;
  int x, t, g;   // whether the tensor is bf16; g: -1 for the forward call
  while (scanf("%ld %ld %ld %d %d %d", &T, &V, &D, &x, &t, &g) == 6) {
    luq::Layout l(T, V, D, x, t, g >= 0);
    if (g < 0) l.forward();
    else l.backward(x, g);
    printf("%d %d %ld", (int)l.z.edge, luq::pairs_of(l.xn, l.tn).count, (long)l.bytes);
    if (g < 0) printf(" %ld\n", (long)l.parts);
    else printf(" %ld %ld %d %d %d %d %d\n", (long)l.pieces, (long)l.piece, l.g_terms(), (int)l.by_x.edge, l.by_x.splits,
                (int)l.by_w.edge, l.by_w.splits);
  }
}
"""
TILES = ["32x64", "128x128", "128x128 deep", "256x256"]
OUT_TILES = TILES[1:]


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
        text = "\n".join(" ".join(str(int(v)) for v in s) for s in shapes)
        out = subprocess.run([str(d / "plan")], input=text, check=True, capture_output=True, text=True).stdout
        return [[int(v) for v in line.split()] for line in out.splitlines()]
    return ask


def _bf16(*types):
    return [int(t == "bf16") for t in types]


def test_shapes_reach_every_kernel(plans):
    from test_gpu_cross_entropy_tiles import SHAPES
    assert all(T == 1 or T % 32 for T, *_ in SHAPES) and any(V % 8 for _, V, *_ in SHAPES)
    logits, grads, rows, tables, joins, pieces = set(), set(), set(), set(), set(), set()
    forward = plans([(*s[:3], *_bf16(s[3], s[4]), -1) for s in SHAPES])
    backward = plans([(*s[:3], *_bf16(*s[3:6])) for s in SHAPES])
    for (T, V, D, xt, tt, gt, add), (edge, pairs, _, parts), (z, _, _, n, piece, terms, bx, sx, bw, sw) in zip(SHAPES, forward, backward):
        logits.add((TILES[edge], pairs))
        # joins: a workgroup a row, or 16 waves four parts at a time, in one round or in several
        joins.add((T <= 128, parts > (1024 if T <= 128 else 64)))
        grads.add((TILES[z], terms))
        rows.add((TILES[bx], sx > 1, xt))
        tables.add((TILES[bw], sw > 1, gt, add))
        if n > 1:   # dx is written by the last piece, or by the join of the splits
            pieces |= {("dx", sx > 1, xt), ("dtable", gt, add), ("last piece ragged", (V - (n - 1) * piece) % 8 > 0)}
    both, types = (True, False), ("bf16", "f32")
    assert logits == {(t, n) for t in TILES for n in (1, 3, 6)}
    assert grads == {(t, n) for t in TILES for n in (1, 3)}
    assert rows == {(t, s, x) for t in OUT_TILES for s in both for x in types}
    assert tables == {(t, s, g, a) for t in OUT_TILES for s in both for g in types for a in (0, 1)}
    assert joins == {(a, b) for a in both for b in both}
    assert pieces >= {("dx", s, x) for s in both for x in types} | {("dtable", g, a) for g in types for a in (0, 1)}
    assert ("last piece ragged", True) in pieces


def _drawn(n, seed):
    rng = random.Random(seed)

    def size(most):
        return int(2 ** rng.uniform(0, most))
    shapes = []
    while len(shapes) < n:
        T, V, D = size(21), size(28), size(17)
        if T * V <= 1 << 37 and T * D <= 1 << 36 and V * D <= 1 << 36:
            x, t, g = rng.choice([(1, 1, 1), (1, 1, 0), (0, 0, 0), (1, 0, 0), (0, 1, 0), (0, 1, 1)])
            shapes.append((T, V, D, x, t, g))
    return shapes + [(1 << 21, 1 << 16, 1 << 15, 1, 1, 1), (1 << 9, 1 << 28, 1 << 8, 1, 1, 0), (1, 1 << 28, 256, 0, 0, 0),
                     (1 << 19, 1 << 18, 1 << 17, 0, 0, 0), (33, 1 << 28, 1, 1, 1, 0), (1 << 21, 1, 1, 0, 0, 0)]


def test_every_size_has_a_grid(plans):
    """Over the accepted sizes: tiles and splits whose grids have below 2^32 threads, pieces that cover the table, rows
    of a piece that a descriptor's 32-bit offsets reach."""
    edge = {"32x64": (32, 64, 128), "128x128": (128, 128, 256), "128x128 deep": (128, 128, 512), "256x256": (256, 256, 512)}

    def threads(tile, M, N):
        m, n, t = edge[TILES[tile]]
        return -(-M // m) * -(-N // n) * t
    shapes = _drawn(2000, 1)
    forward, backward = plans([(*s[:5], -1) for s in shapes]), plans(shapes)
    for s, (z, _, _, parts), (zb, _, _, n, piece, _, bx, sx, bw, sw) in zip(shapes, forward, backward):
        T, V, D = s[:3]
        assert threads(z, T, V) < 1 << 32 and parts == -(-V // edge[TILES[z]][1]), s
        rows = min(piece, V)
        assert (n - 1) * piece < V <= n * piece and piece % 128 == 0 and piece * 2 * 256 < 1 << 31, s
        assert TILES[bx] in OUT_TILES and TILES[bw] in OUT_TILES and 1 <= sx <= 64 and 1 <= sw <= 64, s
        for tile, M, N in ((zb, T, rows), (bx, T, D), (bw, rows, D)):
            assert threads(tile, M, N) < 1 << 32, s


def test_workspaces_are_the_plans(plans):
    names = {0: luq.LUQ_F32, 1: luq.LUQ_BF16}
    shapes = _drawn(300, 2)
    for gt in (False, True):
        for s, plan in zip(shapes, plans([(*s[:5], s[5] if gt else -1) for s in shapes])):
            got = luq.LIB.luq_cross_entropy_workspace(*s[:3], names[s[3]], names[s[4]], names[s[5]] if gt else -1)
            assert got == plan[2], s
