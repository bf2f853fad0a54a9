"""What a linear layer of 16-bit operands runs on (dfk_linear_plan.h), compiled for the host: every choice is one that the launchers have and that fits its workspace."""
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SRC = """
#include <cstdio>
#include "dfk_linear_plan.h"
int main() {
    int m, n, k;
    while (scanf("%d %d %d", &m, &n, &k) == 3) {
        const dfk::LinearPlan p = dfk::linear_plan(m, n, k);
        const dfk::LinearTile t = dfk::kLinearTiles[p.stream ? 0 : p.tile];
        printf("%d %d %d %d %d %d %lld %zu %zu\\n", p.stream, p.nt, p.tile, p.splits, t.bm, t.bn, p.stream ? 0ll : dfk::linear_tiles(t, m, n) * p.splits,
               dfk::linear_partial_bytes(m, n, p.splits), dfk::linear_partial_bound(m, n));
    }
}
"""
MAX_ROWS, MAX_OUT, MAX_IN = 1048576, 1 << 20, 131072
TILES = 9


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("linear_plan") / "plan")
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-I", os.path.join(ROOT, "paper_2602_11808_amd", "csrc"), "-x", "c++", "-", "-o", exe],
                   input=SRC, text=True, check=True)

    def run(rows):
        text = "".join("%d %d %d\n" % r for r in rows)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.split("\n")
        return [tuple(map(int, l.split())) for l in out if l]
    return run


def shapes():
    rnd = random.Random(1)
    rows = [(m, n, k) for m in (1, 8, 9, 16, 17, 64, 65, 300, 4096, MAX_ROWS) for n in (1, 15, 128, 4097, 50257, MAX_OUT) for k in (8, 64, 1000, 4096, MAX_IN)]
    for _ in range(4000):
        rows.append((int(2 ** rnd.uniform(0, 20)), int(2 ** rnd.uniform(0, 20)), 8 * int(2 ** rnd.uniform(0, 14))))
    return rows


def test_choices_can_be_launched(ask):
    rows = shapes()
    for (m, n, k), (stream, nt, tile, splits, bm, bn, wgs, need, bound) in zip(rows, ask(rows), strict=True):
        what = (m, n, k, stream, nt, tile, splits)
        if stream:
            assert m <= 64 and splits == 1 and nt in ((1,) if m <= 8 else (1, 2) if m <= 16 else (1, 2, 4)), what
            continue
        assert m > 8 and 0 <= tile < TILES and splits in (1, 2, 4, 8), what
        assert splits == 1 or (k + 63) // 64 >= 4 * splits, what          # each split has steps
        assert need <= bound, what
        assert wgs + 8 <= 2 ** 31 // 512 or m * n * 2 > 2 ** 37, what     # threads of a launch count in 32 bits (a larger result has no room)


def test_workspace_grows_with_rows(ask):
    for n in (1, 7, 128, 4097, 50257, MAX_OUT):
        bounds = [r[8] for r in ask([(m, n, 64) for m in (1, 2, 7, 8, 9, 64, 100, 1000, 65536, MAX_ROWS)])]
        assert bounds == sorted(bounds)


@pytest.mark.parametrize("m,n,k,stream", [(1, 50257, 4096, 1), (8, 50257, 4096, 1), (8, 128, 64, 1), (16, 50257, 4096, 0), (64, 28672, 8192, 0), (65, 4096, 4096, 0),
                                          (4096, 14336, 4096, 0)])
def test_which_kernel(ask, m, n, k, stream):
    """Up to 8 rows the weight stream; tiles beyond 64 rows, and beyond 8 where there are 5e7 weights and more."""
    assert ask([(m, n, k)])[0][0] == stream
