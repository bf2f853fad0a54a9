"""What a product with MXFP4 weights runs on (dfk_mx_plan.h), compiled for the host: every choice is one that the launchers have and that fits LDS and its workspace; the shapes that the GPU
tests run cover every one."""
import os
import random
import subprocess

import pytest

from tests.mx_ref import EVERY_KERNEL, FP8

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SRC = """
#include <cstdio>
#include "dfk_mx_plan.h"
int main() {
    int m, n, k, x8, gated, f32;
    while (scanf("%d %d %d %d %d %d", &m, &n, &k, &x8, &gated, &f32) == 6) {
        const dfk::MxPlan p = dfk::mx_plan(m, n, k, x8, gated, f32);
        const dfk::MxTile& t = dfk::kMxTiles[p.tile];
        const int cols = gated ? t.bn / 2 : t.bn;
        const size_t lds = p.form >= 0 ? dfk::mx_stream_lds(dfk::kMxStreams[p.form], x8, m, k) : 0;
        printf("%d %d %d %d %zu %lld %zu %zu %d\\n", p.form, p.tile, p.splits, t.per_cu[x8], lds, (long long)((m + t.bm - 1) / t.bm) * ((n + cols - 1) / cols) * p.splits,
               dfk::linear_partial_bytes(m, n, p.splits), dfk::linear_partial_bound(m, n),
               (int)(gated ? p.form >= dfk::kMxStreamGated && p.form < dfk::kMxStreamCount : p.form < dfk::kMxStreamGated));
    }
}
"""
MAX_ROWS, MAX_OUT, MAX_IN = 1048576, 1 << 20, 131072
LDS = 160 * 1024 - 256


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("mx_plan") / "plan")
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-I", os.path.join(ROOT, "paper_2602_11808_amd", "csrc"), "-x", "c++", "-", "-o", exe],
                   input=SRC, text=True, check=True)

    def run(rows):
        text = "".join("%d %d %d %d %d %d\n" % r for r in rows)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.split("\n")
        return [tuple(map(int, l.split())) for l in out if l]
    return run


def shapes():
    rnd = random.Random(1)
    rows = [(m, n, k, x8, g, f) for m in (1, 16, 17, 32, 33, 64, 65, 300, 4096, MAX_ROWS) for n in (32, 128, 4096, 50272, 131072) for k in (32, 96, 256, 4096, MAX_IN)
            for x8, g, f in ((0, 0, 0), (1, 0, 1), (1, 1, 0), (0, 1, 0))]
    for _ in range(4000):
        g = rnd.randint(0, 1)
        n = 32 * int(2 ** rnd.uniform(0, 12)) if g else int(2 ** rnd.uniform(0, 20))
        rows.append((int(2 ** rnd.uniform(0, 20)), n, 32 * int(2 ** rnd.uniform(0, 12)), rnd.randint(0, 1), g, 0 if g else rnd.randint(0, 1)))
    return rows


def test_choices_can_be_launched(ask):
    rows = shapes()
    for (m, n, k, x8, gated, f32), (form, tile, splits, per_cu, lds, wgs, need, bound, offered) in zip(rows, ask(rows), strict=True):
        what = (m, n, k, x8, gated, f32, form, tile, splits)
        if form >= 0:
            assert m <= 64 and splits == 1 and offered and lds <= LDS, what
            continue
        exact = x8 and (m <= 64 or f32)
        assert 0 <= tile < 8 and per_cu > 0 and not (exact and tile == 4), what
        assert k % 256 == 0 or tile in (0, 2), what
        assert splits == 1 or (not gated and splits in (2, 4, 8) and k // 256 >= 2 * splits), what      # each split has steps
        assert need <= bound, what
        # threads of a launch, of at most 2^18 rows, count in 32 bits (a result of more than 2^37 elements has no room)
        assert min(wgs, wgs * 2 ** 18 // m + 1) + 8 < 2 ** 32 // 512 or m * n > 2 ** 37, what


def test_gpu_tests_run_every_kernel(ask):
    """Streams by format and number of row tiles, tiles by format, width off 256 and off 128, with and without sums multiplied apart; k splits."""
    seen = set()
    rows = [(m, n, k, int(x == FP8), int(kind == "gateup"), int(out == "fp32")) for kind, m, k, n, x, out in EVERY_KERNEL]
    for (m, n, k, x8, gated, f32), (form, tile, splits, *_) in zip(rows, ask(rows), strict=True):
        width = 0 if k % 256 == 0 else 1 if k % 128 == 0 else 2
        if form >= 0:
            seen.add(("stream", form, x8, 1 if m <= 16 else 2 if m <= 32 else 4, width == 2))
        else:
            seen.add(("tile", tile, gated, x8, int(bool(x8 and (m <= 64 or f32))), width))
            if splits > 1:
                seen.add(("splits", x8))
    rows = shapes()
    for (m, n, k, x8, gated, f32), (form, tile, splits, *_) in zip(rows, ask(rows), strict=True):
        width = 0 if k % 256 == 0 else 1 if k % 128 == 0 else 2
        if form >= 0:
            what = ("stream", form, x8, 1 if m <= 16 else 2 if m <= 32 else 4, width == 2)
        else:
            what = ("tile", tile, gated, x8, int(bool(x8 and (m <= 64 or f32))), width)
        assert what in seen, (what, (m, k, n))
    assert {("splits", 0), ("splits", 1)} <= seen
