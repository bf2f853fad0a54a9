"""The kernels of the products with MXFP4 weights: those that the library holds are those that the choice (dfk_mx_plan.h) has, and each is one that a call comes to."""
import os
import re
import subprocess

import pytest

from paper_2602_11808_amd import LIB_PATH
from tests.mx_ref import EVERY_KERNEL, FP8

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SRC = """
#include <cstdio>
#include "dfk_mx_plan.h"
using namespace dfk;
int main() {
    for (int x8 = 0; x8 < 2; ++x8) {
        for (int f = 0; f < kMxStreamCount; ++f)
            for (int tiles = 1; tiles <= 4; tiles *= 2)
                for (int words = 0; words < 2; ++words)
                    if (mx_stream_offered(f, x8, tiles, words)) printf("offered stream %d %d %d %d\\n", f, x8, tiles, words);
        for (int t = 0; t < kMxTileCount; ++t)
            for (int gated = 0; gated < 2; ++gated)
                for (int exact = 0; exact <= x8; ++exact)
                    for (int width = 0; width < 3; ++width)
                        if (mx_tile_offered(t, x8, gated, exact, width == 0)) printf("offered tile %d %d %d %d %d\\n", t, x8, gated, exact, width);
    }
    for (int gated = 0; gated < 2; ++gated)
        for (int x8 = 0; x8 < 2; ++x8)
            for (int m = 1; m <= kMxStreamRows; ++m) {
                int most = 0;
                for (int k = 32; k <= 131072; k += 32)
                    for (int f = gated ? kMxStreamGated : 0; f < (gated ? kMxStreamCount : kMxStreamGated); ++f)
                        if (mx_stream_offered(f, x8, mx_stream_tiles(m), k % 128 == 0) && mx_stream_lds(kMxStreams[f], x8, m, k) <= kMxLds) most = k;
                printf("longest %d %d %d %d\\n", gated, x8, m, most);
            }
    int m, n, k, x8, gated, f32;
    while (scanf("%d %d %d %d %d %d", &m, &n, &k, &x8, &gated, &f32) == 6) {
        const MxPlan p = mx_plan(m, n, k, x8, gated, f32);
        if (p.form >= 0) printf("chosen stream %d %d %d %d\\n", p.form, x8, mx_stream_tiles(m), (int)(k % 128 == 0));
        else printf("chosen tile %d %d %d %d %d\\n", p.tile, x8, gated, (int)(x8 && mx_exact_sums(m, f32)), k % 256 == 0 ? 0 : k % 128 == 0 ? 1 : 2);
    }
}
"""


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """(offered, chosen by the shapes that the GPU tests run): sets of (kind, indices); the longest K that the stream has LDS for, by gated, format of the activations and rows."""
    exe = str(tmp_path_factory.mktemp("mx_kernels") / "kernels")
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-I", os.path.join(ROOT, "paper_2602_11808_amd", "csrc"), "-x", "c++", "-", "-o", exe], input=SRC, text=True, check=True)
    rows = "".join(f"{m} {n} {k} {int(x == FP8)} {int(kind == 'gateup')} {int(out == 'fp32')}\n" for kind, m, k, n, x, out in EVERY_KERNEL)
    got, longest = {"offered": set(), "chosen": set()}, {}
    for line in subprocess.run([exe], input=rows, capture_output=True, text=True, check=True).stdout.splitlines():
        what, kind, *of = line.split()
        if what == "longest":
            longest[int(kind), int(of[0]), int(of[1])] = int(of[2])
        else:
            got[what].add((kind, *map(int, of)))
    return got["offered"], got["chosen"], longest


def test_every_kernel_that_is_offered_is_one_that_a_call_comes_to(kernels):
    offered, chosen, _ = kernels
    assert chosen == offered, (offered - chosen, chosen - offered)


def test_the_library_holds_no_others(kernels):
    """Counted by the launch stubs of the built library."""
    if not os.path.exists(LIB_PATH):
        pytest.skip("the library has not been built")
    offered, _, _ = kernels
    names = subprocess.run(["nm", "-C", LIB_PATH], capture_output=True, text=True, check=True).stdout
    for kind in ("stream", "tile"):
        held = set(re.findall(r"__device_stub__(k_mx_%s<[^(]*>)" % kind, names))
        assert len(held) == sum(o[0] == kind for o in offered), (kind, len(held))


@pytest.mark.parametrize("gated,x8,rows", [
    (0, 0, {1: 131072, 16: 12288, 32: 6144, 40: 4096, 64: 2048}), (0, 1, {1: 115712, 16: 7168, 24: 4096, 40: 2048, 64: 1024}),
    (1, 0, {1: 131072, 16: 12288, 32: 4096, 56: 2048, 64: 0}), (1, 1, {1: 107520, 16: 6144, 20: 4096, 32: 2048, 56: 1024, 64: 0})])
def test_how_long_rows_the_stream_takes(kernels, gated, x8, rows):
    """The activations of a call stay in LDS beside the rings and the sums: fewer rows, longer ones."""
    longest = kernels[2]
    assert {m: longest[gated, x8, m] for m in rows} == rows
    assert all(longest[gated, x8, m] >= longest[gated, x8, m + 1] for m in range(1, 64))
