"""Rules of the experts' tile kernel (dfk_moe_plan.h), compiled for the host: which form a call gets, and that a workgroup that looks ahead reads only what has arrived."""
import os
import subprocess

import pytest

from tests.test_moe_look_ahead_gpu import SHAPES, experts_of

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SRC = """
#include <cstdio>
#include <cstring>
#include "dfk_moe_plan.h"
using namespace dfk;
int main() {
    char what[16];
    while (scanf("%15s", what) == 1) {
        int a[5];
        if (!strcmp(what, "form")) {           // M, E, K, d, ff -> row tile, most tiles, then of the gated and of the down product: form, workgroups
            for (int& v : a) scanf("%d", &v);
            const int rows = experts_tile_rows(a[0], a[1], a[2], a[3], a[4]), most = experts_max_tiles(a[0] * a[2], a[1], rows);
            const int g = experts_form(rows, most, a[4], a[3], true), d = experts_form(rows, most, a[3], a[4], false);
            printf("%d %d %d %u %d %u\\n", rows, most, g, experts_grid(kExpertsForms[g], most, a[4], true), d, experts_grid(kExpertsForms[d], most, a[3], false));
        } else if (!strcmp(what, "forms")) {
            for (const ExpertsForm& f : kExpertsForms) printf("%d %d %d %d %d %d %d ", f.bm, f.bn, f.ns, f.per_cu, f.lines, experts_newer_steps(f.ns, f.lines), experts_look_steps(f.ns));
            printf("\\n");
        } else {                               // steps, ns -> the part of each step
            scanf("%d %d", a, a + 1);
            for (int s = 0; s < a[0]; ++s) printf("%d ", experts_look_part(s, a[0], a[1]));
            printf("\\n");
        }
    }
}
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("moe_plan") / "plan")
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Wno-unused-result", "-I", os.path.join(ROOT, "paper_2602_11808_amd", "csrc"), "-x", "c++", "-", "-o", exe],
                   input=SRC, text=True, check=True)

    def run(lines):
        out = subprocess.run([exe], input="\n".join(lines) + "\n", capture_output=True, text=True, check=True).stdout.split("\n")
        return [tuple(map(int, l.split())) for l in out if l]
    return run


def forms(ask):
    v = ask(["forms"])[0]
    return [dict(zip(("bm", "bn", "ns", "per_cu", "lines", "newer", "look_steps"), v[i:i + 7])) for i in range(0, len(v), 7)]


def test_the_next_tile_is_there_when_it_is_read(ask):
    """The memory operations of the wavefront that asks for the next tile's words, in order; a wait leaves the newest ones under way and nothing else is known to have arrived."""
    for f in forms(ask):
        waves = f["bm"] * f["bn"] // 64 // 64 // 2 if (f["bm"], f["bn"]) == (64, 128) else 8
        loads = f["bm"] // 8 // waves + f["bn"] // 8 // waves
        if f["lines"]:
            continue                           # does not look ahead
        for steps in range(f["look_steps"], f["look_steps"] + 30):
            parts = ask(["part %d %d" % (steps, f["ns"])])[0]
            assert [p for p in parts if p >= 0] == [0, 1, 2, 3] and parts[steps - f["ns"]] == 3, (f, parts)
            issued = [("step", s) for s in range(f["ns"]) for _ in range(loads)]
            for s in range(steps):
                under_way = issued[len(issued) - loads * f["newer"]:] if f["newer"] else []
                assert ("step", s + 1) not in under_way, (f, s)      # what the barrier is for
                assert parts[s] != 2 or ("words",) not in under_way, (f, steps, s)
                if parts[s] == 1:
                    issued.append(("words",))
                issued += [("step", s + f["ns"])] * loads


@pytest.mark.parametrize("M,E,K,d,ff,form", SHAPES)
def test_shapes_of_the_look_ahead_tests(ask, M, E, K, d, ff, form):
    rows, most, _, _, got, grid = ask(["form %d %d %d %d %d" % (M, E, K, d, ff)])[0]
    f = forms(ask)[got]
    count = experts_of(M, E, K).flatten().bincount(minlength=E)
    tiles = int(((count + rows - 1) // rows).sum())
    assert got == form and not f["lines"] and rows == f["bm"] and tiles <= most
    assert ff // 64 >= f["look_steps"] and ff % 64 == 0
    assert tiles * -(-d // f["bn"]) > grid, "every workgroup has one tile"


def test_look_ahead_tests_meet_every_form(ask):
    assert {s[5] for s in SHAPES} == {i for i, f in enumerate(forms(ask)) if not f["lines"]}


def test_choices(ask):
    """Every choice is a form with the plan's row tile, and its workgroups are a multiple of the eight parts that the tiles are divided into."""
    fs = forms(ask)
    shapes = [(M, E, K, d, ff) for M in (65, 100, 257, 1000, 4096, 65536) for E, K in ((1, 1), (8, 2), (60, 4), (64, 8), (256, 8), (1024, 32)) for d in (8, 64, 1000, 2048, 32768)
              for ff in (8, 256, 1000, 1024, 32768)]
    for s, (rows, most, g, g_grid, d, d_grid) in zip(shapes, ask(["form %d %d %d %d %d" % s for s in shapes]), strict=True):
        for form, grid, k in ((g, g_grid, s[3]), (d, d_grid, s[4])):
            assert fs[form]["bm"] == rows and (not fs[form]["lines"] or k % 64), s
            assert grid % 8 == 0 and 8 <= grid <= 256 * fs[form]["per_cu"], s
