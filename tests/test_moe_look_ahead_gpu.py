"""dfk_moe_mlp_wdt where a workgroup of the down product takes several tiles and looks ahead for the next one: every form of the kernel that does
(test_moe_plan_host.py checks that these shapes are such calls)."""
import pytest
import torch

import paper_2602_11808_amd as dfk
from tests.operators_ref import RMS_TWO, assert_close, moe_ref
from tests.test_moe_gpu import BF16, FP16, make, run

pytestmark = pytest.mark.gpu

# M, E, K, d, ff, form of the down product (index into kExpertsForms)
SHAPES = [(200, 64, 8, 2048, 384, 0), (150, 64, 8, 2304, 448, 0), (2056, 8, 1, 2048, 512, 2), (2056, 8, 1, 2048, 1024, 2), (2171, 8, 2, 832, 832, 2), (1028, 8, 2, 4096, 384, 3),
          (1028, 8, 2, 4096, 512, 3), (4100, 8, 2, 2048, 1408, 4)]


def experts_of(M, E, K):
    """Slots dealt out in turn: every expert has as many rows, give or take one."""
    return torch.arange(M * K, dtype=torch.int32).remainder(E).view(M, K)


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("M,E,K,d,ff,form", SHAPES)
def test_next_tiles(M, E, K, d, ff, form, dtype):
    t = make(M, E, K, d, ff, dtype)
    t["experts"] = experts_of(M, E, K).cuda()
    refs = []
    for uneven in (False, True):
        if uneven:
            t["experts"][: M // 4] = t["experts"][: M // 4].remainder(max(2, K))      # experts of many and of few rows
        Y = run(t)
        ref, bound = moe_ref(t["X"], t["experts"], t["weights"], t["Wg"], t["Wu"], t["Wd"], t["R"])
        assert_close(Y, ref, bound, (form, uneven), RMS_TWO[dtype])
        refs.append((t["experts"].clone(), Y))
    ws, Z = dfk.new_moe_workspace(M, E, K, d, ff, dtype), torch.empty_like(t["X"])
    run(t, Z, ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(t, Z, ws)
    for i in range(6):                       # in turn: what the last replay left in LDS is another call's
        experts, want = refs[i % 2]
        t["experts"].copy_(experts)
        Z.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(Z, want), i
        run(t, Z, ws)
        torch.cuda.synchronize()
        assert torch.equal(Z, want), i
