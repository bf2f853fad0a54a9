"""Refusals of dfk_linear, dfk_moe_route and dfk_moe_mlp_wdt: found on the host, before anything is launched (no GPU here)."""
import pytest

import paper_2602_11808_amd as dfk
from paper_2602_11808_amd.binding import lib

A = 1 << 40      # fake, aligned addresses, far enough apart not to overlap
P = [A * (i + 1) for i in range(10)]
BIG = 1 << 40


def linear(X=P[0], W=P[1], bias=P[2], residual=P[3], Y=P[4], M=4, n_out=256, n_in=512, dtype=0, out=0, act=0, ws=P[5], n=None):
    if n is None:
        n = max(256, dfk.dfk_linear_workspace_bytes(M, n_out, n_in, 0))
    return lib().dfk_linear(X, W, bias, residual, Y, M, n_out, n_in, dtype, out, act, ws, n, None)


@pytest.mark.parametrize("change,status", [
    (dict(X=0), -1), (dict(W=0), -1), (dict(Y=0), -1), (dict(M=0), -1), (dict(M=-5), -1), (dict(n_out=0), -1), (dict(n_in=0), -1),
    (dict(dtype=3), -1), (dict(dtype=-1), -1), (dict(out=2), -1), (dict(dtype=1, out=0), -1), (dict(act=5), -1), (dict(act=-1), -1),
    (dict(n_in=12), -2), (dict(n_in=131080), -2), (dict(n_out=(1 << 20) + 1), -2), (dict(M=dfk.DFK_MAX_ROWS + 1), -2),
    (dict(X=P[0] + 8), -3), (dict(W=P[1] + 2), -3), (dict(bias=P[2] + 1), -3), (dict(residual=P[3] + 1), -3), (dict(Y=P[4] + 1), -3),
    (dict(out=1, residual=P[3] + 2), -3), (dict(out=1, Y=P[4] + 2), -3), (dict(ws=P[5] + 128), -3),
    (dict(Y=P[0]), -4), (dict(Y=P[1] + 4096), -4), (dict(Y=P[2]), -4), (dict(residual=P[4] + 2), -4), (dict(ws=P[0]), -4), (dict(ws=P[4]), -4),
    (dict(ws=P[3]), -4), (dict(ws=P[2]), -4), (dict(ws=0), -5), (dict(n=0), -5), (dict(n=255), -5),
])
def test_linear_refuses(change, status):
    assert linear(**change) == status


def test_linear_workspace():
    q = dfk.dfk_linear_workspace_bytes
    assert q(1, 1, 8) >= 256 and q(dfk.DFK_MAX_ROWS, 1 << 20, 131072) >= 256
    assert q(0, 16, 16) == q(1, 0, 16) == q(1, 16, 12) == q(1, 16, 16, 5) == q(dfk.DFK_MAX_ROWS + 1, 16, 16) == 0
    for n_out, n_in in ((128, 2048), (4096, 4096), (50257, 4096)):       # a workspace for M_max rows is one for fewer
        sizes = [q(M, n_out, n_in) for M in (1, 8, 16, 17, 32, 33, 48, 64, 65, 100, 128, 200, 256, 257, 400, 512, 700, 1024, 2048, 4096, 100000)]
        assert sizes == sorted(sizes)
    with pytest.raises(ValueError):
        dfk.new_linear_workspace(1, 16, 12, device="cpu")


def route(logits=P[0], bias=P[1], experts=P[2], weights=P[3], M=4, E=64, K=8, dtype=1, score=0, groups=1, top_groups=1, group_top=1, renorm=1, scale=1.0):
    return lib().dfk_moe_route(logits, bias, experts, weights, M, E, K, dtype, score, groups, top_groups, group_top, renorm, scale, None)


@pytest.mark.parametrize("change,status", [
    (dict(logits=0), -1), (dict(experts=0), -1), (dict(weights=0), -1), (dict(M=0), -1), (dict(E=0), -1), (dict(K=0), -1), (dict(dtype=4), -1),
    (dict(score=2), -1), (dict(score=-1), -1), (dict(groups=0), -1), (dict(top_groups=0), -1), (dict(groups=4, top_groups=5), -1),
    (dict(group_top=0), -1), (dict(group_top=3), -1), (dict(scale=float("inf")), -1), (dict(scale=float("nan")), -1),
    (dict(M=dfk.DFK_MAX_ROWS + 1), -2), (dict(E=1025), -2), (dict(E=1024, K=33), -2), (dict(E=4, K=5), -2), (dict(E=65, groups=4), -2),
    (dict(E=130, groups=65), -2), (dict(E=64, groups=8, top_groups=1, K=9), -2),
    (dict(logits=P[0] + 2), -3), (dict(bias=P[1] + 2), -3), (dict(experts=P[2] + 1), -3), (dict(weights=P[3] + 2), -3),
    (dict(experts=P[0]), -4), (dict(weights=P[0] + 64), -4), (dict(experts=P[3]), -4), (dict(experts=P[1]), -4), (dict(weights=P[1] + 4), -4),
])
def test_route_refuses(change, status):
    assert route(**change) == status


def moe(X=P[0], experts=P[1], weights=P[2], Wg=P[3], Wu=P[4], Wd=P[5], residual=P[6], Y=P[7], M=4, E=8, K=2, d=256, ff=128, dtype=0, ws=P[8], n=None):
    if n is None:
        n = max(1, dfk.dfk_moe_workspace_bytes(4, 8, 2, 256, 128))
    return lib().dfk_moe_mlp_wdt(X, experts, weights, Wg, Wu, Wd, residual, Y, M, E, K, d, ff, dtype, ws, n, None)


@pytest.mark.parametrize("change,status", [
    (dict(X=0), -1), (dict(experts=0), -1), (dict(weights=0), -1), (dict(Wg=0), -1), (dict(Wu=0), -1), (dict(Wd=0), -1), (dict(Y=0), -1),
    (dict(M=0), -1), (dict(E=0), -1), (dict(K=0), -1), (dict(d=0), -1), (dict(ff=-8), -1), (dict(dtype=3), -1),
    (dict(M=dfk.DFK_MAX_ROWS + 1), -2), (dict(E=1025), -2), (dict(K=33), -2), (dict(d=260), -2), (dict(ff=132), -2), (dict(d=32776), -2), (dict(ff=32776), -2),
    (dict(X=P[0] + 8), -3), (dict(Wg=P[3] + 8), -3), (dict(Wu=P[4] + 2), -3), (dict(Wd=P[5] + 4), -3), (dict(residual=P[6] + 8), -3), (dict(Y=P[7] + 2), -3),
    (dict(experts=P[1] + 2), -3), (dict(weights=P[2] + 1), -3), (dict(ws=P[8] + 64), -3),
    (dict(Y=P[0]), -4), (dict(Y=P[1]), -4), (dict(Y=P[2]), -4), (dict(Y=P[3] + 256), -4), (dict(Y=P[4]), -4), (dict(Y=P[5]), -4), (dict(residual=P[7] + 16), -4),
    (dict(ws=P[0]), -4), (dict(ws=P[1]), -4), (dict(ws=P[5]), -4), (dict(ws=P[6]), -4), (dict(ws=P[7]), -4),
    (dict(ws=0), -5), (dict(n=0), -5),
])
def test_moe_refuses(change, status):
    assert moe(**change) == status


def test_moe_refuses_a_workspace_one_byte_short():
    assert moe(n=dfk.dfk_moe_workspace_bytes(4, 8, 2, 256, 128) - 1) == -5


def test_moe_workspace():
    q = dfk.dfk_moe_workspace_bytes
    assert q(0, 8, 2, 256, 128) == q(1, 0, 2, 256, 128) == q(1, 8, 33, 256, 128) == q(1, 8, 2, 12, 128) == q(1, 8, 2, 256, 128, 9) == 0
    assert q(dfk.DFK_MAX_ROWS, 1024, 32, 32768, 32768, 1) > 0
    for E, K, d, ff in ((8, 2, 256, 128), (128, 8, 2048, 768), (4, 1, 4096, 14336), (64, 32, 512, 512)):
        sizes = [q(M, E, K, d, ff) for M in (1, 2, 4, 7, 16, 17, 31, 32, 33, 48, 64, 65, 100, 128, 129, 200, 257, 300, 600, 1024, 4096, 8192, 8193, 70000, 1000000)]
        assert sizes == sorted(sizes)
    with pytest.raises(ValueError):
        dfk.new_moe_workspace(1, 8, 2, 12, 128, device="cpu")
