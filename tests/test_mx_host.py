"""Refusals of the calls on microscaled (MX) tensors: found on the host, before anything is launched (no GPU here)."""
import pytest

import paper_2602_11808_amd as dfk
from paper_2602_11808_amd.binding import lib

A = 1 << 40      # fake, aligned addresses, far enough apart not to overlap
P = [A * (i + 1) for i in range(12)]


def quant(X=P[0], Q=P[1], S=P[2], rows=4, cols=256, dtype=0, mx=0):
    return lib().dfk_mx_quantize(X, Q, S, rows, cols, dtype, mx, None)


def dequant(X=P[0], Q=P[1], S=P[2], rows=4, cols=256, dtype=0, mx=0):
    return lib().dfk_mx_dequantize(Q, S, X, rows, cols, mx, dtype, None)


@pytest.mark.parametrize("call", [quant, dequant])
@pytest.mark.parametrize("change,status", [
    (dict(X=0), -1), (dict(Q=0), -1), (dict(S=0), -1), (dict(rows=0), -1), (dict(cols=0), -1), (dict(cols=-32), -1), (dict(dtype=3), -1), (dict(mx=2), -1), (dict(mx=-1), -1),
    (dict(cols=8), -2), (dict(cols=272), -2), (dict(cols=131104), -2), (dict(rows=dfk.DFK_MAX_ROWS + 1), -2),
    (dict(X=P[0] + 8), -3), (dict(Q=P[1] + 4), -3), (dict(S=P[2] + 1), -3),
    (dict(Q=P[0]), -4), (dict(S=P[0] + 2032), -4), (dict(mx=1, X=P[1] + 1008), -4),
])
def test_quantise_and_back_refuse(call, change, status):
    assert call(**change) == status


def test_quantise_refuses_scales_in_elements():
    assert quant(S=P[1] + 496) == -4 and quant(mx=1, S=P[1] + 1008) == -4


def norm(H=P[0], delta=P[1], w=P[2], eps=1e-5, H_out=P[3], N=P[4], Q=P[5], S=P[6], M=4, d=256, dtype=0, mx=1):
    return lib().dfk_add_rmsnorm(H, delta, w, eps, H_out, N, Q, S, M, d, dtype, mx, None)


@pytest.mark.parametrize("change,status", [
    (dict(H=0), -1), (dict(w=0), -1), (dict(delta=0), -1), (dict(H_out=0), -1), (dict(Q=0), -1), (dict(S=0), -1), (dict(N=0, Q=0, S=0), -1),
    (dict(M=0), -1), (dict(d=0), -1), (dict(dtype=3), -1), (dict(mx=2), -1), (dict(eps=-1.0), -1), (dict(eps=float("nan")), -1), (dict(eps=float("inf")), -1),
    (dict(M=dfk.DFK_MAX_ROWS + 1), -2), (dict(d=32800), -2), (dict(d=264), -2), (dict(d=12, Q=0, S=0), -2),
    (dict(H=P[0] + 8), -3), (dict(delta=P[1] + 2), -3), (dict(w=P[2] + 8), -3), (dict(H_out=P[3] + 4), -3), (dict(N=P[4] + 8), -3), (dict(Q=P[5] + 8), -3), (dict(S=P[6] + 4), -3),
    (dict(H_out=P[0] + 16), -4), (dict(H_out=P[1] + 16), -4), (dict(H_out=P[2]), -4), (dict(N=P[0]), -4), (dict(N=P[1]), -4), (dict(N=P[2]), -4), (dict(N=P[3]), -4),
    (dict(Q=P[0]), -4), (dict(Q=P[4]), -4), (dict(S=P[3]), -4), (dict(S=P[5] + 1008), -4),
])
def test_norm_refuses(change, status):
    assert norm(**change) == status


def linear(Xq=P[0], Xs=P[1], Wq=P[2], Ws=P[3], bias=P[4], residual=P[5], Y=P[6], M=4, n_out=256, n_in=512, x_mx=1, dtype=0, out=0, act=0, ws=P[7], n=None):
    if n is None:
        n = max(256, dfk.dfk_mx_linear_workspace_bytes(M, n_out, n_in))
    return lib().dfk_mx_linear(Xq, Xs, x_mx, Wq, Ws, bias, residual, Y, M, n_out, n_in, dtype, out, act, ws, n, None)


@pytest.mark.parametrize("change,status", [
    (dict(Xq=0), -1), (dict(Xs=0), -1), (dict(Wq=0), -1), (dict(Ws=0), -1), (dict(Y=0), -1), (dict(M=0), -1), (dict(n_out=0), -1), (dict(n_in=0), -1),
    (dict(x_mx=2), -1), (dict(x_mx=-1), -1), (dict(dtype=1, out=1), -1), (dict(dtype=3), -1), (dict(out=2), -1), (dict(dtype=2, out=0), -1), (dict(act=5), -1), (dict(act=-1), -1),
    (dict(n_in=520), -2), (dict(n_in=131104), -2), (dict(n_out=(1 << 20) + 1), -2), (dict(M=dfk.DFK_MAX_ROWS + 1), -2),
    (dict(Xq=P[0] + 8), -3), (dict(Xs=P[1] + 4), -3), (dict(Wq=P[2] + 8), -3), (dict(Ws=P[3] + 8), -3), (dict(bias=P[4] + 1), -3), (dict(residual=P[5] + 1), -3), (dict(Y=P[6] + 1), -3),
    (dict(out=1, Y=P[6] + 2), -3), (dict(ws=P[7] + 128), -3),
    (dict(Y=P[0]), -4), (dict(Y=P[1]), -4), (dict(Y=P[2] + 64), -4), (dict(Y=P[3]), -4), (dict(Y=P[4]), -4), (dict(residual=P[6] + 2), -4),
    (dict(ws=P[0]), -4), (dict(ws=P[2]), -4), (dict(ws=P[3]), -4), (dict(ws=P[4]), -4), (dict(ws=P[5]), -4), (dict(ws=P[6]), -4),
    (dict(ws=0), -5), (dict(n=0), -5), (dict(n=255), -5),
])
def test_linear_refuses(change, status):
    assert linear(**change) == status


def gateup(Xq=P[0], Xs=P[1], Wgq=P[2], Wgs=P[3], Wuq=P[4], Wus=P[5], A2=0, A2q=P[6], A2s=P[7], M=4, d=512, ff=256, x_mx=1, dtype=0, out_mx=1, ws=P[8], n=None):
    if n is None:
        n = max(256, dfk.dfk_mx_gateup_workspace_bytes(M, ff, d))
    return lib().dfk_mx_gateup(Xq, Xs, x_mx, Wgq, Wgs, Wuq, Wus, A2, dtype, A2q, A2s, out_mx, M, d, ff, ws, n, None)


@pytest.mark.parametrize("change,status", [
    (dict(Xq=0), -1), (dict(Xs=0), -1), (dict(Wgq=0), -1), (dict(Wgs=0), -1), (dict(Wuq=0), -1), (dict(Wus=0), -1), (dict(A2q=0, A2s=0), -1), (dict(A2q=0), -1), (dict(A2s=0), -1),
    (dict(A2=P[9]), -1), (dict(M=0), -1), (dict(d=0), -1), (dict(ff=0), -1), (dict(x_mx=2), -1), (dict(out_mx=2), -1), (dict(A2=P[9], A2q=0, A2s=0, dtype=1), -1),
    (dict(d=520), -2), (dict(ff=264), -2), (dict(d=131104), -2), (dict(ff=131104), -2), (dict(M=dfk.DFK_MAX_ROWS + 1), -2),
    (dict(Xq=P[0] + 8), -3), (dict(Xs=P[1] + 4), -3), (dict(Wgq=P[2] + 8), -3), (dict(Wgs=P[3] + 8), -3), (dict(Wuq=P[4] + 8), -3), (dict(Wus=P[5] + 2), -3), (dict(A2q=P[6] + 8), -3),
    (dict(A2s=P[7] + 8), -3), (dict(A2=P[9] + 8, A2q=0, A2s=0), -3), (dict(ws=P[8] + 128), -3),
    (dict(A2q=P[0]), -4), (dict(A2q=P[3]), -4), (dict(A2s=P[4]), -4), (dict(A2s=P[6] + 1008), -4), (dict(A2=P[2], A2q=0, A2s=0), -4), (dict(ws=P[5]), -4), (dict(ws=P[6]), -4), (dict(ws=P[1]), -4),
    (dict(ws=0), -5), (dict(n=255), -5),
])
def test_gateup_refuses(change, status):
    assert gateup(**change) == status


@pytest.mark.parametrize("q", [dfk.dfk_mx_linear_workspace_bytes, dfk.dfk_mx_gateup_workspace_bytes])
def test_workspaces(q):
    assert q(1, 32, 32) >= 256 and q(dfk.DFK_MAX_ROWS, 131072, 131072) >= 256
    assert q(0, 32, 32) == q(1, 0, 32) == q(1, 32, 16) == q(dfk.DFK_MAX_ROWS + 1, 32, 32) == 0
    for n_out, n_in in ((128, 2048), (4096, 4096), (14336, 4096)):       # a workspace for M_max rows is one for fewer
        sizes = [q(M, n_out, n_in) for M in (1, 8, 16, 17, 32, 33, 48, 64, 65, 100, 128, 200, 256, 257, 400, 512, 700, 1024, 2048, 4096, 100000)]
        assert sizes == sorted(sizes)
    for new in (dfk.new_mx_linear_workspace, dfk.new_mx_gateup_workspace):
        with pytest.raises(ValueError):
            new(1, 32, 16, device="cpu")
