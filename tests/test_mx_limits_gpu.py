"""The MX calls at the ends of their ranges, on two streams at once, and on matrices that two arguments share."""
import pytest
import torch

import paper_2602_11808_amd as dfk
from tests.mx_ref import FP4, FP8, assert_mx_near, gateup_ref, norm_ref, product_ref, quantise, random_mx, values
from tests.operators_ref import EPS, RMS_ONE, TINY, assert_close

pytestmark = pytest.mark.gpu
BF16, FP32 = torch.bfloat16, torch.float32


def gen(*key):
    g = torch.Generator(device="cuda")
    g.manual_seed(hash(key) % (1 << 31))
    return g


def byte(*s):
    return torch.empty(s, dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("M", [1, 20, 70, 300])
@pytest.mark.parametrize("x_mx", [FP4, FP8])
def test_gateup_with_the_longest_rows(M, x_mx):
    K, F = 131072, 64
    g = gen(M, x_mx)
    Xq, Xs, x = random_mx(M, K, x_mx, g)
    (Gq, Gs, wg), (Uq, Us, wu) = (random_mx(F, K, FP4, g, K ** -0.5) for _ in range(2))
    a, err = gateup_ref(x, wg, wu, x_mx == FP8 and M > 64)
    A, q, s = torch.empty((M, F), dtype=BF16, device="cuda"), byte(M, F), byte(M, F // 32)
    ws = dfk.new_mx_gateup_workspace(M, F, K)
    dfk.dfk_mx_gateup(Xq, Xs, Gq, Gs, Uq, Us, A, None, None, ws)
    dfk.dfk_mx_gateup(Xq, Xs, Gq, Gs, Uq, Us, None, q, s, ws)
    assert_close(A, a, err + 0.5001 * EPS[BF16] * (a.abs() + err) + TINY[BF16], (M, x_mx), RMS_ONE[BF16])
    assert_mx_near(q, s, FP8, a, err, (M, x_mx))


@pytest.mark.parametrize("M", [1, 33, 300])
@pytest.mark.parametrize("K", [32, 256])
def test_gateup_with_the_most_columns(M, K):
    F = 131072
    g = gen(M, K)
    Xq, Xs, x = random_mx(M, K, FP4, g)
    (Gq, Gs, wg), (Uq, Us, wu) = (random_mx(F, K, FP4, g, K ** -0.5) for _ in range(2))
    q, s = byte(M, F // 2), byte(M, F // 32)
    dfk.dfk_mx_gateup(Xq, Xs, Gq, Gs, Uq, Us, None, q, s, dfk.new_mx_gateup_workspace(M, F, K))
    a, err = gateup_ref(x, wg, wu, False)
    assert_mx_near(q, s, FP4, a, err, (M, K))


@pytest.mark.parametrize("x_mx", [FP4, FP8])
def test_the_most_rows(x_mx):
    """DFK_MAX_ROWS of 32 columns through every call: norm, gated half, linear layer onto the residual."""
    M, d = dfk.DFK_MAX_ROWS, 32
    g = gen(x_mx)
    H = torch.randn((M, d), generator=g, device="cuda").to(BF16)
    w = (1.0 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(BF16)
    width = d // 2 if x_mx == FP4 else d
    (Gq, Gs, wg), (Uq, Us, wu), (Dq, Ds, wd) = (random_mx(d, d, FP4, g, d ** -0.5) for _ in range(3))
    nq, ns, aq, as_, out = byte(M, width), byte(M, 1), byte(M, width), byte(M, 1), torch.empty_like(H)
    dfk.dfk_add_rmsnorm(H, None, w, 1e-5, None, None, nq, ns)
    dfk.dfk_mx_gateup(nq, ns, Gq, Gs, Uq, Us, None, aq, as_, dfk.new_mx_gateup_workspace(M, d, d))
    dfk.dfk_mx_linear(aq, as_, Dq, Ds, None, H, out, dfk.DFK_ACT_NONE, dfk.new_mx_linear_workspace(M, d, d))
    for r in (slice(0, 100), slice((1 << 18) - 50, (1 << 18) + 50), slice(3 * (1 << 18) - 50, 3 * (1 << 18) + 50), slice(M - 100, M)):
        _, n, err = norm_ref(H[r], None, w, 1e-5)
        assert_mx_near(nq[r], ns[r], x_mx, n, err, r)
        a, err = gateup_ref(values(nq[r], ns[r], x_mx), wg, wu, x_mx == FP8)
        assert_mx_near(aq[r], as_[r], x_mx, a, err, r)
        ref, bound = product_ref(values(aq[r], as_[r], x_mx), wd, None, H[r], 0, BF16, x_mx == FP8)
        assert_close(out[r], ref, bound, r)


@pytest.mark.parametrize("M", [1, 40, 300])
def test_two_calls_at_once(M):
    """The same weights on two streams, a workspace each: the bits of the calls one after the other."""
    K, N = 4096, 2048
    g = gen(M)
    Wq, Ws, _ = random_mx(N, K, FP4, g, K ** -0.5)
    X = [random_mx(M, K, FP8, g)[:2] for _ in range(2)]
    Y = [torch.empty((M, N), dtype=FP32, device="cuda") for _ in range(2)]
    q, s = [byte(M, N) for _ in range(2)], [byte(M, N // 32) for _ in range(2)]
    lws, gws = [dfk.new_mx_linear_workspace(M, N, K) for _ in range(2)], [dfk.new_mx_gateup_workspace(M, N, K) for _ in range(2)]

    def calls(i, stream=None):
        dfk.dfk_mx_linear(*X[i], Wq, Ws, None, None, Y[i], dfk.DFK_ACT_SILU, lws[i], stream=stream)
        dfk.dfk_mx_gateup(*X[i], Wq, Ws, Wq, Ws, None, q[i], s[i], gws[i], stream=stream)

    calls(0)
    calls(1)
    torch.cuda.synchronize()
    want = [t.clone() for t in (*Y, *q, *s)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for t in (*Y, *q, *s):
        t.zero_()
    torch.cuda.synchronize()
    for _ in range(5):
        for i in range(2):
            calls(i, streams[i])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((*Y, *q, *s), want))


@pytest.mark.parametrize("M", [1, 100])
def test_gate_and_up_of_one_matrix(M):
    K, F = 512, 96
    g = gen(M)
    Xq, Xs, x = random_mx(M, K, FP4, g)
    Wq, Ws, w = random_mx(F, K, FP4, g, K ** -0.5)
    A = torch.empty((M, F), dtype=BF16, device="cuda")
    dfk.dfk_mx_gateup(Xq, Xs, Wq, Ws, Wq, Ws, A, None, None, dfk.new_mx_gateup_workspace(M, F, K))
    a, err = gateup_ref(x, w, w, False)
    assert_close(A, a, err + 0.5001 * EPS[BF16] * (a.abs() + err) + TINY[BF16], M, RMS_ONE[BF16])


@pytest.mark.parametrize("mx", [FP4, FP8])
def test_quantise_the_most_rows(mx):
    X = torch.randn((dfk.DFK_MAX_ROWS, 32), generator=gen(mx), device="cuda").to(BF16)
    q, s = byte(X.shape[0], 16 if mx == FP4 else 32), byte(X.shape[0], 1)
    dfk.dfk_mx_quantize(X, q, s)
    want = quantise(X, mx)
    assert torch.equal(q, want[0]) and torch.equal(s, want[1])


@pytest.mark.parametrize("x_mx", [FP4, FP8])
@pytest.mark.parametrize("M", [1, 24, 64, 65, 300])
def test_elements_that_are_not_numbers_and_infinite_sums(x_mx, M):
    """An e4m3 NaN takes its row; sums beyond fp32 are infinite with their sign, in their own place only."""
    K, N = 288, 48
    g = gen(M, x_mx)
    Xq, Xs, _ = random_mx(M, K, x_mx, g)
    Wq, Ws, _ = random_mx(N, K, FP4, g, K ** -0.5)
    if x_mx == FP8:
        Xq[M // 2, 200] = 0x7F
    Xq[0, :16] = 0x77 if x_mx == FP4 else 0x7E                            # the largest elements at the largest scale, in row 0 ...
    Xs[0, 0] = 254
    Wq[5, :16], Ws[5, 0] = 0xFF, 200                                       # ... beside -6 in column 5
    Wq[6, :16], Ws[6, 0] = 0x77, 200
    Y = torch.empty((M, N), device="cuda")
    dfk.dfk_mx_linear(Xq, Xs, Wq, Ws, None, None, Y, 0, dfk.new_mx_linear_workspace(M, N, K))
    nan = torch.zeros((M, N), dtype=torch.bool, device="cuda")
    if x_mx == FP8:
        nan[M // 2] = True
    assert torch.equal(Y.isnan(), nan)
    if M > 1 or x_mx == FP4:
        assert float(Y[0, 5]) == -float("inf") and float(Y[0, 6]) == float("inf")
    assert bool(torch.isfinite(Y[1:][~nan[1:]]).all())
