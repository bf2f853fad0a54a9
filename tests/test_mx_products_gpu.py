"""Linear layers and the gated half with MXFP4 weights against their 64-bit forms: sizes on both sides of every tile, types, epilogues, scales, streams, graphs."""
import pytest
import torch

import paper_2602_11808_amd as dfk
from tests.mx_ref import EVERY_KERNEL, FP4, FP8, assert_mx_near, codes, gateup_ref, product_ref, quantise, random_mx, values
from tests.operators_ref import EPS, RMS_ONE, TINY, assert_close

pytestmark = pytest.mark.gpu
BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32
GUARD = 64


def gen(*key):
    g = torch.Generator(device="cuda")
    g.manual_seed(hash(key) % (1 << 31))
    return g


def guarded(shape, dtype, offset=0):
    n = 1
    for v in shape:
        n *= v
    buf = torch.full((2 * GUARD + offset + n,), 7, dtype=dtype, device="cuda")
    return buf, buf[GUARD + offset:GUARD + offset + n].view(shape), offset


def untouched(*bufs):
    for b, t, o in bufs:
        assert bool((b[:GUARD + o] == 7).all()) and bool((b[GUARD + o + t.numel():] == 7).all()), "wrote outside"


def workspace(new, *a):
    ws = new(*a)
    ws.fill_(0xFF)                                     # nothing in it is taken for granted
    return ws


def inexact(M, x_mx, out):
    """Whether products of eight neighbours may be added in fixed point."""
    return x_mx == FP8 and M > 64 and out != FP32


def check(M, K, N, x_mx, out=BF16, dtype=None, act=0, bias=True, residual=False, offset=0, seed=0):
    g = gen(M, K, N, x_mx, seed)
    dtype = dtype or (out if out != FP32 else BF16)
    Xq, Xs, x = random_mx(M, K, x_mx, g)
    Wq, Ws, w = random_mx(N, K, FP4, g, K ** -0.5)
    b = torch.randn(N, generator=g, device="cuda").mul_(0.5).to(dtype) if bias else None
    R = torch.randn((M, N), generator=g, device="cuda").to(out) if residual else None
    Y = guarded((M, N), out, offset)
    dfk.dfk_mx_linear(Xq, Xs, Wq, Ws, b, R, Y[1], act, workspace(dfk.new_mx_linear_workspace, M, N, K))
    untouched(Y)
    ref, bound = product_ref(x, w, b, R, act, out, inexact(M, x_mx, out))
    assert_close(Y[1], ref, bound, (M, K, N, x_mx, out, act), RMS_ONE[out])


ROWS = [1, 2, 7, 8, 9, 15, 16, 17, 31, 32, 33, 48, 63, 64, 65, 96, 127, 128, 129, 200, 255, 256, 257, 300, 511, 700]


@pytest.mark.parametrize("M", ROWS)
@pytest.mark.parametrize("K,N", [(128, 64), (544, 130), (2880, 257)])
def test_rows(M, K, N):
    check(M, K, N, FP8 if (M + N) % 2 else FP4, BF16 if M % 3 else FP16, act=M % 5, residual=M % 2 == 0)


@pytest.mark.parametrize("K", [32, 64, 96, 128, 160, 224, 256, 288, 384, 480, 512, 544, 640, 768, 992, 1024, 1056, 2048, 4096, 4128, 8192, 14336])
@pytest.mark.parametrize("M", [1, 20, 40, 130, 600])
@pytest.mark.parametrize("x_mx", [FP4, FP8])
def test_lengths_of_the_sum(M, K, x_mx):
    check(M, K, 96, x_mx, out=FP32 if K % 96 == 0 else BF16)


@pytest.mark.parametrize("N", [1, 2, 3, 5, 8, 15, 16, 17, 31, 33, 60, 64, 65, 100, 127, 128, 129, 255, 256, 258, 300, 513, 1028, 5001])
@pytest.mark.parametrize("M", [1, 5, 24, 70, 513])
def test_columns(M, N):
    check(M, 320, N, FP4 if N % 3 else FP8, out=FP32 if N % 2 else BF16, act=N % 5, residual=M == 5 or M == 513)


@pytest.mark.parametrize("dtype,out", [(BF16, BF16), (BF16, FP32), (FP16, FP16), (FP16, FP32)])
@pytest.mark.parametrize("act", range(5))
@pytest.mark.parametrize("M", [3, 50, 333])
@pytest.mark.parametrize("x_mx", [FP4, FP8])
def test_types_and_activations(M, dtype, out, act, x_mx):
    check(M, 288, 200, x_mx, out, dtype, act, bias=act % 2 == 0, residual=True)
    check(M, 256, 200, x_mx, out, dtype, act, bias=True, residual=False, seed=1)


@pytest.mark.parametrize("M,K,N", [(1, 4096, 4096), (16, 4096, 14336), (64, 4096, 4096), (128, 4096, 4096), (100, 7168, 2304), (1000, 2048, 4096), (2048, 1024, 8192), (4096, 4096, 1024)])
@pytest.mark.parametrize("x_mx", [FP4, FP8])
def test_full_sizes(M, K, N, x_mx):
    check(M, K, N, x_mx, act=dfk.DFK_ACT_GELU, residual=True)


@pytest.mark.parametrize("M", [1, 40, 300])
@pytest.mark.parametrize("out", [BF16, FP32])
@pytest.mark.parametrize("offset", [1, 2, 3, 4, 8])
def test_outputs_at_any_element(M, out, offset):
    check(M, 256, 132, FP8, out, act=4, offset=offset)


def check_gateup(M, K, F, x_mx, out, seed=0):
    """out: a 16-bit type, FP4 or FP8."""
    g = gen(M, K, F, x_mx, seed)
    Xq, Xs, x = random_mx(M, K, x_mx, g)
    Gq, Gs, wg = random_mx(F, K, FP4, g, K ** -0.5)
    Uq, Us, wu = random_mx(F, K, FP4, g, K ** -0.5)
    a, err = gateup_ref(x, wg, wu, inexact(M, x_mx, out))
    ws, what = workspace(dfk.new_mx_gateup_workspace, M, F, K), (M, K, F, x_mx, out)
    if out in (FP4, FP8):
        q, s = guarded((M, F // 2 if out == FP4 else F), torch.uint8), guarded((M, F // 32), torch.uint8)
        dfk.dfk_mx_gateup(Xq, Xs, Gq, Gs, Uq, Us, None, q[1], s[1], ws)
        untouched(q, s)
        assert_mx_near(q[1], s[1], out, a, err, what)
        # and nearly all are the nearest element.  Errors are at most about 2e-5 of the largest values (fixed-point sums; fp32 ones 1e-6); of the values a binade lower than those, half as
        # many but with half the distance between elements (1/16 of the value in e4m3), as large a share changes: 2 x 2e-5 x 16 = 6e-4 a binade, of the 14 that there are, and up to twice
        # that as products are denser near zero
        away = (codes(q[1], out) != codes(quantise(a, out)[0], out)).double().mean()
        assert float(away) <= 0.02 + 1.0 / a.numel(), (what, float(away))
    else:
        y = guarded((M, F), out)
        dfk.dfk_mx_gateup(Xq, Xs, Gq, Gs, Uq, Us, y[1], None, None, ws)
        untouched(y)
        assert_close(y[1], a, err + 0.5001 * EPS[out] * (a.abs() + err) + TINY[out], what, RMS_ONE[out])


@pytest.mark.parametrize("M", ROWS)
@pytest.mark.parametrize("K,F", [(128, 64), (544, 160), (2880, 288)])
def test_gateup_rows(M, K, F):
    check_gateup(M, K, F, FP8 if (M + F // 32) % 2 else FP4, (BF16, FP16, FP4, FP8)[(M + K // 32) % 4])


@pytest.mark.parametrize("F", [32, 64, 96, 128, 160, 224, 256, 288, 544, 4864])
@pytest.mark.parametrize("M", [1, 24, 70, 300])
@pytest.mark.parametrize("out", [BF16, FP4, FP8])
def test_gateup_columns(M, F, out):
    check_gateup(M, 320, F, FP4 if F % 64 else FP8, out)


@pytest.mark.parametrize("K", [32, 96, 128, 256, 288, 512, 544, 1024, 4096, 8192])
@pytest.mark.parametrize("M", [1, 40, 130])
@pytest.mark.parametrize("x_mx", [FP4, FP8])
def test_gateup_lengths(M, K, x_mx):
    check_gateup(M, K, 96, x_mx, FP8 if K % 64 else BF16)
    check_gateup(M, K, 128, x_mx, FP4, seed=1)


@pytest.mark.parametrize("kind,M,K,N,x_mx,out", EVERY_KERNEL)
def test_every_kernel(kind, M, K, N, x_mx, out):
    """One call that reaches each form, tile and width (tests/test_mx_plan_host.py holds the list against the choice)."""
    if kind == "linear":
        check(M, K, N, x_mx, FP32 if out == "fp32" else BF16, act=M % 2, residual=N % 2 == 0)
    else:
        check_gateup(M, K, N, x_mx, BF16 if out == "bf16" else FP4 if M % 2 else FP8)


def test_rows_of_two_launches():
    """More rows than a launch takes: both parts' rows, scales, residual and results."""
    M, K, N = (1 << 18) + 300, 64, 96
    g = gen(8)
    Wq, Ws, w = random_mx(N, K, FP4, g, K ** -0.5)
    Uq, Us, wu = random_mx(N, K, FP4, g, K ** -0.5)
    for x_mx in (FP4, FP8):
        Xq = torch.randint(0, 256, (M, K // 2 if x_mx == FP4 else K), generator=g, device="cuda", dtype=torch.uint8)
        if x_mx == FP8:
            Xq &= 0xF7                                                  # (no NaN)
        Xs = torch.randint(120, 128, (M, K // 32), generator=g, device="cuda", dtype=torch.uint8)
        R = torch.randn((M, N), generator=g, device="cuda")
        Y, A = torch.empty_like(R), torch.empty((M, N), dtype=BF16, device="cuda")
        q, s = torch.empty((M, N), dtype=torch.uint8, device="cuda"), torch.empty((M, N // 32), dtype=torch.uint8, device="cuda")
        dfk.dfk_mx_linear(Xq, Xs, Wq, Ws, None, R, Y, 0, dfk.new_mx_linear_workspace(M, N, K))
        gws = dfk.new_mx_gateup_workspace(M, N, K)
        dfk.dfk_mx_gateup(Xq, Xs, Wq, Ws, Uq, Us, None, q, s, gws)
        dfk.dfk_mx_gateup(Xq, Xs, Wq, Ws, Uq, Us, A, None, None, gws)
        for rows in (slice(0, 200), slice((1 << 18) - 100, (1 << 18) + 100), slice(M - 100, M)):
            x = values(Xq[rows], Xs[rows], x_mx)
            ref, bound = product_ref(x, w, None, R[rows], 0, FP32, False)
            assert_close(Y[rows], ref, bound, (x_mx, rows), RMS_ONE[FP32])
            a, err = gateup_ref(x, w, wu, x_mx == FP8)
            assert_mx_near(q[rows], s[rows], FP8, a, err, (x_mx, rows))
            assert_close(A[rows], a, err + 0.5001 * EPS[BF16] * (a.abs() + err) + TINY[BF16], (x_mx, rows), RMS_ONE[BF16])


@pytest.mark.parametrize("M,K,F", [(1, 4096, 14336), (16, 4096, 4096), (48, 8192, 7168), (128, 4096, 4096), (1000, 2048, 4096), (4096, 4096, 1024)])
@pytest.mark.parametrize("x_mx,out", [(FP4, FP4), (FP8, FP8), (FP8, BF16)])
def test_gateup_full_sizes(M, K, F, x_mx, out):
    check_gateup(M, K, F, x_mx, out)


@pytest.mark.parametrize("M", [1, 9, 40, 70, 300])
@pytest.mark.parametrize("x_mx", [FP4, FP8])
def test_every_scale_of_a_row_and_of_a_column(M, x_mx):
    """Blocks whose scales run over many powers of two, element by element of one side: an exchanged or missed scale shows in whole."""
    g = gen(M, x_mx)
    K, N = 1312, 160
    Xq, Xs, _ = random_mx(M, K, x_mx, g)
    Wq, Ws, _ = random_mx(N, K, FP4, g)
    Xs.copy_((120 + torch.randint(0, 15, Xs.shape, generator=g, device="cuda")).to(torch.uint8))
    Ws.copy_((110 + torch.randint(0, 15, Ws.shape, generator=g, device="cuda")).to(torch.uint8))
    x, w = values(Xq, Xs, x_mx), values(Wq, Ws, FP4)
    Y = torch.empty((M, N), device="cuda")
    dfk.dfk_mx_linear(Xq, Xs, Wq, Ws, None, None, Y, 0, dfk.new_mx_linear_workspace(M, N, K))
    ref, bound = product_ref(x, w, None, None, 0, FP32, False)
    assert_close(Y, ref, bound, M)
    for blk in (0, 3, 4, 7, 8, 40):                    # one block of X alone
        one = torch.zeros_like(Xq)
        lo, hi = (16 * blk, 16 * blk + 16) if x_mx == FP4 else (32 * blk, 32 * blk + 32)
        one[:, lo:hi] = Xq[:, lo:hi]
        dfk.dfk_mx_linear(one, Xs, Wq, Ws, None, None, Y, 0, dfk.new_mx_linear_workspace(M, N, K))
        ref, bound = product_ref(values(one, Xs, x_mx), w, None, None, 0, FP32, False)
        assert_close(Y, ref, bound, (M, blk))


@pytest.mark.parametrize("M", [1, 16, 40, 70, 300])
def test_eight_bit_sums_beside_large_products(M):
    """448 x 6 and its negative beside the smallest elements: fp32 results keep what is left."""
    K, N = 256, 64
    Xq = torch.full((M, K), 0x01, dtype=torch.uint8, device="cuda")      # 2^-9
    Wq = torch.full((N, K // 2), 0x11, dtype=torch.uint8, device="cuda")  # 0.5
    Xq[:, 0], Xq[:, 1], Xq[:, 128], Xq[:, 131] = 0x7E, 0xFE, 0xFE, 0x7E  # +-448
    Wq[:, 0], Wq[:, 64], Wq[:, 65] = 0x77, 0x17, 0x71                     # 6
    Xs, Ws = torch.full((M, K // 32), 127, dtype=torch.uint8, device="cuda"), torch.full((N, K // 32), 127, dtype=torch.uint8, device="cuda")
    Y = torch.empty((M, N), device="cuda")
    dfk.dfk_mx_linear(Xq, Xs, Wq, Ws, None, None, Y, 0, dfk.new_mx_linear_workspace(M, N, K))
    ref = values(Xq, Xs, FP8) @ values(Wq, Ws, FP4).t()
    # every product is a multiple of 2^-10 and partial sums stay below 2^12 + 2^-1: 24 bits hold them but for one rounding at 2^-12 while a large one is in
    assert float((Y.double() - ref).abs().max()) <= 8 * 2.0 ** -12, float((Y.double() - ref).abs().max())


@pytest.mark.parametrize("M", [4, 40, 200, 600])
@pytest.mark.parametrize("K", [256, 288])
@pytest.mark.parametrize("x_mx", [FP4, FP8])
def test_a_bad_block_stays_in_its_row_or_column(M, K, x_mx):
    g = gen(M, K)
    Xq, Xs, _ = random_mx(M, K, x_mx, g)
    Wq, Ws, _ = random_mx(77, K, FP4, g)
    Xs[M // 2, 3] = 255
    Ws[13, K // 32 - 1] = 255
    Y = torch.empty((M, 77), dtype=BF16, device="cuda")
    dfk.dfk_mx_linear(Xq, Xs, Wq, Ws, None, None, Y, 0, dfk.new_mx_linear_workspace(M, 77, K))
    bad = Y.isnan()
    assert bad[M // 2].all() and bad[:, 13].all()
    bad[M // 2] = False
    bad[:, 13] = False
    assert not bad.any()


@pytest.mark.parametrize("M", [4, 40, 200])
def test_gateup_a_bad_column_takes_its_block(M):
    g = gen(M)
    Xq, Xs, _ = random_mx(M, 256, FP8, g)
    (Gq, Gs, _), (Uq, Us, _) = (random_mx(128, 256, FP4, g) for _ in range(2))
    Gs[40, 2] = 255
    Us[127, 7] = 255
    q, s = torch.empty((M, 64), dtype=torch.uint8, device="cuda"), torch.empty((M, 4), dtype=torch.uint8, device="cuda")
    dfk.dfk_mx_gateup(Xq, Xs, Gq, Gs, Uq, Us, None, q, s, dfk.new_mx_gateup_workspace(M, 128, 256))
    assert bool((s[:, [1, 3]] == 255).all()) and bool((s[:, [0, 2]] < 255).all())
    assert not bool(q[:, 16:32].any()) and not bool(q[:, 48:].any())


@pytest.mark.parametrize("M", [1, 40, 300])
def test_residual_in_place(M):
    g = gen(M)
    Xq, Xs, x = random_mx(M, 512, FP8, g)
    Wq, Ws, w = random_mx(384, 512, FP4, g, 512 ** -0.5)
    R = torch.randn((M, 384), generator=g, device="cuda").to(BF16)
    ref, bound = product_ref(x, w, None, R, 0, BF16, inexact(M, FP8, BF16))
    dfk.dfk_mx_linear(Xq, Xs, Wq, Ws, None, R, R, 0, dfk.new_mx_linear_workspace(M, 384, 512))
    assert_close(R, ref, bound, "in place")


@pytest.mark.parametrize("M", [1, 8, 24, 64, 70, 130, 300])
@pytest.mark.parametrize("K,N", [(992, 72), (2880, 300), (2048, 260), (4864, 64)])
@pytest.mark.parametrize("x_mx", [FP4, FP8])
def test_bases_anywhere(M, K, N, x_mx):
    """Elements and scales that start 16 to 112 bytes into a cache line."""
    g = gen(M, K, N)
    Xq, Xs, x = random_mx(M, K, x_mx, g)
    Wq, Ws, w = random_mx(N, K, FP4, g, K ** -0.5)
    ref, bound = product_ref(x, w, None, None, 4, FP32, False)

    def moved(t, n):
        b = torch.full((t.numel() + 256,), 0xFF, dtype=torch.uint8, device="cuda")
        v = b[16 * n:16 * n + t.numel()].view(t.shape)
        v.copy_(t)
        return v

    for d in ((1, 0, 2, 0), (0, 3, 0, 5), (7, 1, 5, 3)):
        Y = torch.empty((M, N), device="cuda")
        dfk.dfk_mx_linear(moved(Xq, d[0]), moved(Xs, d[1]), moved(Wq, d[2]), moved(Ws, d[3]), None, None, Y, 4, dfk.new_mx_linear_workspace(M, N, K))
        assert_close(Y, ref, bound, (M, d))


def test_a_row_does_not_depend_on_the_others():
    """Within the same kernel a row's result has the same bits wherever the row is."""
    g = gen(1)
    Xq, Xs, _ = random_mx(200, 1024, FP8, g)
    Wq, Ws, _ = random_mx(256, 1024, FP4, g)
    order = torch.randperm(200, device="cuda")
    A, B = torch.empty((200, 256), dtype=BF16, device="cuda"), torch.empty((200, 256), dtype=BF16, device="cuda")
    ws = dfk.new_mx_linear_workspace(200, 256, 1024)
    dfk.dfk_mx_linear(Xq, Xs, Wq, Ws, None, None, A, 4, ws)
    dfk.dfk_mx_linear(Xq[order].contiguous(), Xs[order].contiguous(), Wq, Ws, None, None, B, 4, ws)
    assert torch.equal(A[order], B)


@pytest.mark.parametrize("M,K,N", [(1, 2048, 128), (8, 4096, 1000), (48, 2880, 768), (128, 4096, 512), (300, 1024, 520)])
def test_same_bits_every_time_and_in_a_graph(M, K, N):
    g = gen(M)
    Xq, Xs, _ = random_mx(M, K, FP8, g)
    Wq, Ws, _ = random_mx(N, K, FP4, g, K ** -0.5)
    R = torch.randn((M, N), generator=g, device="cuda").to(BF16)
    ws = dfk.new_mx_linear_workspace(M, N, K)
    Y = torch.empty_like(R)

    def call():
        dfk.dfk_mx_linear(Xq, Xs, Wq, Ws, None, R, Y, 2, ws)

    call()
    first = Y.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(Y, first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(4):
        Y.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(Y, first)
        ws.fill_(0x55)
        call()
        torch.cuda.synchronize()
        assert torch.equal(Y, first)


def test_two_graphs_share_a_workspace():
    """Split sums of one shape where another's were, replayed in turn with eager calls between them."""
    shapes = ((300, 4096, 512), (128, 2048, 520), (1, 2048, 128))
    g = gen(3)
    ws = dfk.new_mx_linear_workspace(300, 520, 4096)
    sets = [random_mx(M, K, FP8, g)[:2] + random_mx(N, K, FP4, g, K ** -0.5)[:2] for M, K, N in shapes]
    outs = [torch.empty((M, N), dtype=BF16, device="cuda") for M, _, N in shapes]
    call = lambda s, Y: dfk.dfk_mx_linear(*s, None, None, Y, 2, ws)  # noqa: E731
    for s, Y in zip(sets, outs):
        call(s, Y)
    want = [Y.clone() for Y in outs]
    graphs = [torch.cuda.CUDAGraph() for _ in sets[:2]]
    for gr, s, Y in zip(graphs, sets, outs):
        with torch.cuda.graph(gr):
            call(s, Y)
    for i in range(4):
        for Y in outs:
            Y.fill_(float("nan"))
        graphs[i % 2].replay()
        call(sets[2], outs[2])
        graphs[1 - i % 2].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), i


def test_more_than_four_gib_of_outputs():
    M, K, N = 70000, 64, 33000
    g = gen(4)
    Xq, Xs, x = random_mx(M, K, FP8, g)
    Wq, Ws, w = random_mx(N, K, FP4, g)
    Y = torch.empty((M, N), dtype=BF16, device="cuda")
    dfk.dfk_mx_linear(Xq, Xs, Wq, Ws, None, None, Y, 0, dfk.new_mx_linear_workspace(M, N, K))
    for rows in (slice(0, 300), slice(35000, 35300), slice(M - 300, M)):
        ref, bound = product_ref(x[rows], w, None, None, 0, BF16, True)
        assert_close(Y[rows], ref, bound, rows, RMS_ONE[BF16])


def test_weights_beyond_four_gib():
    N, K = 1 << 20, 8704
    g = gen(5)
    Wq = torch.randint(0, 256, (N, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    Ws = torch.randint(118, 124, (N, K // 32), generator=g, device="cuda", dtype=torch.uint8)
    for M in (1, 30, 200):
        Xq, Xs, x = random_mx(M, K, FP4, g)
        Y = torch.empty((M, N), device="cuda")
        dfk.dfk_mx_linear(Xq, Xs, Wq, Ws, None, None, Y, 0, dfk.new_mx_linear_workspace(M, N, K))
        for cols in (slice(0, 300), slice(N // 2 - 100, N // 2 + 100), slice(N - 300, N)):
            ref, bound = product_ref(x, values(Wq[cols], Ws[cols], FP4), None, None, 0, FP32, False)
            assert_close(Y[:, cols], ref, bound, (M, cols), RMS_ONE[FP32])


@pytest.mark.parametrize("M", [1, 20, 70, 300])
@pytest.mark.parametrize("x_mx", [FP4, FP8])
def test_longest_rows(M, x_mx):
    check(M, 131072, 200, x_mx, FP32, act=0)


@pytest.mark.parametrize("M", [1, 8, 40, 100, 300])
@pytest.mark.parametrize("mx", [FP4, FP8])
def test_the_sub_block_as_it_is_used(M, mx):
    """Norm, gated half and down projection onto the residual stream, two layers, eager and in a graph, each against the 64-bit form of its own inputs."""
    d, ff = 896, 2304
    g = gen(M, mx)
    H = torch.randn((M, d), generator=g, device="cuda").to(BF16)
    w = (1.0 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(BF16)
    layers = [[random_mx(ff, d, FP4, g, d ** -0.5), random_mx(ff, d, FP4, g, d ** -0.5), random_mx(d, ff, FP4, g, ff ** -0.5)] for _ in range(2)]
    width = lambda n: n // 2 if mx == FP4 else n  # noqa: E731
    byte = lambda *s: torch.empty(s, dtype=torch.uint8, device="cuda")  # noqa: E731
    nq, ns, aq, as_ = byte(M, width(d)), byte(M, d // 32), byte(M, width(ff)), byte(M, ff // 32)
    gws, lws = dfk.new_mx_gateup_workspace(M, ff, d), dfk.new_mx_linear_workspace(M, d, ff)
    X, D = H.clone(), torch.empty_like(H)

    def layer(i, checked=False):
        (Gq, Gs, wg), (Uq, Us, wu), (Dq, Ds, wd) = layers[i]
        before, last = X.clone() if checked else None, D.clone() if checked else None
        if i == 0:
            dfk.dfk_add_rmsnorm(X, None, w, 1e-5, None, None, nq, ns)
        else:
            dfk.dfk_add_rmsnorm(X, D, w, 1e-5, X, None, nq, ns)        # the addition of the layer before
        dfk.dfk_mx_gateup(nq, ns, Gq, Gs, Uq, Us, None, aq, as_, gws)
        dfk.dfk_mx_linear(aq, as_, Dq, Ds, None, X if i == 1 else None, X if i == 1 else D, 0, lws)
        if checked:
            from tests.mx_ref import norm_ref
            s, n, err = norm_ref(before, last if i else None, w, 1e-5)
            assert_mx_near(nq, ns, mx, n, err, "norm")
            x = values(nq, ns, mx)
            a, err = gateup_ref(x, wg, wu, inexact(M, mx, mx))
            assert_mx_near(aq, as_, mx, a, err, "gated half")
            res = s.to(BF16) if i else None
            ref, bound = product_ref(values(aq, as_, mx), wd, None, res, 0, BF16, inexact(M, mx, BF16))
            assert_close(X if i else D, ref, bound, "down")

    layer(0, True)
    layer(1, True)
    want = X.clone()
    graph = torch.cuda.CUDAGraph()
    X.copy_(H)
    with torch.cuda.graph(graph):
        layer(0)
        layer(1)
    for _ in range(3):
        X.copy_(H)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(X, want)


def test_python_refuses_what_does_not_fit():
    g = gen(1)
    X, W = random_mx(4, 64, FP8, g)[:2], random_mx(32, 64, FP4, g)[:2]
    Y, ws = torch.empty((4, 32), dtype=BF16, device="cuda"), dfk.new_mx_linear_workspace(4, 32, 64)
    b = torch.zeros(32, dtype=BF16, device="cuda")
    for bad in (lambda: dfk.dfk_mx_linear(X[0][:3], X[1], *W, None, None, Y, 0, ws), lambda: dfk.dfk_mx_linear(*X, *X, None, None, torch.empty((4, 4), dtype=BF16, device="cuda"), 0, ws),
                lambda: dfk.dfk_mx_linear(*X, W[0][:, :16], W[1], None, None, Y, 0, ws), lambda: dfk.dfk_mx_linear(*X, *W, b[:8], None, Y, 0, ws),
                lambda: dfk.dfk_mx_linear(*X, *W, b, Y[:2], Y, 0, ws), lambda: dfk.dfk_mx_gateup(*X, *W, *W, Y, X[0], X[1], ws), lambda: dfk.dfk_mx_gateup(*X, *W, *W, Y[:, :16], None, None, ws),
                lambda: dfk.dfk_mx_gateup(*X, *W, *W, None, X[0], None, ws), lambda: dfk.dfk_mx_linear(X[0].cpu(), X[1], *W, None, None, Y, 0, ws)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        dfk.dfk_mx_linear(*X, *W, b, Y.float(), Y, 0, ws)
    with pytest.raises(dfk.DfkError):
        dfk.dfk_mx_linear(*X, *W, b.to(FP16), None, Y, 0, ws)
    with pytest.raises(dfk.DfkError):
        dfk.dfk_mx_gateup(*X, *W, *W, None, None, None, ws)
    with pytest.raises(dfk.DfkError):
        dfk.dfk_mx_linear(*X, *W, b, None, Y, 0, ws[:256 - 1] if ws.numel() == 256 else ws[:255])


@pytest.mark.parametrize("N", [65540, 65552])
def test_weights_past_4_gib(N):
    """Rows of 64 KB, so that the distance from a tile's first row to the last one passes 2^32 bytes: the first columns, those past 4 GiB, the last ones."""
    M, K = 1, 131072
    g = gen(10, N)
    Xq, Xs, x = random_mx(M, K, FP4, g)
    Wq = torch.randint(0, 256, (N, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    Ws = torch.randint(112, 119, (N, K // 32), generator=g, device="cuda", dtype=torch.uint8)
    Y = torch.zeros((M, N), device="cuda")
    dfk.dfk_mx_linear(Xq, Xs, Wq, Ws, None, None, Y, 0, workspace(dfk.new_mx_linear_workspace, M, N, K))
    for rows in (slice(0, 48), slice(32752, 32800), slice(N - 48, N)):
        ref, bound = product_ref(x, values(Wq[rows], Ws[rows], FP4), None, None, 0, FP32, False)
        assert_close(Y[:, rows], ref, bound, (N, rows), RMS_ONE[FP32])


@pytest.mark.parametrize("M", [1, 100])
@pytest.mark.parametrize("x_mx", [FP4, FP8])
def test_gate_far_below_zero_beside_a_very_large_up_value(M, x_mx):
    """SiLU(gate) is zero there, or small, and so is its product with up, although gate times up is beyond fp32's range.  A block of columns for each pair; the gate's sum and the up value are exact."""
    K, code = 64, {0.5: 1, 4.0: 6, 6.0: 7}
    # gate as (elements, scale's exponent), up as a power of two: -84 * e^-84 = -2.8e-35 beside 2^120 = 1.3e36 is -37
    pairs = [((6.0, 4.0, 0.5), 3, 120), ((6.0,), 60, 125), ((6.0,), 5, 126), ((6.0, 4.0), 2, 60)]
    F = 32 * len(pairs)
    X = torch.zeros((M, K), dtype=BF16, device="cuda")
    X[:, :3] = 1.0
    Xq, Xs = torch.empty((M, K // 2 if x_mx == FP4 else K), dtype=torch.uint8, device="cuda"), torch.empty((M, K // 32), dtype=torch.uint8, device="cuda")
    dfk.dfk_mx_quantize(X, Xq, Xs)
    g, u = (torch.zeros((F, K), dtype=torch.uint8) for _ in range(2))
    gs, us = (torch.full((F, K // 32), 127, dtype=torch.uint8) for _ in range(2))
    want = torch.zeros(F, dtype=torch.float64)
    for j, (elements, exponent, up) in enumerate(pairs):
        rows = slice(32 * j, 32 * j + 32)
        for k, v in enumerate(elements):
            g[rows, k] = 8 | code[v]
        u[rows, 0] = 2                                                  # 1.0
        gs[rows, 0], us[rows, 0] = 127 + exponent, 127 + up
        gate = torch.tensor(-sum(elements) * 2.0 ** exponent, dtype=torch.float64)
        want[rows] = gate / (1.0 + torch.exp(-gate)) * 2.0 ** up
    pack = lambda t: (t[:, 0::2] | (t[:, 1::2] << 4)).cuda()            # noqa: E731
    gw, uw = (pack(g), gs.cuda()), (pack(u), us.cuda())
    ws = dfk.new_mx_gateup_workspace(M, F, K)
    A = torch.empty((M, F), dtype=BF16, device="cuda")
    dfk.dfk_mx_gateup(Xq, Xs, *gw, *uw, A, None, None, ws)
    want = want.cuda().expand(M, F).contiguous()
    # fp32 results: an exponential of an argument of 84, off by half a step of 2^-18 in the product with log2 e (6e-6 of the value), is the largest error; then a rounding to bf16
    err = 2e-5 * want.abs() + 2.0 ** -100
    assert bool(((A.double() - want).abs() <= err + 0.5001 * EPS[BF16] * (want.abs() + err)).all())
    q, s = torch.empty((M, F), dtype=torch.uint8, device="cuda"), torch.empty((M, F // 32), dtype=torch.uint8, device="cuda")
    dfk.dfk_mx_gateup(Xq, Xs, *gw, *uw, None, q, s, ws)
    assert_mx_near(q, s, FP8, want, err, (M, x_mx))
