"""dfk_linear against its 64-bit form: sizes on both sides of every tile, types, epilogues, in place, unaligned outputs, streams, graphs."""
import pytest
import torch

import paper_2602_11808_amd as dfk
from tests.operators_ref import RMS_ONE, assert_close, linear_ref

pytestmark = pytest.mark.gpu
BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32


def make(M, n_in, n_out, dtype, seed=0, bias=True, residual=None):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1000003 + M * 7919 + n_in * 31 + n_out)
    rand = lambda *s, std=1.0, dt=dtype: (torch.randn(s, generator=g, device="cuda") * std).to(dt)  # noqa: E731
    X, W = rand(M, n_in), rand(n_out, n_in, std=n_in ** -0.5)
    return X, W, rand(n_out, std=0.5) if bias else None, rand(M, n_out, dt=residual) if residual is not None else None


def run(X, W, b, R, out, act, offset=0):
    """The call into a buffer with guard values before and behind Y (`offset` elements of misalignment)."""
    M, n_out = X.shape[0], W.shape[0]
    guard = 64
    buf = torch.full((2 * guard + offset + M * n_out,), 7.0, dtype=out, device="cuda")
    Y = buf[guard + offset:guard + offset + M * n_out].view(M, n_out)
    ws = dfk.new_linear_workspace(M, n_out, X.shape[1], X.dtype)
    ws.fill_(0xFF)                                     # nothing in it is taken for granted
    dfk.dfk_linear(X, W, b, R, Y, act, ws)
    assert (buf[:guard + offset] == 7.0).all() and (buf[guard + offset + M * n_out:] == 7.0).all(), "wrote outside Y"
    return Y


def check(M, n_in, n_out, dtype, out=None, act=0, bias=True, residual=False, seed=0, offset=0):
    out = out or dtype
    X, W, b, R = make(M, n_in, n_out, dtype, seed, bias, out if residual else None)
    Y = run(X, W, b, R, out, act, offset)
    ref, bound = linear_ref(X, W, b, R, act, out)
    assert_close(Y, ref, bound, (M, n_in, n_out, dtype, out, act), RMS_ONE[out])


@pytest.mark.parametrize("M", [1, 2, 7, 15, 16, 17, 31, 32, 33, 48, 63, 64, 65, 96, 127, 128, 129, 200, 255, 256, 257, 300, 511, 700])
@pytest.mark.parametrize("n_in,n_out", [(128, 64), (520, 130), (2888, 257)])
def test_rows(M, n_in, n_out):
    check(M, n_in, n_out, BF16 if (M + n_out) % 3 else FP16, act=M % 5, residual=M % 2 == 0)


@pytest.mark.parametrize("n_in", [8, 16, 24, 56, 64, 72, 120, 128, 136, 192, 256, 264, 504, 512, 1000, 1024, 1032, 4096, 4104, 8192])
@pytest.mark.parametrize("M", [1, 20, 40, 130, 600])
def test_lengths_of_the_sum(M, n_in):
    check(M, n_in, 96, BF16 if n_in % 16 else FP16, out=FP32 if n_in % 3 == 0 else None)


@pytest.mark.parametrize("n_out", [1, 2, 3, 5, 8, 15, 16, 17, 31, 33, 60, 64, 65, 100, 127, 128, 129, 255, 256, 258, 300, 513, 1028, 5001])
@pytest.mark.parametrize("M", [1, 5, 24, 70, 513])
def test_columns(M, n_out):
    check(M, 320, n_out, BF16, out=FP32 if n_out % 2 else BF16, act=n_out % 5, residual=M == 5 or M == 513)


@pytest.mark.parametrize("dtype,out", [(BF16, BF16), (BF16, FP32), (FP16, FP16), (FP16, FP32), (FP32, FP32)])
@pytest.mark.parametrize("act", range(5))
@pytest.mark.parametrize("M", [3, 50, 333])
def test_types_and_activations(M, dtype, out, act):
    check(M, 264, 200, dtype, out, act, bias=act % 2 == 0, residual=True)
    check(M, 264, 200, dtype, out, act, bias=True, residual=False, seed=1)


@pytest.mark.parametrize("M,n_in,n_out", [(1, 4096, 4096), (16, 4096, 14336), (64, 4096, 4096), (128, 4096, 4096), (100, 7168, 2304), (1000, 2048, 4096),
                                          (2048, 1024, 8192), (4096, 4096, 1024)])
@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_full_sizes(M, n_in, n_out, dtype):
    check(M, n_in, n_out, dtype, act=dfk.DFK_ACT_GELU, residual=True)


@pytest.mark.parametrize("M", [1, 40, 300])
@pytest.mark.parametrize("out", [BF16, FP32])
@pytest.mark.parametrize("offset", [1, 2, 3, 4, 8])
def test_outputs_at_any_element(M, out, offset):
    check(M, 256, 132, BF16, out, act=4, offset=offset)


@pytest.mark.parametrize("M", [1, 17, 65, 400])
def test_residual_in_place(M):
    X, W, b, R = make(M, 512, 384, BF16, residual=BF16)
    ref, bound = linear_ref(X, W, b, R, 0, BF16)
    ws = dfk.new_linear_workspace(M, 384, 512, BF16)
    dfk.dfk_linear(X, W, b, R, R, 0, ws)
    assert_close(R, ref, bound, "in place")


@pytest.mark.parametrize("M", [4, 40, 200, 600])
def test_a_bad_row_or_column_stays_alone(M):
    """NaN and infinities in one row of X or of W reach that row or column only: rows that fill up a tile are not summed."""
    X, W, _, _ = make(M, 200, 77, BF16, bias=False)
    X[M // 2, 5] = float("nan")
    W[13, 199] = float("inf")
    Y = run(X, W, None, None, BF16, 0)
    bad = ~torch.isfinite(Y)
    assert bad[M // 2].all() and bad[:, 13].all()
    bad[M // 2] = False
    bad[:, 13] = False
    assert not bad.any()


@pytest.mark.parametrize("act", range(5))
def test_activations_far_out(act):
    """Sums of +-1e4, +-80 and 0: no overflow inside an activation shows."""
    X = torch.tensor([[1.0] + [0.0] * 7, [100.0] + [0.0] * 7], device="cuda")
    W = torch.zeros((64, 8), device="cuda")
    W[:, 0] = torch.linspace(-100.0, 100.0, 64, device="cuda")
    W[7, 0] = 0.0
    for dtype in (BF16, FP32):
        x, w = X.to(dtype), W.to(dtype)
        Y = run(x, w, None, None, FP32, act)
        ref, bound = linear_ref(x, w, None, None, act, FP32)
        # exp in fp32 is off by 2^-24 of its argument: up to 240 of it matters where the result is still above 2^-149
        bound = bound + 1e-5 * ref.abs() + 1e-36
        assert_close(Y, ref, bound, act)


@pytest.mark.parametrize("M,n_in,n_out", [(1, 2048, 128), (8, 4096, 1000), (48, 2888, 768), (128, 4096, 512), (300, 1024, 520)])
def test_same_bits_every_time_and_in_a_graph(M, n_in, n_out):
    X, W, b, R = make(M, n_in, n_out, BF16, residual=BF16)
    ws = dfk.new_linear_workspace(M, n_out, n_in, BF16)
    Y = torch.empty_like(R)
    dfk.dfk_linear(X, W, b, R, Y, 2, ws)
    first = Y.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        dfk.dfk_linear(X, W, b, R, Y, 2, ws)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(Y, first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dfk.dfk_linear(X, W, b, R, Y, 2, ws)
    for _ in range(4):
        Y.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(Y, first)
        ws.fill_(0x55)
        dfk.dfk_linear(X, W, b, R, Y, 2, ws)
        torch.cuda.synchronize()
        assert torch.equal(Y, first)


def test_a_row_does_not_depend_on_the_others():
    """Within the same kernel a row's result has the same bits wherever the row is."""
    X, W, b, _ = make(200, 1024, 256, BF16)
    order = torch.randperm(200, device="cuda")
    A = run(X, W, b, None, BF16, 4)
    B = run(X[order].contiguous(), W, b, None, BF16, 4)
    assert torch.equal(A[order], B)


def test_more_than_four_gib_of_outputs():
    M, n_out = 70000, 33000
    X, W, _, _ = make(M, 64, n_out, BF16, bias=False)
    Y = torch.empty((M, n_out), dtype=BF16, device="cuda")
    dfk.dfk_linear(X, W, None, None, Y, 0, dfk.new_linear_workspace(M, n_out, 64, BF16))
    for rows in (slice(0, 300), slice(35000, 35300), slice(M - 300, M)):
        ref, bound = linear_ref(X[rows], W, None, None, 0, BF16)
        assert_close(Y[rows], ref, bound, rows, RMS_ONE[BF16])


@pytest.mark.parametrize("M", [1, 8, 12, 16, 40, 64, 70, 130, 300])
@pytest.mark.parametrize("n_in,n_out", [(1000, 72), (2888, 300), (2048, 260), (5000, 64)])
def test_bases_anywhere(M, n_in, n_out):
    """X and W that start 16 to 112 bytes into a cache line."""
    X, W, b, _ = make(M, n_in, n_out, BF16)
    for dx, dw in ((1, 0), (0, 3), (7, 5)):
        x, w = torch.empty(M * n_in + 64, dtype=BF16, device="cuda"), torch.empty(n_out * n_in + 64, dtype=BF16, device="cuda")
        x, w = x[8 * dx:8 * dx + M * n_in].view(M, n_in), w[8 * dw:8 * dw + n_out * n_in].view(n_out, n_in)
        x.copy_(X)
        w.copy_(W)
        ref, bound = linear_ref(X, W, b, None, 4, FP32)
        assert_close(run(x, w, b, None, FP32, 4), ref, bound, (M, dx, dw))


def test_weights_beyond_four_gib():
    n_out, n_in = 1 << 20, 4096
    W = torch.empty((n_out, n_in), dtype=BF16, device="cuda")
    for i in range(0, n_out, 1 << 16):
        W[i:i + (1 << 16)] = torch.randn((1 << 16, n_in), device="cuda").mul_(n_in ** -0.5)
    for M in (1, 30, 200):
        X = torch.randn((M, n_in), device="cuda").to(BF16)
        Y = torch.empty((M, n_out), device="cuda")
        dfk.dfk_linear(X, W, None, None, Y, 0, dfk.new_linear_workspace(M, n_out, n_in, BF16))
        for cols in (slice(0, 300), slice(n_out // 2 - 100, n_out // 2 + 100), slice(n_out - 300, n_out)):
            ref, bound = linear_ref(X, W[cols], None, None, 0, FP32)
            assert_close(Y[:, cols], ref, bound, (M, cols), RMS_ONE[FP32])


@pytest.mark.parametrize("M", [1, 20, 70, 300])
def test_longest_rows(M):
    X, W, b, _ = make(M, 131072, 200, BF16)
    Y = run(X, W, b, None, FP32, 0)
    ref, bound = linear_ref(X, W, b, None, 0, FP32)
    assert_close(Y, ref, bound, M)


def test_two_graphs_share_a_workspace():
    """Split sums of one shape where another's were, replayed in turn with eager calls between them."""
    shapes = ((300, 4096, 512), (128, 2048, 520), (1, 2048, 128))
    ws = dfk.new_linear_workspace(300, 520, 4096, BF16)
    sets = [make(*s, BF16, residual=BF16) for s in shapes]
    outs = [torch.empty_like(s[3]) for s in sets]
    for s, Y in zip(sets, outs):
        dfk.dfk_linear(*s, Y, 2, ws)
    want = [Y.clone() for Y in outs]
    graphs = [torch.cuda.CUDAGraph() for _ in sets[:2]]
    for g, s, Y in zip(graphs, sets, outs):
        with torch.cuda.graph(g):
            dfk.dfk_linear(*s, Y, 2, ws)
    for i in range(4):
        for Y in outs:
            Y.fill_(float("nan"))
        graphs[i % 2].replay()
        dfk.dfk_linear(*sets[2], outs[2], 2, ws)
        graphs[1 - i % 2].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), i
