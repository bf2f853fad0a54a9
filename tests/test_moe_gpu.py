"""dfk_moe_mlp_wdt against its 64-bit form, and with the router and the linear layer that feed it."""
import pytest
import torch

import paper_2602_11808_amd as dfk
from tests.operators_ref import RMS_ONE, RMS_TWO, assert_close, linear_ref, moe_ref, route_ref

pytestmark = pytest.mark.gpu
BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32


def make(M, E, K, d, ff, dtype, seed=0, residual=True):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1000003 + M * 7919 + E * 31 + K + d + ff)
    rand = lambda *s, std=1.0: (torch.randn(s, generator=g, device="cuda") * std).to(dtype)  # noqa: E731
    t = {"X": rand(M, d), "Wg": rand(E, ff, d, std=d ** -0.5), "Wu": rand(E, ff, d, std=d ** -0.5), "Wd": rand(E, d, ff, std=ff ** -0.5)}
    scores = torch.randn((M, E), generator=g, device="cuda")
    top = torch.topk(scores, K, dim=1)
    t["experts"], t["weights"] = top.indices.to(torch.int32), torch.softmax(top.values, 1)
    t["R"] = rand(M, d) if residual else None
    return t


def run(t, Y=None, ws=None):
    M, d = t["X"].shape
    E, ff = t["Wg"].shape[:2]
    K = t["experts"].shape[1]
    if ws is None:
        ws = dfk.new_moe_workspace(M, E, K, d, ff, t["X"].dtype)
        ws.fill_(0xFF)
    guard = 64
    if Y is None:
        buf = torch.full((M * d + 2 * guard,), 7.0, dtype=t["X"].dtype, device="cuda")
        Y = buf[guard:-guard].view(M, d)
        dfk.dfk_moe_mlp_wdt(t["X"], t["experts"], t["weights"], t["Wg"], t["Wu"], t["Wd"], t["R"], Y, ws)
        assert (buf[:guard] == 7.0).all() and (buf[-guard:] == 7.0).all(), "wrote outside Y"
    else:
        dfk.dfk_moe_mlp_wdt(t["X"], t["experts"], t["weights"], t["Wg"], t["Wu"], t["Wd"], t["R"], Y, ws)
    return Y


def check(t, what=None):
    Y = run(t)
    ref, bound = moe_ref(t["X"], t["experts"], t["weights"], t["Wg"], t["Wu"], t["Wd"], t["R"])
    assert_close(Y, ref, bound, what, RMS_TWO[t["X"].dtype])
    return Y


@pytest.mark.parametrize("M", [1, 2, 3, 8, 15, 16, 17, 31, 32, 33, 64, 65, 100, 128, 129, 257, 600])
@pytest.mark.parametrize("E,K,d,ff", [(8, 2, 256, 128), (64, 6, 136, 264), (5, 5, 512, 72)])
def test_tokens(M, E, K, d, ff):
    check(make(M, E, K, d, ff, BF16 if M % 2 else FP16, residual=M % 3 == 0))


@pytest.mark.parametrize("d,ff", [(8, 8), (8, 128), (128, 8), (64, 64), (120, 200), (128, 1000), (1000, 128), (2304, 1408), (2888, 1000), (4096, 256), (72, 4104)])
@pytest.mark.parametrize("M", [1, 12, 40, 90, 300])
def test_widths(M, d, ff):
    check(make(M, 6, 2, d, ff, BF16 if (d + ff) % 16 else FP16))


@pytest.mark.parametrize("E,K", [(1, 1), (2, 2), (3, 1), (16, 16), (128, 8), (257, 9), (1024, 4), (40, 32)])
@pytest.mark.parametrize("M", [1, 20, 80, 400])
def test_expert_counts(M, E, K):
    check(make(M, E, K, 128, 64, BF16, residual=False))


@pytest.mark.parametrize("dtype", [BF16, FP16, FP32])
@pytest.mark.parametrize("M", [1, 30, 200])
def test_types(M, dtype):
    check(make(M, 12, 3, 264, 136, dtype))
    check(make(M, 12, 3, 264, 136, dtype, residual=False))


@pytest.mark.parametrize("M,E,K,d,ff,dtype", [(1, 128, 8, 2048, 768, BF16), (16, 64, 6, 2048, 1408, BF16), (64, 32, 4, 4096, 1024, FP16), (256, 64, 8, 2048, 1024, BF16),
                                              (1024, 16, 2, 4096, 2048, BF16), (4096, 64, 8, 1024, 512, FP16)])
def test_full_sizes(M, E, K, d, ff, dtype):
    check(make(M, E, K, d, ff, dtype))


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("M,E,K,d,ff", [(1, 16, 4, 1024, 512), (20, 16, 4, 1024, 512), (200, 16, 4, 1024, 512), (200, 16, 8, 1000, 520), (2000, 8, 4, 2048, 1024)])
def test_two_roundings(M, E, K, d, ff, dtype):
    """w * A_2 and Y are rounded to the type, each as much as Y alone, and nothing else is: sqrt(2) of that in the root mean square, and a little for the sums."""
    t = make(M, E, K, d, ff, dtype, residual=False)
    ref, _ = moe_ref(t["X"], t["experts"], t["weights"], t["Wg"], t["Wu"], t["Wd"], None)
    rms = lambda e: float((e * e).mean().sqrt())  # noqa: E731
    assert rms(run(t).double() - ref) <= 1.05 * 2 ** 0.5 * rms(ref.to(dtype).double() - ref)


@pytest.mark.parametrize("M,E,K,d,ff,dtype", [(300, 64, 2, 2048, 1160, BF16), (300, 64, 2, 2104, 72, FP16), (800, 32, 2, 4096, 1160, FP16), (800, 32, 2, 4096, 328, BF16),
                                              (1700, 8, 1, 8200, 6152, BF16), (1700, 8, 1, 8200, 264, FP16), (3000, 14, 1, 2056, 4104, BF16)])
def test_more_tiles_than_workgroups(M, E, K, d, ff, dtype):
    """A workgroup takes several tiles, and which ones differs from run to run: the results do not."""
    t = make(M, E, K, d, ff, dtype)
    t["experts"][: M // 3] %= 5                      # experts of many and of few rows, some listed twice
    ws = dfk.new_moe_workspace(M, E, K, d, ff, dtype)
    Y = check(t)
    Z = torch.empty_like(Y)
    graph = torch.cuda.CUDAGraph()
    run(t, Z, ws)
    with torch.cuda.graph(graph):
        run(t, Z, ws)
    for _ in range(4):
        Z.zero_()
        torch.cuda.synchronize()
        graph.replay()
        assert torch.equal(Y, Z)


@pytest.mark.parametrize("M", [1, 18, 150, 500])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_slots_that_take_no_part(M, dtype):
    """Padded tokens, experts elsewhere, lists with an expert twice; what is not taken is not read: NaN there shows nowhere."""
    t = make(M, 10, 4, 200, 88, dtype)
    e = t["experts"]
    e[::3] = -1
    e[1::5, 2] = 10
    e[2::4, 1] = 2 ** 31 - 1
    e[3::4, 0] = -2 ** 31
    if M > 10:
        e[4::7, 3] = e[4::7, 0]
        e[5::7] = e[5::7, :1]
        e[7::9, 1] = e[7::9, 2]
        e[e == 6] = 5
        for name in ("Wg", "Wu", "Wd"):
            t[name][6] = float("nan")
        t["X"][::3] = float("nan")
    t["weights"][(e < 0) | (e >= 10)] = float("nan")
    if M > 10:
        X = t["X"].clone()
        t["X"] = torch.nan_to_num(t["X"])
        ref, bound = moe_ref(t["X"], e, torch.nan_to_num(t["weights"]), torch.nan_to_num(t["Wg"]), torch.nan_to_num(t["Wu"]), torch.nan_to_num(t["Wd"]), t["R"])
        t["X"] = X
    else:
        ref, bound = moe_ref(t["X"], e, torch.nan_to_num(t["weights"]), t["Wg"], t["Wu"], t["Wd"], t["R"])
    assert_close(run(t), ref, bound, M)


@pytest.mark.parametrize("M", [1, 20, 100, 400])
@pytest.mark.parametrize("residual", [False, True])
def test_no_experts_at_all(M, residual):
    t = make(M, 4, 2, 128, 64, BF16, residual=residual)
    t["experts"].fill_(-1)
    Y = run(t)
    assert torch.equal(Y, t["R"] if residual else torch.zeros_like(Y))


@pytest.mark.parametrize("M", [16, 33, 64, 65, 300, 1000])
def test_one_expert_for_all(M):
    t = make(M, 16, 2, 256, 128, BF16)
    t["experts"][:, 0] = 11
    t["experts"][:, 1] = torch.arange(M, device="cuda") % 2 + 3
    check(t)


@pytest.mark.parametrize("M", [4, 40, 200])
def test_an_expert_with_infinities_reaches_its_tokens_only(M):
    t = make(M, 8, 2, 128, 64, BF16)
    t["experts"][:, 0] = torch.arange(M, device="cuda") % 4
    t["experts"][:, 1] = 4 + torch.arange(M, device="cuda") % 3
    for name in ("Wg", "Wu", "Wd"):
        t[name][2] = float("inf")
    Y = run(t)
    mine = (t["experts"] == 2).any(1)
    assert not torch.isfinite(Y[mine]).any() and torch.isfinite(Y[~mine]).all()


@pytest.mark.parametrize("M", [1, 9, 70, 300])
def test_in_place(M):
    t = make(M, 8, 2, 256, 128, BF16)
    ref, bound = moe_ref(t["X"], t["experts"], t["weights"], t["Wg"], t["Wu"], t["Wd"], t["R"])
    run(t, Y=t["R"])
    assert_close(t["R"], ref, bound, M)


@pytest.mark.parametrize("M,E,K,d,ff", [(1, 32, 4, 512, 256), (12, 16, 3, 512, 264), (60, 8, 2, 256, 256), (150, 8, 4, 512, 128), (700, 8, 2, 256, 128)])
def test_same_bits_every_time_and_in_a_graph(M, E, K, d, ff):
    t = make(M, E, K, d, ff, BF16)
    ws = dfk.new_moe_workspace(M, E, K, d, ff, BF16)
    Y = torch.empty_like(t["X"])
    run(t, Y, ws)
    first = Y.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(t, Y, ws)
    for _ in range(4):
        Y.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(Y, first)
        ws.fill_(0x7F)
        run(t, Y, ws)
        torch.cuda.synchronize()
        assert torch.equal(Y, first)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run(t, Y, ws)
    s.synchronize()
    assert torch.equal(Y, first)


def test_a_graph_follows_its_inputs():
    """Another routing in the same buffers: the launches of a captured call fit any."""
    for M in (5, 50, 200):
        a, b = make(M, 16, 4, 256, 128, BF16, seed=1), make(M, 16, 4, 256, 128, BF16, seed=2)
        ws = dfk.new_moe_workspace(M, 16, 4, 256, 128, BF16)
        Y = torch.empty_like(a["X"])
        run(a, Y, ws)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run(a, Y, ws)
        a["experts"].copy_(b["experts"])
        a["experts"][0] = 3                              # one expert four times
        a["weights"].copy_(b["weights"])
        a["X"].copy_(b["X"])
        graph.replay()
        ref, bound = moe_ref(a["X"], a["experts"], a["weights"], a["Wg"], a["Wu"], a["Wd"], a["R"])
        assert_close(Y, ref, bound, M)


def test_tokens_beyond_one_chunk():
    """More (token, expert) pairs than are gathered at a time."""
    for M, K in ((70000, 1), (9000, 8)):
        check(make(M, 8, K, 64, 32, BF16))


def test_offsets_beyond_four_gib():
    """Of X, Y and the rows that are summed (32768 columns), and of the experts' weights."""
    M, E, d, ff = 70000, 2, 32768, 8
    t = {"X": torch.randn((1000, d), device="cuda").to(BF16).repeat(M // 1000, 1), "R": None, "Wg": torch.randn((E, ff, d), device="cuda").mul_(d ** -0.5).to(BF16),
         "Wu": torch.randn((E, ff, d), device="cuda").mul_(d ** -0.5).to(BF16), "Wd": torch.randn((E, d, ff), device="cuda").to(BF16),
         "experts": torch.randint(0, E, (M, 1), device="cuda", dtype=torch.int32), "weights": torch.rand((M, 1), device="cuda")}
    Y = run(t)
    for rows in (slice(0, 40), slice(65500, 65600), slice(M - 40, M)):
        ref, bound = moe_ref(t["X"][rows], t["experts"][rows], t["weights"][rows], t["Wg"], t["Wu"], t["Wd"], None)
        assert_close(Y[rows], ref, bound, rows, RMS_TWO[BF16])
    del t, Y
    E, d, ff = 40, 8192, 8192
    W = [torch.empty((E, 8192, 8192), dtype=BF16, device="cuda") for _ in range(3)]
    for w in W:
        for e in range(E):
            w[e] = torch.randn((8192, 8192), device="cuda").mul_(8192 ** -0.5)
    for M in (2, 70):
        t = {"X": torch.randn((M, d), device="cuda").to(BF16), "R": None, "Wg": W[0], "Wu": W[1], "Wd": W[2], "weights": torch.rand((M, 2), device="cuda"),
             "experts": torch.tensor([[39, 2], [33, 39]], dtype=torch.int32, device="cuda").repeat(M // 2, 1)}
        check(t, M)


@pytest.mark.parametrize("M", [1, 7, 14, 60, 200, 900])
@pytest.mark.parametrize("d,ff", [(1000, 264), (264, 1000), (512, 328)])
def test_bases_anywhere(M, d, ff):
    """Inputs that start 16 to 112 bytes into a cache line, each elsewhere."""
    t = make(M, 9, 2, d, ff, BF16)
    for shift in (1, 4):
        u = dict(t)
        for i, name in enumerate(("X", "Wg", "Wu", "Wd")):
            n, at = t[name].numel(), 8 * ((shift * (i + 1)) % 8)
            u[name] = torch.empty(n + 64, dtype=BF16, device="cuda")[at:at + n].view(t[name].shape)
            u[name].copy_(t[name])
        check(u, (M, shift))


@pytest.mark.parametrize("M", [2, 40, 130])
@pytest.mark.parametrize("d,ff", [(32768, 72), (72, 32768)])
def test_largest_widths(M, d, ff):
    check(make(M, 3, 2, d, ff, BF16))


def test_two_graphs_share_a_workspace():
    """Replayed in turn, with eager calls of a third shape between them."""
    ts = [make(M, E, 2, d, 256, BF16, seed=M) for M, E, d in ((3, 16, 512), (300, 16, 512), (40, 4, 1024))]
    ws = dfk.new_moe_workspace(300, 16, 2, 1024, 256, BF16)
    outs = [torch.empty_like(t["X"]) for t in ts]
    want = [run(t).clone() for t in ts]
    graphs = [torch.cuda.CUDAGraph() for _ in ts[:2]]
    for g, t, Y in zip(graphs, ts, outs):
        with torch.cuda.graph(g):
            run(t, Y, ws)
    for i in range(4):
        for Y in outs:
            Y.fill_(float("nan"))
        graphs[i % 2].replay()
        run(ts[2], outs[2], ws)
        graphs[1 - i % 2].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), i


def test_two_calls_at_once():
    ts = [make(M, 16, 4, 512, 256, BF16, seed=M) for M in (6, 300)]
    want = [run(t).clone() for t in ts]
    streams = [torch.cuda.Stream() for _ in ts]
    wss = [dfk.new_moe_workspace(t["X"].shape[0], 16, 4, 512, 256, BF16) for t in ts]
    outs = [torch.empty_like(t["X"]) for t in ts]
    torch.cuda.synchronize()
    for _ in range(5):
        for t, s, ws, Y in zip(ts, streams, wss, outs):
            with torch.cuda.stream(s):
                run(t, Y, ws)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))


@pytest.mark.parametrize("M", [1, 24, 200])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_router_and_experts_together(M, score):
    """A layer's MLP as a mixture of experts on the residual stream: logits, choice, experts, as a program calls them."""
    E, K, d, ff = 32, 4, 512, 256
    t = make(M, E, K, d, ff, BF16)
    g = torch.Generator(device="cuda")
    g.manual_seed(M)
    Wr = (torch.randn((E, d), generator=g, device="cuda") * d ** -0.5).to(BF16)
    bias = torch.randn(E, generator=g, device="cuda") * 0.05
    logits = torch.empty((M, E), device="cuda")
    sig = score == "sigmoid"
    dfk.dfk_linear(t["X"], Wr, None, None, logits, dfk.DFK_ACT_NONE, dfk.new_linear_workspace(M, E, d, BF16))
    dfk.dfk_moe_route(logits, bias if sig else None, t["experts"], t["weights"], dfk.DFK_SCORE_SIGMOID if sig else dfk.DFK_SCORE_SOFTMAX,
                      8 if sig else 1, 4 if sig else 1, 2 if sig else 1, True, 2.5 if sig else 1.0)
    H = t["R"].clone()
    dfk.dfk_moe_mlp_wdt(t["X"], t["experts"], t["weights"], t["Wg"], t["Wu"], t["Wd"], H, H, dfk.new_moe_workspace(M, E, K, d, ff, BF16))
    ref, bound = linear_ref(t["X"], Wr, None, None, 0, FP32)
    assert_close(logits, ref, bound, "logits", RMS_ONE[FP32])
    idx, wts, _ = route_ref(logits, bias if sig else None, K, sig, 8 if sig else 1, 4 if sig else 1, 2 if sig else 1, True, 2.5 if sig else 1.0)
    assert torch.equal(t["experts"].cpu().long(), idx)
    ref, bound = moe_ref(t["X"], idx.cuda().int(), wts.cuda().float(), t["Wg"], t["Wu"], t["Wd"], t["R"])
    assert_close(H, ref, bound + 1e-5 * ref.abs(), "layer", RMS_TWO[BF16])
