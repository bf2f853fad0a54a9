"""dfk_add_rmsnorm is off by its fp32 roundings and no more: the sum of squares has 64 bits, however long the row and however different its elements."""
import pytest
import torch

import paper_2602_11808_amd as dfk
from tests.mx_ref import FP4, FP8, assert_mx_near
from tests.operators_ref import EPS, TINY

pytestmark = pytest.mark.gpu
BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32
# of the sum H + delta (in the element itself, and at most as much in the root of the mean of squares), of the reciprocal, of two products: half a step of fp32 each
ROUNDINGS = 5.05 * 2.0 ** -24


def rows(d, kind, g):
    x = torch.randn((4, d), generator=g, device="cuda")
    if kind == "one large":                            # its square is 2^24 times the others': a sum in 24 bits loses those beside it
        x = x.sign()
        x[:, ::257] = 4096.0
    elif kind == "rising":
        x *= torch.exp2(torch.linspace(-12.0, 12.0, d, device="cuda"))
    return x


@pytest.mark.parametrize("d", [32, 256, 512, 1024, 2048, 4096, 8192, 16384, 32768])
@pytest.mark.parametrize("dtype", [FP32, BF16, FP16])
@pytest.mark.parametrize("kind", ["normal", "one large", "rising"])
@pytest.mark.parametrize("delta", [False, True])
def test_a_row_is_off_by_five_roundings(d, dtype, kind, delta):
    g = torch.Generator(device="cuda")
    g.manual_seed(d + len(kind))
    H = rows(d, kind, g).to(dtype)
    D = (0.3 * torch.randn((4, d), generator=g, device="cuda")).to(dtype) if delta else None
    w = (1.0 + 0.3 * torch.randn(d, generator=g, device="cuda")).to(dtype)
    eps = torch.tensor(1e-6, dtype=FP32).double().item()                 # as the call takes it
    s = H.double() + (D.double() if delta else 0.0)
    n = s / torch.sqrt((s * s).mean(1, keepdim=True) + eps) * w.double()
    err = ROUNDINGS * n.abs()
    out, N = torch.empty_like(H) if delta else None, torch.empty_like(H)
    for mx in (FP4, FP8):
        q, sc = torch.empty((4, d // 2 if mx == FP4 else d), dtype=torch.uint8, device="cuda"), torch.empty((4, d // 32), dtype=torch.uint8, device="cuda")
        dfk.dfk_add_rmsnorm(H, D, w, 1e-6, out, N, q, sc)
        half = 0.0 if dtype == FP32 else 0.5001 * EPS[dtype]
        assert bool(((N.double() - n).abs() <= err + half * (n.abs() + err) + TINY[dtype]).all()), float(((N.double() - n).abs() / n.abs().clamp(min=1e-30)).max() * 2.0 ** 24)
        assert_mx_near(q, sc, mx, n, err, (d, dtype, kind, mx))
