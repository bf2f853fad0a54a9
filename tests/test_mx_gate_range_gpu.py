"""The MX gated half where SiLU(gate) is below the smallest values whose reciprocal fp32 has (gate < -87.3) and the up value brings the product back: every value that fp32 can hold counts."""
import pytest
import torch

import paper_2602_11808_amd as dfk
from tests.mx_ref import FP4, FP8, assert_mx_near
from tests.operators_ref import EPS, TINY

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
CODES = {0.5: 1, 4.0: 6, 6.0: 7}
# (gate, exponent of up): SiLU(-87.5) = -8.7e-37, beside 2^120 -1.2; the last ones as far as gate and up reach
PAIRS = [(-87.5, 120), (-88.0, 120), (-88.5, 119), (-90.0, 124), (-92.0, 60), (-100.0, 126), (-120.0, 127), (-150.0, 127), (-174.0, 127), (-86.5, 121), (-8.0, 3), (-2.0, 0)]


def parts(gate):
    """A gate as a sum of elements, all negative."""
    left, out = -gate, []
    for v in (6.0, 4.0, 0.5):
        while left >= v:
            out.append(v)
            left -= v
    assert left == 0 and len(out) <= 32
    return out


def weights(gates, ups):
    """MXFP4 weights whose products with 32 ones are exactly these values, and 2^up."""
    F = len(gates)
    g, u = (torch.zeros((F, 64), dtype=torch.uint8) for _ in range(2))
    gs, us = (torch.full((F, 2), 127, dtype=torch.uint8) for _ in range(2))
    for j in range(F):
        for k, v in enumerate(parts(gates[j])):
            g[j, k] = 8 | CODES[v]
        u[j, 0] = 2                                     # 1.0
        us[j, 0] = 127 + ups[j]
    pack = lambda t: (t[:, 0::2] | (t[:, 1::2] << 4)).cuda()            # noqa: E731
    return pack(g), gs.cuda(), pack(u), us.cuda()


@pytest.mark.parametrize("M", [1, 40, 100, 300])
@pytest.mark.parametrize("x_mx", [FP4, FP8])
@pytest.mark.parametrize("mixed", [False, True])
def test_products_of_far_gates_and_large_up_values(M, x_mx, mixed):
    """A block of columns for each pair, or the pairs in turn along the columns."""
    n = 32 * len(PAIRS)
    pairs = [PAIRS[j % len(PAIRS)] if mixed else PAIRS[j // 32] for j in range(n)]
    X = torch.zeros((M, 64), dtype=BF16, device="cuda")
    X[:, :32] = 1.0
    Xq, Xs = torch.empty((M, 32 if x_mx == FP4 else 64), dtype=torch.uint8, device="cuda"), torch.empty((M, 2), dtype=torch.uint8, device="cuda")
    dfk.dfk_mx_quantize(X, Xq, Xs)
    W = weights(*zip(*pairs))
    gate, up = (torch.tensor(v, dtype=torch.float64, device="cuda") for v in zip(*pairs))
    want = (gate / (1.0 + torch.exp(-gate)) * torch.exp2(up)).expand(M, n).contiguous()
    # fp32: three exponentials of a third (one unit of 2^-23 and a rounding each) and four products, 6.5 x 2^-23; above -87 one exponential, whose argument 16-bit results round to 2^-18
    # (6e-6 of the value)
    err = torch.where(gate < -87.0, 8 * 2.0 ** -23, 2e-5) * want.abs() + 2.0 ** -149
    ws = dfk.new_mx_gateup_workspace(M, n, 64)
    A = torch.empty((M, n), dtype=BF16, device="cuda")
    dfk.dfk_mx_gateup(Xq, Xs, *W, A, None, None, ws)
    off = (A.double() - want).abs() > err + 0.5001 * EPS[BF16] * (want.abs() + err) + TINY[BF16]
    assert not bool(off.any()), sorted({pairs[j] for j in off[0].nonzero().flatten().tolist()})
    for mx in (FP4, FP8):
        q, s = torch.empty((M, n // 2 if mx == FP4 else n), dtype=torch.uint8, device="cuda"), torch.empty((M, n // 32), dtype=torch.uint8, device="cuda")
        dfk.dfk_mx_gateup(Xq, Xs, *W, None, q, s, ws)
        assert_mx_near(q, s, mx, want, err, (M, x_mx, mx))
