"""GELU of dfk_linear element by element, relative to its value: far below zero it is small but no less exact."""
import math

import pytest
import torch

import paper_2602_11808_amd as dfk
from tests.operators_ref import EPS, TINY

pytestmark = pytest.mark.gpu
BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32


def results(M, n_in, dtype, out):
    """(sums, results): row m, column n has the sum s_m w_n of one product, exact in fp32, with w from -12.5 to 12.5 and s 1 or 1/2."""
    n_out = 515
    X, W = torch.zeros((M, n_in), device="cuda", dtype=dtype), torch.zeros((n_out, n_in), device="cuda", dtype=dtype)
    X[:, n_in // 2] = 1.0
    X[::3, n_in // 2] = 0.5
    W[:, n_in // 2] = torch.linspace(-12.5, 12.5, n_out, device="cuda").to(dtype)
    Y = torch.empty((M, n_out), device="cuda", dtype=out)
    dfk.dfk_linear(X, W, None, None, Y, dfk.DFK_ACT_GELU, dfk.new_linear_workspace(M, n_out, n_in, dtype))
    return X[:, n_in // 2].double()[:, None] * W[:, n_in // 2].double()[None], Y.double()


def gelu(v):
    return 0.5 * v * torch.special.erfc(-v / math.sqrt(2.0))


@pytest.mark.parametrize("M,n_in", [(2, 8), (20, 512), (100, 8), (100, 4096)])
@pytest.mark.parametrize("dtype", [BF16, FP16, FP32])
def test_fp32_results(M, n_in, dtype):
    """The exponent -v^2 / 2 log2(e) has three roundings, which exp2 multiplies by itself, and the fit's part that grows with v^2 is a quarter of a 2^-24: below 2 of 2^-24 (1 + v^2); exp2, the
    reciprocal, eight steps of a polynomial and three products are below 18 steps of 2^-23."""
    v, y = results(M, n_in, dtype, FP32)
    ref = gelu(v)
    bound = (18 * 2.0 ** -23 + 2 * 2.0 ** -24 * (1.0 + v * v)) * ref.abs() + TINY[FP32]
    assert float(((y - ref).abs() - bound).max()) <= 0.0, float(((y - ref).abs() / ref.abs()).nan_to_num(0.0).max())


@pytest.mark.parametrize("M,n_in", [(2, 8), (20, 512), (100, 8), (100, 4096)])
@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_16_bit_results(M, n_in, dtype):
    """Half a step of the type beside what is done in fp32 before: the exponent's three roundings and the fit's part that grows with v^2 (0.75 of 2^-20 v^2 together), the rest of the fit,
    exp2, the reciprocal, six steps of a polynomial and three products (0.8 of 2^-20)."""
    v, y = results(M, n_in, dtype, dtype)
    ref = gelu(v)
    before = 2.0 ** -20 * (1.0 + v * v) * ref.abs()
    bound = before + 0.5 * EPS[dtype] * (ref.abs() + before) + TINY[dtype]
    assert float(((y - ref).abs() - bound).max()) <= 0.0, float(((y - ref).abs() / ref.abs()).nan_to_num(0.0).max())
