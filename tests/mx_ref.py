"""Plain 64-bit forms of the calls on microscaled (MX) tensors, and the bounds on what rounding may do.

Quantisation of given values has one right answer, bit for bit.  Where the quantised values are computed in fp32 first (norm, gated half), an element may be
that of any value within the fp32 error of the 64-bit one: rounding is monotonic, so it lies between the elements of the two ends."""
import torch

from tests.operators_ref import EPS, TINY, linear_ref  # noqa: F401

FP4, FP8 = 0, 1
EMAX = {FP4: 2, FP8: 8}


def pow2(e):
    """2^e in 64 bits, exactly (torch.pow is off by a step for some whole exponents)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def grid(mx, device):
    """The values of codes 0, 1, ... that are not negative."""
    if mx == FP4:
        return torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=device)
    c = torch.arange(127, device=device)
    e, m = c // 8, (c % 8).double()
    return torch.where(e > 0, pow2(e - 7) * (1 + m / 8), m / 512)


def code_of(u, mx):
    """Codes (sign in the highest bit of 4 or 8) of the nearest elements, ties to the even code, larger values to the largest."""
    g = grid(mx, u.device)
    mid, a = (g[1:] + g[:-1]) / 2, u.abs().contiguous()
    lo, hi = torch.bucketize(a, mid), torch.bucketize(a, mid, right=True)
    c = torch.where(lo % 2 == 0, lo, hi)
    return c + torch.where(torch.signbit(u), 8 if mx == FP4 else 128, 0)


def exponent_of(top, mx):
    """Exponent of a block's scale from its largest magnitude."""
    e = torch.frexp(top).exponent.long() - 1 - EMAX[mx]
    return torch.where(top > 0, e, -127).clamp(-127, 127)


def quantise(X, mx):
    """(elements [rows, bytes], scales [rows, blocks]) as the format stores them."""
    rows, cols = X.shape
    b = X.double().view(rows, -1, 32)
    bad = ~torch.isfinite(b).all(2, keepdim=True)
    clean = torch.where(bad, 0.0, b)
    e = exponent_of(clean.abs().amax(2, keepdim=True), mx)
    c = torch.where(bad, 0, code_of(clean * pow2(-e), mx))
    s = torch.where(bad, 255, e + 127).to(torch.uint8).view(rows, -1)
    if mx == FP8:
        return c.to(torch.uint8).view(rows, cols), s
    c = c.view(rows, -1, 2)
    return (c[:, :, 0] + 16 * c[:, :, 1]).to(torch.uint8), s


def codes(Q, mx):
    return torch.stack([Q & 15, Q >> 4], 2).view(Q.shape[0], -1).long() if mx == FP4 else Q.long()


def values(Q, S, mx):
    """What elements and scales stand for, in 64 bits."""
    c, g, n = codes(Q, mx), grid(mx, Q.device), 8 if mx == FP4 else 128
    m = c % n
    v = torch.where(m < len(g), g[m.clamp(max=len(g) - 1)], float("nan")) * torch.where(c >= n, -1.0, 1.0)
    f = torch.where(S == 255, float("nan"), pow2(S.long() - 127))
    return v * torch.repeat_interleave(f, 32, dim=1)


def assert_mx_near(Q, S, mx, ref, err, what):
    """Elements and scales of values within `err` of `ref` (64 bits)."""
    rows = ref.shape[0]
    b, d = ref.view(rows, -1, 32), err.view(rows, -1, 32)
    top = b.abs()
    lo, hi = exponent_of((top - d).clamp(min=0).amax(2), mx), exponent_of((top + d).amax(2), mx)
    e = S.long() - 127
    assert bool(((e >= lo) & (e <= hi)).all()), (what, "scales")
    f = pow2(-e)[:, :, None]
    g, n = grid(mx, ref.device), 8 if mx == FP4 else 128
    val = lambda c: (torch.where(c >= n, -1.0, 1.0) * g[c % n]).view(rows, -1)  # noqa: E731
    below, above = val(code_of((b - d) * f, mx)), val(code_of((b + d) * f, mx))
    got = codes(Q, mx)
    assert bool((got % n < len(g)).all()), (what, "not a number")
    got = val(got)
    assert bool(((got >= below) & (got <= above)).all()), (what, "elements", int(((got < below) | (got > above)).sum()))


def random_mx(rows, cols, mx, gen, std=1.0, device="cuda"):
    """Quantised N(0, std^2) with some columns larger, and the 64-bit values they stand for."""
    x = torch.randn((rows, cols), generator=gen, device=device) * std
    x *= 1.0 + 15.0 * (torch.rand(cols, generator=gen, device=device) < 0.01)
    Q, S = quantise(x, mx)
    return Q, S, values(Q, S, mx)


def product_ref(x, w, bias, residual, act, out, inexact):
    """(result, bound); `inexact`: products of eight neighbours are added in fixed point, each cut off at 2^-13 of the largest one's binade: together no more than 2^-10 of their
    magnitudes."""
    y, bound = linear_ref(x, w, bias, residual, act, out)
    if inexact:
        bound = bound + 1.2 * 1.01 * 2.0 ** -10 * (x.abs() @ w.abs().t().contiguous())
    return y, bound


def gateup_ref(x, wg, wu, inexact):
    """(A_2, error of its fp32 value) in 64 bits."""
    gate, up = x @ wg.t().contiguous(), x @ wu.t().contiguous()
    step = x.shape[1] * 2.0 ** -23 + (2.0 ** -10 if inexact else 0.0)
    eg, eu = step * (x.abs() @ wg.abs().t().contiguous()), step * (x.abs() @ wu.abs().t().contiguous())
    silu = gate / (1.0 + torch.exp(-gate))
    a = silu * up
    return a, 1.01 * (1.2 * eg * up.abs() + silu.abs() * eu + 1.2 * eg * eu + 32 * 2.0 ** -23 * a.abs()) + 2.0 ** -149


def norm_ref(H, delta, w, eps):
    """(s, n, error of n's fp32 value): three roundings of products and one of the sum, and half of what the sum of d squares may be off."""
    s = H.double() + (delta.double() if delta is not None else 0.0)
    n = s / torch.sqrt((s * s).mean(1, keepdim=True) + eps) * w.double()
    # s, s r, (s r) w: one rounding each; r: of its square root, its division, the mean, the sum (a tree of at most 48 additions: 32 of a thread, then 10 + 16 at most over the lanes and wavefronts)
    return s, n, (3 + 3 + 32) * 2.0 ** -24 * n.abs() + 2.0 ** -149


# (kind, rows, K, columns, format of the activations, result): every kernel that the choice has, at some of the smallest shapes that reach it
EVERY_KERNEL = [
    ("gateup", 1, 32, 32, FP4, "bf16"), ("gateup", 1, 32, 32, FP8, "bf16"), ("gateup", 1, 128, 32, FP4, "bf16"), ("gateup", 1, 128, 32, FP8, "bf16"),
    ("gateup", 1, 1056, 32, FP4, "bf16"), ("gateup", 1, 1056, 32, FP8, "bf16"), ("gateup", 1, 1152, 32, FP8, "bf16"), ("gateup", 2, 1152, 32, FP4, "mx"),
    ("gateup", 17, 32, 32, FP4, "mx"), ("gateup", 17, 32, 32, FP8, "mx"), ("gateup", 17, 128, 32, FP4, "mx"), ("gateup", 17, 128, 32, FP8, "mx"),
    ("gateup", 18, 1056, 32, FP4, "mx"), ("gateup", 20, 1120, 32, FP8, "mx"), ("gateup", 20, 1152, 32, FP4, "mx"), ("gateup", 20, 1152, 32, FP8, "mx"),
    ("gateup", 33, 32, 32, FP4, "mx"), ("gateup", 33, 128, 32, FP4, "mx"), ("gateup", 33, 256, 32, FP8, "mx"), ("gateup", 33, 512, 32, FP8, "mx"),
    ("gateup", 33, 3584, 32, FP4, "mx"), ("gateup", 34, 256, 17344, FP4, "mx"), ("gateup", 34, 2048, 32, FP8, "bf16"), ("gateup", 35, 32, 32, FP8, "mx"),
    ("gateup", 35, 128, 32, FP8, "mx"), ("gateup", 35, 128, 8448, FP8, "mx"), ("gateup", 36, 256, 16512, FP8, "bf16"), ("gateup", 37, 288, 32, FP8, "bf16"),
    ("gateup", 43, 384, 32, FP8, "bf16"), ("gateup", 54, 32, 32, FP4, "mx"), ("gateup", 54, 32, 8416, FP8, "mx"), ("gateup", 60, 128, 32, FP4, "mx"),
    ("gateup", 60, 256, 32, FP4, "mx"), ("gateup", 65, 32, 32, FP8, "mx"), ("gateup", 65, 256, 32, FP8, "mx"), ("gateup", 66, 256, 8576, FP4, "mx"),
    ("gateup", 69, 128, 32, FP8, "mx"), ("gateup", 73, 128, 4320, FP4, "mx"), ("gateup", 81, 5120, 32, FP8, "mx"), ("gateup", 129, 256, 22976, FP4, "mx"),
    ("gateup", 131, 256, 2752, FP8, "bf16"), ("gateup", 142, 1536, 10976, FP4, "bf16"), ("gateup", 194, 32, 2112, FP4, "mx"), ("gateup", 518, 32, 928, FP8, "bf16"),
    ("gateup", 2510, 256, 416, FP8, "mx"), ("gateup", 2690, 256, 736, FP4, "bf16"), ("gateup", 2721, 128, 192, FP8, "bf16"), ("gateup", 2823, 256, 1440, FP8, "bf16"),
    ("gateup", 4113, 256, 256, FP4, "mx"), ("gateup", 5016, 256, 416, FP8, "mx"), ("gateup", 5472, 512, 192, FP8, "bf16"), ("linear", 1, 32, 16, FP4, "bf16"),
    ("linear", 1, 32, 16, FP8, "fp32"), ("linear", 1, 32, 5371, FP8, "bf16"), ("linear", 1, 128, 16, FP4, "bf16"), ("linear", 1, 128, 16, FP8, "bf16"),
    ("linear", 1, 128, 5489, FP8, "bf16"), ("linear", 1, 1088, 9326, FP8, "bf16"), ("linear", 1, 1152, 12849, FP4, "bf16"), ("linear", 1, 2304, 16, FP8, "bf16"),
    ("linear", 2, 128, 15695, FP4, "bf16"), ("linear", 2, 2080, 17, FP4, "bf16"), ("linear", 2, 2176, 16, FP4, "bf16"), ("linear", 3, 32, 4310, FP4, "bf16"),
    ("linear", 3, 128, 13668, FP8, "bf16"), ("linear", 3, 2080, 16, FP8, "bf16"), ("linear", 7, 128, 4287, FP4, "fp32"), ("linear", 8, 16128, 17, FP8, "fp32"),
    ("linear", 9, 1280, 8232, FP8, "fp32"), ("linear", 14, 32, 8566, FP4, "bf16"), ("linear", 15, 32, 8363, FP8, "bf16"), ("linear", 16, 1088, 8985, FP4, "bf16"),
    ("linear", 17, 128, 19, FP8, "bf16"), ("linear", 17, 1184, 10059, FP4, "bf16"), ("linear", 18, 1280, 8322, FP4, "bf16"), ("linear", 19, 32, 8846, FP8, "fp32"),
    ("linear", 19, 128, 8933, FP8, "fp32"), ("linear", 19, 1184, 4747, FP8, "bf16"), ("linear", 20, 32, 8390, FP4, "fp32"), ("linear", 20, 2528, 16, FP4, "bf16"),
    ("linear", 21, 2176, 17, FP8, "bf16"), ("linear", 22, 32, 16, FP8, "bf16"), ("linear", 22, 128, 16, FP4, "bf16"), ("linear", 22, 128, 8449, FP4, "bf16"),
    ("linear", 24, 32, 16, FP4, "bf16"), ("linear", 24, 32, 4203, FP8, "fp32"), ("linear", 24, 2080, 18, FP8, "bf16"), ("linear", 27, 32, 4097, FP4, "bf16"),
    ("linear", 28, 1408, 4749, FP8, "bf16"), ("linear", 28, 2304, 16, FP4, "fp32"), ("linear", 29, 128, 4821, FP8, "bf16"), ("linear", 32, 128, 4682, FP4, "bf16"),
    ("linear", 33, 32, 16, FP8, "bf16"), ("linear", 33, 128, 17, FP8, "bf16"), ("linear", 33, 256, 16, FP8, "bf16"), ("linear", 34, 640, 5246, FP8, "bf16"),
    ("linear", 37, 32, 4130, FP4, "bf16"), ("linear", 37, 288, 4194, FP8, "bf16"), ("linear", 37, 1280, 5874, FP8, "fp32"), ("linear", 38, 2304, 17, FP4, "bf16"),
    ("linear", 39, 32, 16, FP4, "bf16"), ("linear", 41, 1056, 6492, FP8, "fp32"), ("linear", 42, 2080, 17, FP4, "bf16"), ("linear", 45, 1536, 16, FP8, "bf16"),
    ("linear", 46, 128, 4655, FP4, "bf16"), ("linear", 46, 1632, 16, FP8, "bf16"), ("linear", 48, 128, 17, FP4, "bf16"), ("linear", 64, 1216, 6552, FP4, "bf16"),
    ("linear", 65, 256, 16, FP4, "bf16"), ("linear", 69, 32, 17, FP8, "bf16"), ("linear", 70, 512, 21, FP8, "fp32"), ("linear", 71, 2048, 17, FP4, "fp32"),
    ("linear", 77, 32, 16, FP4, "bf16"), ("linear", 81, 128, 21, FP8, "bf16"), ("linear", 81, 256, 16, FP8, "bf16"), ("linear", 91, 128, 16, FP4, "bf16"),
    ("linear", 92, 32, 16, FP8, "fp32"), ("linear", 92, 128, 20, FP8, "fp32"), ("linear", 98, 2816, 25199, FP8, "fp32"), ("linear", 608, 256, 1607, FP8, "bf16"),
    ("linear", 916, 128, 1106, FP8, "bf16"), ("linear", 1559, 768, 5154, FP4, "fp32"), ("linear", 1631, 256, 1245, FP4, "fp32"), ("linear", 1678, 128, 901, FP8, "fp32"),
    ("linear", 3653, 32, 390, FP8, "fp32"), ("linear", 3656, 256, 522, FP4, "bf16"), ("linear", 4069, 256, 960, FP4, "bf16"), ("linear", 4166, 5632, 65, FP8, "bf16"),
    ("linear", 4168, 3584, 38, FP4, "fp32"), ("linear", 4297, 32, 198, FP8, "bf16"), ("linear", 4321, 128, 229, FP4, "bf16"), ("linear", 4362, 256, 945, FP8, "fp32"),
    ("linear", 4400, 256, 2912, FP8, "bf16"), ("linear", 4848, 256, 397, FP8, "fp32"), ("linear", 5027, 256, 791, FP4, "bf16"), ("linear", 5179, 1536, 791, FP4, "bf16"),
    ("linear", 5602, 512, 329, FP8, "bf16"), ("linear", 5605, 256, 322, FP8, "bf16"), ("linear", 5630, 32, 141, FP4, "fp32"), ("linear", 5724, 256, 716, FP8, "bf16"),
]
