"""Plain 64-bit forms of dfk_linear, dfk_moe_route and dfk_moe_mlp_wdt, and the bounds on what rounding may do.

The inputs are the values the kernels get (exactly representable), so a result may differ from the 64-bit one by
  * its rounding to the output type: half a step, eps / 2 of the value;
  * fp32 sums of n terms: at most n steps of 2^-23 of the sum of their magnitudes (twice what rounded additions can do, for
    matrix instructions that cut off instead of rounding), and a handful of such steps for the functions applied to them;
  * where A_2 is kept in 16 bits: half a step of each A_2, carried through the down projection."""
import math

import torch

EPS = {torch.bfloat16: 2.0 ** -7, torch.float16: 2.0 ** -10, torch.float32: 2.0 ** -23}   # torch.finfo(t).eps
# smallest step of the type (results below its normal range)
TINY = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24, torch.float32: 2.0 ** -149}


def act_ref(v, act):
    if act == 1:
        return torch.where(v > 0, v, torch.zeros_like(v))
    if act == 2:
        return 0.5 * v * torch.special.erfc(-v / math.sqrt(2.0))
    if act == 3:
        return v / (1.0 + torch.exp(-2.0 * math.sqrt(2.0 / math.pi) * (v + 0.044715 * v ** 3)))
    if act == 4:
        return v / (1.0 + torch.exp(-v))
    return v


def linear_ref(X, W, bias, residual, act, out_dtype):
    """(result, bound) in 64 bits."""
    X, W = X.double(), W.double()
    v, mag = X @ W.t().contiguous(), X.abs() @ W.abs().t().contiguous()
    if bias is not None:
        v, mag = v + bias.double(), mag + bias.double().abs()
    y = act_ref(v, act)
    # every activation here has a slope below 1.2
    err = 1.2 * (X.shape[1] + 2) * 2.0 ** -23 * mag + 16 * 2.0 ** -23 * y.abs()
    if residual is not None:
        y = y + residual.double()
        err = err + 2.0 ** -23 * y.abs()
    return y, err * 1.01 + 0.5001 * EPS[out_dtype] * y.abs() + TINY[out_dtype]


def route_ref(logits, bias, top_k, sigmoid, groups=1, top_groups=1, group_top=1, renorm=True, scale=1.0):
    """(experts, weights, gap): token by token, in Python; gap: the smallest relative difference of two scores that decided
    something without being equal."""
    import numpy as np
    L = logits.double().cpu().numpy()
    B = None if bias is None else bias.double().cpu().numpy()
    M, E = L.shape
    size = E // groups
    idx, wts, gap = np.full((M, top_k), -1, np.int64), np.zeros((M, top_k)), math.inf

    def ordered(pairs):
        nonlocal gap
        pairs = sorted(pairs, key=lambda p: (-p[0], p[1]))
        for (a, _), (b, _) in zip(pairs, pairs[1:]):
            if a != b and math.isfinite(a):
                gap = min(gap, abs(a - b) / max(abs(a), abs(b)))
        return pairs

    for m in range(M):
        row = L[m].copy()
        bad = np.isnan(row) | (np.isposinf(row) & (not sigmoid))
        row[bad] = -np.inf
        if sigmoid:
            s = np.array([0.0 if v == -np.inf else (1.0 / (1.0 + math.exp(-v)) if v > -700 else 0.0) for v in row])
        else:
            t = row.max()
            e = np.array([0.0 if v == -np.inf else math.exp(v - t) for v in row])
            s = e / e.sum() if e.sum() > 0 else e
        c = s if B is None else s + B
        open_ = [e for e in range(E) if row[e] > -np.inf and c[e] > -np.inf]
        if groups > 1:
            val = []
            for g in range(groups):
                mine = sorted((c[e] for e in open_ if e // size == g), reverse=True)
                if mine:
                    val.append((sum(mine[:group_top]), g))
            kept = {g for _, g in ordered(val)[:top_groups]}
            open_ = [e for e in open_ if e // size in kept]
        got = ordered([(c[e], e) for e in open_])[:top_k]
        w = np.array([s[e] for _, e in got])
        if renorm and len(got):
            w = w / w.sum() if w.sum() > 0 else w * 0.0
        for j, (_, e) in enumerate(got):
            idx[m, j], wts[m, j] = e, scale * w[j]
        if bad.any():
            wts[m, :] = np.nan
    return torch.from_numpy(idx), torch.from_numpy(wts), gap


def moe_ref(X, experts, weights, Wg, Wu, Wd_t, residual):
    """(result, bound) in 64 bits: expert by expert."""
    dt = X.dtype
    M, d = X.shape
    E, ff = Wg.shape[0], Wg.shape[1]
    half = 0.5001 * EPS[dt]
    y = torch.zeros((M, d), dtype=torch.float64, device=X.device)
    err, mag = torch.zeros_like(y), torch.zeros_like(y)
    for e in range(E):
        hit = experts == e
        t = torch.nonzero(hit.any(1)).flatten()
        if not t.numel():
            continue
        w = torch.where(hit[t], weights[t].double(), torch.zeros((), dtype=torch.float64, device=X.device)).sum(1, keepdim=True)
        x, g, u, dn = X[t].double(), Wg[e].double(), Wu[e].double(), Wd_t[e].double()
        gate, up = x @ g.t().contiguous(), x @ u.t().contiguous()
        eg, eu = (d * 2.0 ** -23) * (x.abs() @ g.abs().t().contiguous()), (d * 2.0 ** -23) * (x.abs() @ u.abs().t().contiguous())
        silu = gate / (1.0 + torch.exp(-gate))
        a = w * silu * up
        ea = w.abs() * (1.2 * eg * up.abs() + silu.abs() * eu + 1.2 * eg * eu) + 32 * 2.0 ** -23 * a.abs()
        ea = ea + half * (a.abs() + ea) + TINY[dt]
        y.index_add_(0, t, a @ dn.t().contiguous())
        err.index_add_(0, t, ea @ dn.abs().t().contiguous())
        mag.index_add_(0, t, (a.abs() + ea) @ dn.abs().t().contiguous())
    err = err + (ff + experts.shape[1] + 2) * 2.0 ** -23 * mag
    if residual is not None:
        y = y + residual.double()
        err = err + 2.0 ** -23 * y.abs()
    return y, err * 1.01 + half * (y.abs() + err) + TINY[dt]


# Root-mean-square error over many outputs, relative: one rounding to p bits leaves 2^(1-p) / sqrt(12) / 1.4 (1.6e-3 in bf16, 2.0e-4 in half),
# two independent ones sqrt(2) of it.  1.5 times that; it holds where there are at least 256 outputs.
RMS_ONE = {torch.bfloat16: 2.5e-3, torch.float16: 3.1e-4, torch.float32: 1e-5}
RMS_TWO = {torch.bfloat16: 3.5e-3, torch.float16: 4.4e-4, torch.float32: 1e-5}


def assert_close(Y, ref, bound, what, rms=None):
    got = Y.double()
    assert torch.isfinite(got).all(), (what, "not finite")
    over = (got - ref).abs() - bound
    assert float(over.max()) <= 0.0, (what, "off by", float((got - ref).abs().max()), "over the bound by", float(over.max()))
    if rms is not None and ref.numel() >= 256:
        r = float((got - ref).norm() / ref.norm())
        assert r <= rms, (what, "rms", r, rms)
