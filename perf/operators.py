"""What the framework's further decode and prefill operators are measured on, as a serving program calls them: the
linear layers around the MLP, the choice of experts, and the experts' SwiGLU MLPs.

Every case is one call through the public entry points.  The fp32 test mode is left out, it exists to check the other types.

Fields of a case:
    op      "linear"  Y = act(X W^T + bias) + residual
            "route"   scores of all experts -> indexes and weights of the top_k of each token
            "moe"     Y = residual + sum over a token's experts of weight * SwiGLU MLP of that expert
    m       tokens of the call;  dtype: "bf16" or "fp16" (of route's scores also "fp32")
    linear: n_in, n_out;  out: type of Y (and of the residual);  act;  bias, residual: whether there are any
    route:  experts, top_k;  groups, top_groups, group_top: experts come from the best groups;  score: "softmax" or "sigmoid";
            bias: whether there is a bias for balance;  renorm, scale: of the weights;  padded: share of tokens without experts
    moe:    experts, top_k, d, ff;  residual;  padded: share of tokens without experts
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


def _linear(m, n_in, n_out, dtype="bf16", out=None, act="none", bias=False, residual=False):
    return {"op": "linear", "m": m, "n_in": n_in, "n_out": n_out, "dtype": dtype, "out": out or dtype, "act": act, "bias": bias, "residual": residual}


def _route(m, experts, top_k, dtype="fp32", score="softmax", bias=False, groups=1, top_groups=1, group_top=1, renorm=True, scale=1.0, padded=0.0):
    return {"op": "route", "m": m, "experts": experts, "top_k": top_k, "dtype": dtype, "score": score, "bias": bias, "groups": groups,
            "top_groups": top_groups, "group_top": group_top, "renorm": renorm, "scale": scale, "padded": padded}


def _moe(m, experts, top_k, d, ff, dtype="bf16", residual=False, padded=0.0):
    return {"op": "moe", "m": m, "experts": experts, "top_k": top_k, "d": d, "ff": ff, "dtype": dtype, "residual": residual, "padded": padded}


def listed():
    cases = {
        # one token's scores for 128 experts: launches and host work are all there is
        "linear router M1": _linear(1, 2048, 128, out="fp32"),
        # attention's output projection of an 8B-shaped layer onto the residual stream, a few users
        "linear proj M8": _linear(8, 4096, 4096, residual=True),
        # first half of a plain (not gated) MLP at widths that are no multiples of 128, a ragged decode batch
        "linear gelu M48 fp16": _linear(48, 2888, 7688, "fp16", act="gelu_tanh", bias=True),
        # logits of a vocabulary of odd size, a decode batch
        "linear vocab M16": _linear(16, 4096, 50257, out="fp32"),
        # the same first half over a prefill chunk: the largest product
        "linear gelu M4096": _linear(4096, 4096, 14336, act="gelu", bias=True),
        # one token's choice: latency
        "route M1": _route(1, 128, 8),
        # a prefill chunk with a bias for balance and experts from the best 4 of 8 groups
        "route groups M4096": _route(4096, 256, 8, score="sigmoid", bias=True, groups=8, top_groups=4, group_top=2, scale=2.5),
        # a large padded batch, 16-bit scores (many ties), an expert count that is no power of two
        "route M30001 bf16": _route(30001, 60, 4, "bf16", renorm=False, padded=0.1),
        # decode of one user with many small experts
        "moe M1": _moe(1, 128, 8, 2048, 768),
        # a ragged, padded decode batch in half
        "moe M24 fp16": _moe(24, 60, 4, 2304, 1408, "fp16", padded=0.1),
        # a short prompt at widths that are no multiples of 128
        "moe M300": _moe(300, 32, 4, 2888, 1000, residual=True),
        # a prefill chunk
        "moe M4096": _moe(4096, 64, 8, 2048, 1024, residual=True),
    }
    return [dict(c, name=n) for n, c in cases.items()]


def _spread(rng, lo, hi):
    """Spread over the logarithm, both ends included."""
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _draw_any(rng):
    op = rng.choice(["linear", "route", "moe"])
    if op == "linear":
        step = rng.choice([8, 64, 128])
        dtype = rng.choice(["bf16", "bf16", "fp16"])
        return _linear(int(_spread(rng, 1, 4097)), max(step, int(_spread(rng, 256, 16385)) // step * step), int(_spread(rng, 32, 60000)), dtype,
                       rng.choice([dtype, dtype, "fp32"]), rng.choice(ACTS), rng.random() < 0.5, rng.random() < 0.4)
    if op == "route":
        groups = rng.choice([1, 1, 4, 8])
        experts = groups * int(_spread(rng, 4, 64)) if groups > 1 else int(_spread(rng, 8, 512))
        top_groups = rng.randint(1, groups)
        score = rng.choice(["softmax", "sigmoid"])
        return _route(int(_spread(rng, 1, 32769)), experts, rng.randint(1, min(16, experts // groups * top_groups)), rng.choice(["fp32", "fp32", "bf16", "fp16"]),
                      score, rng.random() < 0.5, groups, top_groups, rng.choice([1, 2]), rng.random() < 0.6, rng.choice([1.0, 2.5]), rng.choice([0.0, 0.0, 0.1]))
    step = rng.choice([8, 64, 128])
    experts = int(_spread(rng, 4, 257))
    return _moe(int(_spread(rng, 1, 4097)), experts, rng.randint(1, min(8, experts)), int(_spread(rng, 512, 4097)) // step * step,
                int(_spread(rng, 256, 4097)) // step * step, rng.choice(["bf16", "bf16", "fp16"]), rng.random() < 0.5, rng.choice([0.0, 0.0, 0.1]))


def draw(rng):
    while True:
        c = _draw_any(rng)
        w = work(c)
        held = 6 * c["experts"] * c["d"] * c["ff"] if c["op"] == "moe" else w["bytes"]
        if w["flops"] <= 4.8e11 and held <= 2.5e9:   # no more than the largest listed calls
            return c


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, shape, std, dtype):
    """N(0, std^2) rounded to the type, made in pieces (the 32-bit values of a large weight are not held whole)."""
    t = torch.empty(shape, dtype=dtype, device="cuda")
    flat = t.view(-1)
    for lo in range(0, flat.numel(), 1 << 26):
        n = min(1 << 26, flat.numel() - lo)
        flat[lo:lo + n] = torch.randn(n, generator=g, device="cuda") * std
    return t


def prepare(case, seed):
    g = _generator(seed)
    m, dt = case["m"], DTYPES[case["dtype"]]
    s = {"case": case}
    if case["op"] == "linear":
        n_in, n_out, out = case["n_in"], case["n_out"], DTYPES[case["out"]]
        s["x"] = _normal(g, (m, n_in), 1.0, dt)
        s["w"] = _normal(g, (n_out, n_in), n_in ** -0.5, dt)
        s["bias"] = _normal(g, (n_out,), 0.5, dt) if case["bias"] else None
        s["residual"] = _normal(g, (m, n_out), 1.0, out) if case["residual"] else None
        s["y"] = torch.empty((m, n_out), dtype=out, device="cuda")
        return s
    padded = torch.rand(m, generator=g, device="cuda") < case["padded"]
    if case["op"] == "route":
        logits = torch.randn((m, case["experts"]), generator=g, device="cuda") * 1.5
        logits[padded] = -math.inf
        s["logits"] = logits.to(dt)
        s["bias"] = torch.randn(case["experts"], generator=g, device="cuda") * 0.05 if case["bias"] else None
        s["experts"] = torch.empty((m, case["top_k"]), dtype=torch.int32, device="cuda")
        s["weights"] = torch.empty((m, case["top_k"]), device="cuda")
        return s
    e, k, d, ff = case["experts"], case["top_k"], case["d"], case["ff"]
    s["x"] = _normal(g, (m, d), 1.0, dt)
    # scores with some experts better liked than others; a token's weights add up to one
    scores = torch.randn((m, e), generator=g, device="cuda") + 0.3 * torch.randn(e, generator=g, device="cuda")
    top = torch.topk(scores, k, dim=1)
    s["weights"] = torch.softmax(top.values, 1)
    s["experts"] = torch.where(padded[:, None], -1, top.indices).to(torch.int32)
    s["gate"] = _normal(g, (e, ff, d), d ** -0.5, dt)
    s["up"] = _normal(g, (e, ff, d), d ** -0.5, dt)
    s["down"] = _normal(g, (e, d, ff), ff ** -0.5, dt)
    s["residual"] = _normal(g, (m, d), 1.0, dt) if case["residual"] else None
    s["y"] = torch.empty_like(s["x"])
    return s


def _act(v, name):
    if name == "relu":
        return torch.clamp_min(v, 0.0)
    if name == "gelu":
        return 0.5 * v * (1.0 + torch.erf(v * 2 ** -0.5))
    if name == "gelu_tanh":
        return 0.5 * v * (1.0 + torch.tanh((2.0 / math.pi) ** 0.5 * (v + 0.044715 * v * v * v)))
    if name == "silu":
        return v * torch.sigmoid(v)
    return v


def _plain_linear(s):
    v = s["x"].float() @ s["w"].float().t()
    if s["bias"] is not None:
        v = v + s["bias"].float()
    v = _act(v, s["case"]["act"])
    if s["residual"] is not None:
        v = v + s["residual"].float()
    return v.to(s["y"].dtype)


def _plain_route(s):
    """Scores in 64 bits: which of two near experts is better has one answer then."""
    c = s["case"]
    m, e, k = c["m"], c["experts"], c["top_k"]
    logits = s["logits"].double()
    masked = logits == -math.inf
    if c["score"] == "softmax":
        score = torch.exp(logits - torch.where(masked, -1e30, logits).max(1, keepdim=True).values)
        score = score / torch.where(masked.all(1, keepdim=True), 1.0, score.sum(1, keepdim=True))
    else:
        score = torch.sigmoid(logits)
    pick = score if s["bias"] is None else score + s["bias"].double()
    pick = torch.where(masked, -math.inf, pick)
    if c["groups"] > 1:
        by_group = pick.view(m, c["groups"], e // c["groups"])
        best = torch.sort(by_group, dim=2, descending=True).values[:, :, :c["group_top"]]
        none = best[:, :, 0] == -math.inf
        of_group = torch.where(none, -math.inf, torch.where(best == -math.inf, 0.0, best).sum(2))
        order = torch.sort(of_group, dim=1, descending=True, stable=True).indices[:, :c["top_groups"]]
        kept = torch.zeros((m, c["groups"]), dtype=torch.bool, device="cuda").scatter_(1, order, True)
        pick = torch.where(kept[:, :, None], by_group, -math.inf).view(m, e)
    top = torch.sort(pick, dim=1, descending=True, stable=True)   # equal scores: the lower index first
    index, none = top.indices[:, :k], top.values[:, :k] == -math.inf
    weight = torch.where(none, 0.0, torch.gather(score, 1, index))
    if c["renorm"]:
        total = weight.sum(1, keepdim=True)
        weight = weight / torch.where(total == 0, 1.0, total)
    return torch.where(none, -1, index).to(torch.int32), (weight * c["scale"]).float()


def _plain_moe(s):
    """The rows of every expert that has any, side by side (as many as the fullest has), through three batched products."""
    c = s["case"]
    m, k, d = c["m"], c["top_k"], c["d"]
    flat = s["experts"].flatten().long()
    order = torch.argsort(flat, stable=True)
    order = order[flat[order] >= 0]
    used, place, count = torch.unique_consecutive(flat[order], return_inverse=True, return_counts=True)
    y = torch.zeros((m * k, d), device="cuda")
    if used.numel():
        within = torch.arange(order.numel(), device="cuda") - (torch.cumsum(count, 0) - count)[place]
        x = torch.zeros((used.numel(), int(count.max()), d), device="cuda")
        x[place, within] = s["x"][order // k].float()
        gate = torch.bmm(x, s["gate"][used].float().transpose(1, 2))
        up = torch.bmm(x, s["up"][used].float().transpose(1, 2))
        out = torch.bmm(gate * torch.sigmoid(gate) * up, s["down"][used].float().transpose(1, 2))
        y[order] = out[place, within] * s["weights"].flatten()[order, None]
    y = y.view(m, k, d).sum(1)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(s["y"].dtype)


def _workspace(s):
    """The scratch that a program keeps for its calls."""
    if "ws" not in s:
        import paper_2602_11808_amd as dfk
        c = s["case"]
        if c["op"] == "linear":
            s["ws"] = dfk.new_linear_workspace(c["m"], c["n_out"], c["n_in"], s["x"].dtype)
        else:
            s["ws"] = dfk.new_moe_workspace(c["m"], c["experts"], c["top_k"], c["d"], c["ff"], s["x"].dtype)
    return s["ws"]


def _own(s):
    import paper_2602_11808_amd as dfk
    c = s["case"]
    if c["op"] == "linear":
        act = {"none": dfk.DFK_ACT_NONE, "relu": dfk.DFK_ACT_RELU, "gelu": dfk.DFK_ACT_GELU, "gelu_tanh": dfk.DFK_ACT_GELU_TANH,
               "silu": dfk.DFK_ACT_SILU}[c["act"]]
        dfk.dfk_linear(s["x"], s["w"], s["bias"], s["residual"], s["y"], act, _workspace(s))
        return s["y"]
    if c["op"] == "route":
        score = dfk.DFK_SCORE_SOFTMAX if c["score"] == "softmax" else dfk.DFK_SCORE_SIGMOID
        dfk.dfk_moe_route(s["logits"], s["bias"], s["experts"], s["weights"], score, c["groups"], c["top_groups"], c["group_top"], c["renorm"], c["scale"])
        return s["experts"], s["weights"]
    dfk.dfk_moe_mlp_wdt(s["x"], s["experts"], s["weights"], s["gate"], s["up"], s["down"], s["residual"], s["y"], _workspace(s))
    return s["y"]


def run(state):
    if own:
        return _own(state)
    return {"linear": _plain_linear, "route": _plain_route, "moe": _plain_moe}[state["case"]["op"]](state)


def work(case):
    m, size = case["m"], SIZE[case["dtype"]]
    if case["op"] == "linear":
        n_in, n_out, out = case["n_in"], case["n_out"], SIZE[case["out"]]
        return {"bytes": float(size * (m * n_in + n_out * n_in + (n_out if case["bias"] else 0)) + out * m * n_out * (2 if case["residual"] else 1)),
                "flops": float(2 * m * n_in * n_out)}
    if case["op"] == "route":
        e, k = case["experts"], case["top_k"]
        return {"bytes": float(size * m * e + 8 * m * k + (4 * e if case["bias"] else 0)), "flops": float(8 * m * e)}
    e, k, d, ff = case["experts"], case["top_k"], case["d"], case["ff"]
    rows = (1.0 - case["padded"]) * m * k
    used = e * (1.0 - (1.0 - k / e) ** ((1.0 - case["padded"]) * m))     # experts that some token takes, on the average
    return {"bytes": float(size * (3 * used * d * ff + m * d * (3 if case["residual"] else 2)) + 8 * m * k), "flops": float(6 * rows * d * ff)}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "linear":
        v = torch.empty((case["m"], case["n_out"]), dtype=torch.float64, device="cuda")
        x = s["x"].double()
        for lo in range(0, case["n_out"], 8192):
            v[:, lo:lo + 8192] = torch.matmul(x, s["w"][lo:lo + 8192].double().t().contiguous())
        if s["bias"] is not None:
            v += s["bias"].double()
        if case["act"] == "relu":
            v = torch.where(v > 0, v, 0.0)
        elif case["act"] == "gelu":
            v = v * 0.5 * torch.erfc(-v / math.sqrt(2.0))
        elif case["act"] == "gelu_tanh":
            v = v / (1.0 + torch.exp(-2.0 * math.sqrt(2.0 / math.pi) * (v + 0.044715 * v ** 3)))
        elif case["act"] == "silu":
            v = v / (1.0 + torch.exp(-v))
        return v if s["residual"] is None else v + s["residual"].double()
    if case["op"] == "route":
        e, k, groups = case["experts"], case["top_k"], case["groups"]
        a = s["logits"].double()
        open_ = a > -math.inf
        if case["score"] == "softmax":
            score = torch.nan_to_num(torch.exp(a - torch.logsumexp(a, 1, keepdim=True)), nan=0.0)
        else:
            score = 1.0 / (1.0 + torch.exp(-a))
        pick = torch.where(open_, score + (s["bias"].double() if case["bias"] else 0.0), -math.inf)
        if groups > 1:
            kept = torch.zeros_like(open_)
            best = torch.stack([torch.topk(p, min(case["group_top"], e // groups), dim=1).values for p in pick.chunk(groups, 1)], 1)
            total = torch.where(best[:, :, 0] > -math.inf, torch.where(best > -math.inf, best, 0.0).sum(2), -math.inf)
            for _ in range(case["top_groups"]):
                g = torch.argmax((total == total.max(1, keepdim=True).values).int(), 1, keepdim=True)   # the first of the largest
                kept |= torch.arange(e, device="cuda")[None, :] // (e // groups) == g
                total.scatter_(1, g, -math.inf)
            pick = torch.where(kept, pick, -math.inf)
        index, weight = [], []
        for _ in range(k):
            top = pick.max(1, keepdim=True).values
            i = torch.argmax((pick == top).int(), 1, keepdim=True)
            none = top == -math.inf
            index.append(torch.where(none, -1, i))
            weight.append(torch.where(none, 0.0, score.gather(1, i)))
            pick = pick.scatter(1, i, -math.inf)
        index, weight = torch.cat(index, 1), torch.cat(weight, 1)
        if case["renorm"]:
            weight = weight / torch.clamp_min(weight.sum(1, keepdim=True), 1e-300)
        return index.to(torch.int32), weight * case["scale"]
    y = s["residual"].double() if case["residual"] else torch.zeros_like(s["x"], dtype=torch.float64)
    for e in range(case["experts"]):
        t, k = torch.nonzero(s["experts"] == e, as_tuple=True)
        if t.numel():
            x = s["x"][t].double()
            gate, up = x @ s["gate"][e].double().t().contiguous(), x @ s["up"][e].double().t().contiguous()
            y.index_add_(0, t, (gate / (1.0 + torch.exp(-gate)) * up @ s["down"][e].double().t().contiguous()) * s["weights"][t, k].double()[:, None])
    return y
