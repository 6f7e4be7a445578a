"""The feed-forward half of a served decoder layer beyond its bare linears, as cases that can be timed and checked:

- fused: a linear over byte planes with bias, activation (or the product of an activated gate and an up projection) and
  residual in its epilogue;
- route: the router of a mixture of experts: logits, scores, the chosen experts of every token and their weights;
- moe: the experts of a few tokens: gate and up products, activation, down products, weighted sum;
- layer: router and experts one after the other, as a layer runs them.

`listed()` holds the cases, `draw(rng)` makes more of the same ranges, `prepare` makes what a serving program has in
hand (activations, weights, their planes, output buffers and workspaces), `run` is one pass in elementary torch
operations or, where `own` is true, through the entry points of `paper_2506_02024_amd.binding`, and `exact` the same values in
64 bits.

FP16 mode multiplies the FP16 weights.  FP8 mode multiplies their E4M3 roundings (of the weight times 256): a linear with activations
in E4M3 and a scale per token, the experts with activations in FP16.  Gate rows stand before up rows in the weights here.
"""
import math

import torch

own = False

DEVICE = "cuda:0"


def _fused(name, tokens, rows, cols, mode, gated=False, act="none", bias=False, residual=False, packed=False, codes=False):
    return dict(name=name, kind="fused", tokens=tokens, rows=rows, cols=cols, mode=mode, gated=gated, act=act, bias=bias, residual=residual,
                packed=packed, codes=codes)


def _route(name, tokens, hidden, experts, top_k, scoring="softmax", renormalize=True, bias=False, factor=1.0):
    return dict(name=name, kind="route", tokens=tokens, hidden=hidden, experts=experts, top_k=top_k, scoring=scoring,
                renormalize=renormalize, bias=bias, factor=factor)


def _moe(name, tokens, hidden, ffn, experts, top_k, mode, act="silu", residual=False, kind="moe"):
    return dict(name=name, kind=kind, tokens=tokens, hidden=hidden, ffn=ffn, experts=experts, top_k=top_k, mode=mode, act=act,
                residual=residual)


def listed():
    return [
        # one user of a small model with a ragged width, gate and up in one linear: latency alone
        _fused("fused_m1_h1040_gated", 1, 4160, 1040, "fp16", gated=True, act="silu"),
        # the usual decode batch through an 8B model's gate and up projections, codes from the norm
        _fused("fused_m16_gate_up_fp8", 16, 28672, 4096, "fp8", gated=True, act="silu", codes=True),
        # a middle batch through a linear of odd width with everything that an epilogue can hold
        _fused("fused_m40_odd_gelu", 40, 5023, 2048, "fp16", act="gelu", bias=True, residual=True),
        # prompts of odd length through a down projection that adds the residual stream
        _fused("fused_m777_down_residual", 777, 4096, 14336, "fp8", bias=True, residual=True),
        # the largest prefill batch through gate and up, planes packed
        _fused("fused_m8192_gate_up", 8192, 28672, 4096, "fp16", gated=True, act="silu", packed=True),
        # one user in front of many small experts
        _route("route_m1_e128", 1, 2048, 128, 8),
        # a prefill batch, sigmoid scores with a bias that balances the load
        _route("route_m4000_e256", 4000, 4096, 256, 8, "sigmoid", True, True, 2.5),
        # one user of a small model: latency alone
        _moe("moe_m1_h1040_e8", 1, 1040, 528, 8, 2, "fp16"),
        # one user, many small experts
        _moe("moe_m1_e128", 1, 2048, 768, 128, 8, "fp16"),
        # the usual decode batch over middle-sized experts in FP8 mode
        _moe("moe_m16_e64_fp8", 16, 4096, 1408, 64, 6, "fp8", residual=True),
        # a few users of few large experts, the shapes of an 8B model's feed-forward
        _moe("moe_m4_e8_large", 4, 4096, 14336, 8, 2, "fp16"),
        # router and experts of a larger batch, the residual stream added
        _moe("layer_m48_e96", 48, 5120, 1520, 96, 6, "fp16", residual=True, kind="layer"),
    ]


def draw(rng):
    def log_int(lo, hi, mult=1):
        v = lo * (hi / lo) ** rng.random()
        return max(mult, int(round(v / mult)) * mult)

    kind = rng.choice(["fused", "fused", "fused", "route", "moe", "moe", "layer"])
    if kind == "fused":
        gated = rng.random() < 0.5
        mode = rng.choice(["fp16", "fp8"])
        tokens = log_int(1, 64) if rng.random() < 0.5 else log_int(1, 8192)
        rows, cols = log_int(64, 28672), log_int(256, 14336, 16)
        while rows * cols > 28672 * 4096:
            rows = max(64, rows * 3 // 4)
        return dict(kind=kind, tokens=tokens, rows=rows // 2 * 2 if gated else rows, cols=cols, mode=mode, gated=gated,
                    act=rng.choice(["silu", "gelu", "relu"] if gated else ["none", "silu", "gelu", "relu"]), bias=rng.random() < 0.5,
                    residual=rng.random() < 0.5, packed=rng.random() < 0.5, codes=mode == "fp8" and rng.random() < 0.5)
    experts = rng.choice([4, 8, 16, 60, 64, 96, 128, 160, 256])
    top_k = rng.choice([k for k in (1, 2, 4, 6, 8) if k <= experts])
    if kind == "route":
        return dict(kind=kind, tokens=log_int(1, 64) if rng.random() < 0.5 else log_int(1, 4096), hidden=log_int(256, 7168, 16), experts=experts,
                    top_k=top_k, scoring=rng.choice(["softmax", "sigmoid"]), renormalize=rng.random() < 0.7, bias=rng.random() < 0.5,
                    factor=rng.choice([1.0, 2.5]))
    hidden, ffn = log_int(256, 7168, 16), log_int(128, 14336, 16)
    while experts * hidden * ffn > 96 * 5120 * 1520:
        ffn = max(128, ffn * 3 // 4 // 16 * 16)
        hidden = max(256, hidden * 7 // 8 // 16 * 16)
    return dict(kind=kind, tokens=log_int(1, 48), hidden=hidden, ffn=ffn, experts=experts, top_k=top_k, mode=rng.choice(["fp16", "fp8"]),
                act=rng.choice(["silu", "silu", "gelu", "relu"]), residual=rng.random() < 0.5)


# ---- what follows from a case alone --------------------------------------------------------------------------------------------

def _experts_met(case):
    """Distinct experts that a batch chooses, on average, if every one is as likely as the others."""
    e = case["experts"]
    return e * (1.0 - (1.0 - case["top_k"] / e) ** case["tokens"])


def work(case):
    m = case["tokens"]
    if case["kind"] == "fused":
        n, k = case["rows"], case["cols"]
        out = n // 2 if case["gated"] else n
        data = n * k * (2 if case["mode"] == "fp16" else 1) + m * k * (1 if case["codes"] else 2) + 2 * m * out
        return {"bytes": data + (2 * m * out if case["residual"] else 0) + (2 * n if case["bias"] else 0), "flops": 2 * m * n * k}
    k, e = case["hidden"], case["experts"]
    router = {"bytes": 2 * m * k + 2 * e * k + 8 * m * case["top_k"], "flops": 2 * m * e * k}
    if case["kind"] == "route":
        return router
    weights = _experts_met(case) * 3 * k * case["ffn"] * (2 if case["mode"] == "fp16" else 1)
    got = {"bytes": int(weights) + 2 * m * k * (3 if case["residual"] else 2) + 8 * m * case["top_k"],
           "flops": 6 * m * case["top_k"] * k * case["ffn"]}
    if case["kind"] == "layer":                        # (the router's activations are the experts')
        got = {"bytes": got["bytes"] + 2 * e * k, "flops": got["flops"] + router["flops"]}
    return got


# ---- inputs --------------------------------------------------------------------------------------------------------------------

def _normal(g, shape, sigma=1.0):
    return torch.empty(shape, dtype=torch.float16, device=DEVICE).normal_(0.0, sigma, generator=g)


def _scales(x):
    """Largest magnitude of every row over 448, one division (by a number, torch multiplies by its reciprocal); 1 for a row of zeros."""
    amax = x.abs().amax(1)
    return torch.where(amax == 0, torch.ones_like(amax), amax / torch.full_like(amax, 448.0))


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    s = {"case": case}
    m = case["tokens"]
    if case["kind"] == "fused":
        n, k = case["rows"], case["cols"]
        out = n // 2 if case["gated"] else n
        s["x"], s["w"] = _normal(g, (m, k)), _normal(g, (n, k), 0.02)
        s["bias"] = _normal(g, (n,), 0.5) if case["bias"] else None
        s["residual"] = _normal(g, (m, out)) if case["residual"] else None
        if case["codes"]:                              # (what the norm in front of the linear left)
            x = s["x"].float()
            s["scales"] = _scales(x)
            s["codes"] = (x / s["scales"][:, None]).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)
    else:
        k, e, top = case["hidden"], case["experts"], case["top_k"]
        s["x"] = _normal(g, (m, k))
        if case["kind"] != "moe":
            s["router"] = _normal(g, (e, k), 1.0 / math.sqrt(k))
            s["bias"] = 0.1 * torch.randn(e, generator=g, device=DEVICE) if case.get("bias") else None
        if case["kind"] != "route":
            s["gate_up"], s["down"] = _normal(g, (e, 2 * case["ffn"], k), 0.02), _normal(g, (e, k, case["ffn"]), 0.02)
            s["residual"] = _normal(g, (m, k)) if case["residual"] else None
        if case["kind"] == "moe":                      # (a router's choice)
            chosen = torch.randn((m, e), generator=g, device=DEVICE).softmax(1).topk(top, 1)
            s["ids"] = chosen.indices.to(torch.int32).contiguous()
            s["weights"] = (chosen.values / chosen.values.sum(1, keepdim=True)).contiguous()
    if own:
        _handles(s)
    elif case.get("mode") == "fp8":
        _e4m3_weights(s)
    return s


def _e4m3_weights(s):
    """The weights in FP8 mode, as a program without the planes would keep them: E4M3 of 256 w."""
    for name in ("w", "gate_up", "down"):
        if name in s:
            got = torch.empty(s[name].shape, dtype=torch.float8_e4m3fn, device=DEVICE)
            for part, whole in zip(got if got.dim() == 3 else [got], s[name] if got.dim() == 3 else [s[name]]):
                part.copy_((whole.float() * 256.0).to(torch.float8_e4m3fn))
            s[name + "_e4m3"] = got


# ---- the framework's calls -----------------------------------------------------------------------------------------------------

def _handles(s):
    """What a program keeps between calls: the planes, output buffers, workspaces."""
    from paper_2506_02024_amd import binding as nfp

    case, m = s["case"], s["case"]["tokens"]
    s["nfp"] = nfp
    if "mode" in case:
        s["mode"] = nfp.MODE_FP16 if case["mode"] == "fp16" else nfp.MODE_FP8
        s["act"] = {"none": nfp.ACT_NONE, "relu": nfp.ACT_RELU, "silu": nfp.ACT_SILU, "gelu": nfp.ACT_GELU}[case["act"]]
    if case["kind"] == "fused":
        turn = nfp.interleave_gate_up if case["gated"] else (lambda t: t)
        s["layer"] = nfp.Layer(turn(s["w"]), packed=case["packed"])
        s["own_bias"] = None if s["bias"] is None else turn(s["bias"])
        s["out"] = torch.empty((m, case["rows"] // 2 if case["gated"] else case["rows"]), dtype=torch.float16, device=DEVICE)
        s["workspace"] = nfp.new_workspace(nfp.linear_fused_workspace_size(m, s["layer"], s["mode"]), DEVICE)
        return
    if case["kind"] != "moe":
        s["ids"] = torch.empty((m, case["top_k"]), dtype=torch.int32, device=DEVICE)
        s["weights"] = torch.empty((m, case["top_k"]), dtype=torch.float32, device=DEVICE)
        s["route_workspace"] = nfp.new_workspace(nfp.moe_route_workspace_size(m, case["experts"], case["hidden"]), DEVICE)
    if case["kind"] != "route":
        s["experts"] = nfp.Experts(s["gate_up"], s["down"], s["act"])
        s["out"] = torch.empty((m, case["hidden"]), dtype=torch.float16, device=DEVICE)
        s["workspace"] = nfp.new_workspace(nfp.moe_workspace_size(m, s["experts"], case["top_k"], s["mode"]), DEVICE)


def _run_own(s):
    if "nfp" not in s:
        _handles(s)
    nfp, case = s["nfp"], s["case"]
    if case["kind"] == "fused":
        x, scales = (s["codes"], s["scales"]) if case["codes"] else (s["x"], None)
        return nfp.linear_fused(x, s["layer"], s["mode"], bias=s["own_bias"], activation=s["act"], gated=case["gated"], residual=s["residual"],
                                scales=scales, out=s["out"], workspace=s["workspace"])
    if case["kind"] != "moe":
        nfp.moe_route(s["x"], s["router"], case["top_k"], scoring=case.get("scoring", "softmax"), renormalize=case.get("renormalize", True),
                      bias=s["bias"], factor=case.get("factor", 1.0), ids=s["ids"], weights=s["weights"], workspace=s["route_workspace"])
    got = {} if case["kind"] == "moe" else {"ids": s["ids"], "weights": s["weights"]}
    if case["kind"] != "route":
        got["y"] = nfp.moe(s["x"], s["experts"], s["ids"], s["weights"], s["mode"], residual=s["residual"], out=s["out"], workspace=s["workspace"])
    return got


# ---- plain forms ---------------------------------------------------------------------------------------------------------------

def _activate(z, act):
    if act == "relu":
        return z * (z > 0)
    if act == "silu":
        return z / (1.0 + (-z).exp())
    if act == "gelu":
        return 0.5 * z * (1.0 + (math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)).tanh())
    return z


def _weight(s, name, part=None):
    """Weights in 32 bits, as the mode has them."""
    if s["case"]["mode"] == "fp16":
        return (s[name] if part is None else s[name][part]).float()
    if name + "_e4m3" not in s:
        _e4m3_weights(s)
    w = s[name + "_e4m3"]
    return (w if part is None else w[part]).float() * 2.0 ** -8


def _run_fused(s):
    case = s["case"]
    if case["mode"] == "fp16":
        x = s["x"].float()
    elif case["codes"]:
        x = s["codes"].view(torch.float8_e4m3fn).float() * s["scales"][:, None]
    else:
        x = s["x"].float()
        scale = _scales(x)[:, None]
        x = (x / scale).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).float() * scale
    z = x @ _weight(s, "w").T
    if s["bias"] is not None:
        z = z + s["bias"].float()
    if case["gated"]:
        f = case["rows"] // 2
        z = _activate(z[:, :f], case["act"]) * z[:, f:]
    else:
        z = _activate(z, case["act"])
    if s["residual"] is not None:
        z = z + s["residual"].float()
    return z.half()


def _run_route(s):
    """The logits and what follows in 64 bits: which experts are the largest may not depend on the order of a sum."""
    case = s["case"]
    logits = s["x"].double() @ s["router"].double().T
    sigmoid = case.get("scoring", "softmax") == "sigmoid"
    score = 1.0 / (1.0 + (-logits).exp()) if sigmoid else (logits - logits.amax(1, keepdim=True)).exp()
    if not sigmoid:
        score = score / score.sum(1, keepdim=True)
    choice = score + s["bias"].double() if s["bias"] is not None else logits
    ids = choice.sort(dim=1, descending=True, stable=True).indices[:, :case["top_k"]]
    weights = score.gather(1, ids)
    if case.get("renormalize", True):
        weights = weights / weights.sum(1, keepdim=True)
    return ids.to(torch.int32), (weights * case.get("factor", 1.0)).float()


def _run_moe(s, ids, weights):
    case, f = s["case"], s["case"]["ffn"]
    x, ids = s["x"].float(), ids.long()
    y = s["residual"].float() if s["residual"] is not None else torch.zeros_like(x)
    for e in ids.unique().tolist():
        token, slot = (ids == e).nonzero(as_tuple=True)
        z = x[token] @ _weight(s, "gate_up", e).T
        h = _activate(z[:, :f], case["act"]) * z[:, f:]
        y = y.index_add(0, token, (h @ _weight(s, "down", e).T) * weights[token, slot][:, None])
    return y.half()


def run(state):
    if own:
        return _run_own(state)
    kind = state["case"]["kind"]
    if kind == "fused":
        return _run_fused(state)
    got = {}
    ids, weights = (state["ids"], state["weights"]) if kind == "moe" else _run_route(state)
    if kind != "moe":
        got = {"ids": ids, "weights": weights}
    if kind != "route":
        got["y"] = _run_moe(state, ids, weights)
    return got


# ---- 64 bits -------------------------------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    wide = torch.float64

    def weight(w):
        if case["mode"] == "fp16":
            return w.to(wide)
        return (w.float() * 256.0).to(torch.float8_e4m3fn).to(wide) / 256.0

    def sigma(t):
        return torch.where(t >= 0, 1.0 / (1.0 + torch.exp(-t.abs())), torch.exp(-t.abs()) / (1.0 + torch.exp(-t.abs())))

    def act(z):
        if case["act"] == "silu":
            return z * sigma(z)
        if case["act"] == "gelu":                      # 1 + tanh(u) = 2 sigma(2 u)
            return z * sigma(2.0 * (2.0 / math.pi) ** 0.5 * (z + 0.044715 * z ** 3))
        return z.clamp(min=0.0) if case["act"] == "relu" else z

    if case["kind"] == "fused":
        x = s["x"].to(wide)
        if case["mode"] == "fp8":                      # (codes and scales are part of the definition, in 32 bits)
            amax = s["x"].abs().amax(1).float()
            scale = torch.where(amax == 0, torch.ones_like(amax), torch.div(amax, torch.tensor([448.0], device=DEVICE)))
            codes = (s["x"].float() / scale[:, None]).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
            x = codes.to(wide) * scale.to(wide)[:, None]
        z = torch.matmul(x, weight(s["w"]).t().contiguous())
        if s["bias"] is not None:
            z += s["bias"].to(wide)
        if case["gated"]:
            gate, up = z.chunk(2, dim=1)
            z = act(gate) * up
        else:
            z = act(z)
        return z if s["residual"] is None else z + s["residual"].to(wide)

    got = {}
    if case["kind"] == "moe":
        ids, weights = s["ids"].long(), s["weights"].to(wide)
    else:
        logits = torch.nn.functional.linear(s["x"].to(wide), s["router"].to(wide))
        score = sigma(logits) if case.get("scoring") == "sigmoid" else torch.softmax(logits, dim=1)
        # the largest one after the other; the first of equal ones
        left = logits.clone() if s["bias"] is None else score + s["bias"].to(wide)
        rows, picked = torch.arange(case["tokens"], device=DEVICE), []
        for _ in range(case["top_k"]):
            best = left.amax(1, keepdim=True)
            at = torch.where(left == best, torch.arange(case["experts"], device=DEVICE), case["experts"]).amin(1)
            picked.append(at)
            left[rows, at] = -math.inf
        ids = torch.stack(picked, 1)
        weights = torch.stack([score[rows, at] for at in picked], 1)
        if case.get("renormalize", True):
            weights = weights / weights.sum(1, keepdim=True)
        weights = weights * case.get("factor", 1.0)
        got = {"ids": ids.to(torch.int32), "weights": weights}
    if case["kind"] == "route":
        return got
    y = torch.zeros((case["tokens"], case["hidden"]), dtype=wide, device=DEVICE) if s["residual"] is None else s["residual"].to(wide).clone()
    # a matrix of the experts' weights, zero where a token has not chosen one
    share = torch.zeros((case["tokens"], case["experts"]), dtype=wide, device=DEVICE).scatter_add_(1, ids, weights)
    for e in range(case["experts"]):
        who = share[:, e].nonzero()[:, 0]
        if who.numel():
            gate, up = torch.matmul(s["x"][who].to(wide), weight(s["gate_up"][e]).t().contiguous()).chunk(2, dim=1)
            y[who] += share[who, e, None] * torch.matmul(act(gate) * up, weight(s["down"][e]).t().contiguous())
    return {**got, "y": y}
