"""The operators that stand around the linears of a served decoder layer, as cases that can be timed and checked:

- norm: the residual's addition, the root-mean-square norm and, in FP8 mode, the E4M3 codes with a scale per
  token that the next linear takes as they are;
- append: rotary positions on the queries and keys of new tokens, and the write of keys and values into a
  paged cache in FP16 or E4M3;
- decode: attention of one new token (or a few drafted ones) of every sequence over the paged cache;
- prefill: the same of whole prompt chunks, alone or in one batch with decoding sequences.

`listed()` holds the cases, `draw(rng)` makes more of the same ranges, `prepare` makes what a serving program
has in hand (activations, tables, cache, page table, lengths, output buffers), `run` is one pass in elementary
torch operations or, where `own` is true, through the entry points of `paper_2506_02024_amd.binding`, and
`exact` the same values in 64 bits.

Cache storage (both sides read it): pages of `page` tokens; per page and key/value head the tokens go in blocks of 16.
With E elements in 16 bytes (8 FP16, 16 E4M3), a key block is [D / E][16 tokens][E dims] and a value block
[16 / E][D][E tokens].
"""
import math

import torch

own = False

DEVICE = "cuda:0"
EPS = 1e-5
THETA = 500000.0

# (query heads, key/value heads, head size, hidden size) of the models whose linears this repository measures
LLAMA_8B = dict(heads=32, kv_heads=8, dim=128, hidden=4096)
LLAMA_70B = dict(heads=64, kv_heads=8, dim=128, hidden=8192)
PHI_14B = dict(heads=40, kv_heads=10, dim=128, hidden=5120)
SMALL_1B = dict(heads=16, kv_heads=4, dim=64, hidden=1040)


def _norm(name, tokens, hidden, out):
    return dict(name=name, kind="norm", tokens=tokens, hidden=hidden, out=out)


def _heads(model):
    return {k: model[k] for k in ("heads", "kv_heads", "dim")}


def _append(name, model, batch, new, context, page, cache, rotary=0):
    return dict(_heads(model), name=name, kind="append", batch=batch, new=new, context=context, page=page, cache=cache,
                rotary=rotary or model["dim"])


def _decode(name, model, batch, shortest, longest, page, cache, drafts=1, window=0, sinks=0):
    return dict(_heads(model), name=name, kind="decode", batch=batch, shortest=shortest, longest=longest, page=page, cache=cache,
                drafts=drafts, window=window, sinks=sinks)


def _prefill(name, model, chunks, chunk, context, decoding, longest, page, cache, window=0, sinks=0):
    return dict(_heads(model), name=name, kind="prefill", chunks=chunks, chunk=chunk, context=context, decoding=decoding,
                longest=longest, page=page, cache=cache, window=window, sinks=sinks)


def listed():
    return [
        # one user of a small model with a ragged width: latency alone
        _norm("norm_m1_h1040_fp16", 1, SMALL_1B["hidden"], "fp16"),
        # a decode batch of a layer with an exception among its linears, which wants FP16 beside the codes
        _norm("norm_m48_h5120_both", 48, PHI_14B["hidden"], "both"),
        # the largest prefill batch in FP8 mode: codes only
        _norm("norm_m8192_h4096_e4m3", 8192, LLAMA_8B["hidden"], "e4m3"),
        # the usual decode batch into an 8-bit cache
        _append("append_b16_e4m3", LLAMA_8B, 16, 1, 1900, 64, "e4m3"),
        # three prompt chunks of odd length into an FP16 cache
        _append("append_b3_m1367_fp16", LLAMA_8B, 3, 1367, 0, 16, "fp16"),
        # a single user early in an answer: latency alone
        _decode("decode_b1_l613_fp16", LLAMA_8B, 1, 613, 613, 16, "fp16"),
        # a decode batch of ragged lengths
        _decode("decode_b32_l8192_fp16", LLAMA_8B, 32, 500, 8192, 64, "fp16"),
        # a large batch with long contexts in an 8-bit cache
        _decode("decode_b48_l20000_e4m3", LLAMA_70B, 48, 1000, 20000, 64, "e4m3"),
        # three drafted tokens per sequence, a window and a few first tokens that stay visible
        _decode("decode_b12_l50000_window", PHI_14B, 12, 3000, 50000, 32, "fp16", drafts=3, window=4096, sinks=4),
        # a short prompt of odd length of a small model
        _prefill("prefill_m777_d64", SMALL_1B, 1, 777, 0, 0, 0, 16, "fp16"),
        # two prompt chunks with context in one batch with decoding sequences, 8-bit cache
        _prefill("mixed_m600_e4m3", LLAMA_8B, 2, 600, 5200, 24, 6000, 64, "e4m3"),
        # the largest prompt
        _prefill("prefill_m8192_fp16", LLAMA_8B, 1, 8192, 0, 0, 0, 64, "fp16"),
    ]


def draw(rng):
    def log_int(lo, hi, mult=1):
        v = lo * (hi / lo) ** rng.random()
        return max(mult, int(round(v / mult)) * mult)

    kind = rng.choice(["norm", "append", "decode", "decode", "prefill", "prefill"])
    if kind == "norm":
        return dict(kind=kind, tokens=log_int(1, 8192), hidden=log_int(512, 4096 if rng.random() < 0.5 else 8192, 16) // 16 * 16,
                    out=rng.choice(["fp16", "e4m3", "both"])) if rng.random() < 0.7 else dict(
                        kind=kind, tokens=log_int(1, 2048), hidden=log_int(4096, 16384, 16), out=rng.choice(["fp16", "e4m3", "both"]))
    kv_heads = rng.choice([1, 2, 4, 8, 8, 10])
    dim = rng.choice([64, 96, 128, 128, 128, 256])
    heads = kv_heads * rng.choice([1, 3, 4, 4, 5, 7, 8, 16])
    if heads * dim > 8192:
        heads = kv_heads
    dims = dict(kind=kind, heads=heads, kv_heads=kv_heads, dim=dim, page=rng.choice([16, 16, 32, 64, 128, 256]),
                cache=rng.choice(["fp16", "e4m3"]))
    if kind == "append":
        batch = log_int(1, 64)
        return dict(dims, batch=batch, new=1 if rng.random() < 0.5 else log_int(1, max(1, 8192 // batch)), context=log_int(1, 4096),
                    rotary=rng.choice([dim, dim, dim // 2, 32]))
    window, sinks = rng.choice([(0, 0), (0, 0), (0, 0), (log_int(64, 8192), rng.choice([0, 1, 4, 17, 64]))])
    if kind == "decode":
        batch = log_int(1, 256)
        longest = log_int(1, min(131072, 300000 // batch))
        drafts = rng.choice([1, 1, 1, 2, 4, 7])
        shortest = log_int(1, longest) if longest > 1 else 1
        return dict(dims, batch=batch, shortest=min(shortest, longest), longest=longest, drafts=drafts, window=window, sinks=sinks)
    chunks = rng.choice([1, 1, 1, 2, 3, 5])
    chunk = log_int(2, 4096)
    context = rng.choice([0, log_int(1, 16384)])
    decoding = rng.choice([0, 0, log_int(1, 32)])
    longest = log_int(1, 8192) if decoding else 0
    most = 8192 * 8192 // 2 * 32 * 128
    while heads * dim * (chunks + decoding) * chunk * max(chunk + context, longest) > most:   # (the padded plain form too)
        chunk, context, longest = max(2, chunk * 3 // 4), context * 3 // 4, longest * 3 // 4
        decoding, longest = (decoding, longest) if longest else (0, 0)
    return dict(dims, chunks=chunks, chunk=chunk, context=context, decoding=decoding, longest=longest, window=window, sinks=sinks)


# ---- what follows from a case alone --------------------------------------------------------------------------------------------

def _spread(n, lo, hi):
    """n lengths from lo to hi, evenly over the logarithm, in a fixed mixed order."""
    got = [int(round(lo * (hi / lo) ** (i / (n - 1) if n > 1 else 1.0))) for i in range(n)]
    return [got[i * 7 % n] for i in range(n)] if n % 7 else got[::-1]


def _sequences(case):
    """(new tokens, tokens in the cache with the new ones) of every sequence."""
    if case["kind"] == "append":
        return [(case["new"], case["new"] + case["context"] + i % 5) for i in range(case["batch"])]
    if case["kind"] == "decode":
        t = case["drafts"]
        return [(t, max(t, n)) for n in _spread(case["batch"], case["shortest"], case["longest"])]
    # chunks of a length up to the largest, decoding sequences of any length between them
    got = [(max(1, case["chunk"] - 37 * i), max(1, case["chunk"] - 37 * i) + max(0, case["context"] - 211 * i)) for i in range(case["chunks"])]
    if case["decoding"]:
        one = [(1, n) for n in _spread(case["decoding"], max(1, case["longest"] // 16), case["longest"])]
        got = one[: len(one) // 2] + got + one[len(one) // 2:]
    return got


def _visible(case):
    """Pairs of a new token and a token that it sees, and tokens of the cache that some new token sees, over all sequences."""
    w, s = case.get("window", 0), case.get("sinks", 0)
    pairs = seen = 0
    for new, length in _sequences(case):
        first = length - new
        if w <= 0:
            pairs += sum(range(first + 1, length + 1))
            seen += length
            continue
        for pos in range(first, length):
            near = min(w, pos + 1)
            pairs += near + min(s, pos + 1 - near)
        low = max(0, first - w + 1)
        seen += length - low + min(s, low)
    return pairs, seen


def work(case):
    """Each input read once, each output written once; two flops per multiply-add."""
    if case["kind"] == "norm":
        m, h = case["tokens"], case["hidden"]
        out = {"fp16": 2, "e4m3": 1, "both": 3}[case["out"]]
        return {"bytes": m * h * (6 + out) + 2 * h + (0 if case["out"] == "fp16" else 4 * m), "flops": 6 * m * h}
    element = 2 if case["cache"] == "fp16" else 1
    tokens = sum(new for new, _ in _sequences(case))
    q, kv = case["heads"] * case["dim"], case["kv_heads"] * case["dim"]
    if case["kind"] == "append":
        positions = len({p for new, length in _sequences(case) for p in range(length - new, length)})
        return {"bytes": tokens * (4 * q + 4 * kv + 2 * element * kv + 8) + 4 * case["rotary"] * positions,
                "flops": 6 * tokens * (q + kv)}
    pairs, seen = _visible(case)
    return {"bytes": 2 * element * kv * seen + 4 * q * tokens, "flops": 4 * q * pairs}


# ---- inputs --------------------------------------------------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed))
    return g


def _normal(g, shape, sigma=1.0, dtype=torch.float16):
    return torch.empty(shape, dtype=torch.float32, device=DEVICE).normal_(0.0, sigma, generator=g).to(dtype)


def _storage(case, pages):
    """Shapes of the key and the value storage."""
    e = 8 if case["cache"] == "fp16" else 16
    head = (pages, case["kv_heads"], case["page"] // 16)
    return head + (case["dim"] // e, 16, e), head + (16 // e, case["dim"], e)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEVICE)


def prepare(case, seed):
    g = _generator(seed)
    state = dict(case)
    if case["kind"] == "norm":
        m, h = case["tokens"], case["hidden"]
        state["x"] = _normal(g, (m, h))
        # a residual stream: tokens of different magnitude, a few columns far larger than the rest
        state["residual"] = _normal(g, (m, h)) * torch.empty((m, 1), device=DEVICE).uniform_(0.5, 4.0, generator=g).half()
        state["residual"][:, h // 3] *= 30.0
        state["weight"] = (1.0 + 0.2 * _normal(g, (h,), dtype=torch.float32)).half()
        state["sum"] = torch.empty((m, h), dtype=torch.float16, device=DEVICE)
        if case["out"] != "e4m3":
            state["y"] = torch.empty((m, h), dtype=torch.float16, device=DEVICE)
        if case["out"] != "fp16":
            state["codes"] = torch.empty((m, h), dtype=torch.uint8, device=DEVICE)
            state["scales"] = torch.empty((m,), dtype=torch.float32, device=DEVICE)
        return state
    sequences = _sequences(case)
    page, kv, dim, heads = case["page"], case["kv_heads"], case["dim"], case["heads"]
    tokens = sum(new for new, _ in sequences)
    # the page table: pages in any order, a few more than the sequences need
    counts = [-(-length // page) for _, length in sequences]
    pages = sum(counts) + 3
    order = torch.randperm(pages, generator=g, device=DEVICE).to(torch.int32)
    columns = max(counts)
    place = torch.arange(columns, device=DEVICE)[None, :]
    starts = torch.cumsum(_ints(counts), 0) - _ints(counts)
    held = place < _ints(counts)[:, None]
    table = torch.where(held, order[torch.where(held, starts[:, None] + place, 0)], -1).to(torch.int32).contiguous()
    k_shape, v_shape = _storage(case, pages)
    if case["cache"] == "fp16":
        k, v = _normal(g, k_shape), _normal(g, v_shape)
        state["k_scale"] = state["v_scale"] = None
    else:
        # codes of keys and values whose scale was fixed by a calibration, another one for every head
        k, v = ((_normal(g, s, 60.0, torch.float32).clamp(-448.0, 448.0)).to(torch.float8_e4m3fn).view(torch.uint8)
                for s in (k_shape, v_shape))
        state["k_scale"], state["v_scale"] = (torch.empty(kv, device=DEVICE).uniform_(0.5, 2.0, generator=g) / 60.0 for _ in range(2))
    state.update(k=k, v=v, table=table)
    lens = _ints([length for _, length in sequences])
    firsts = [0]
    for new, _ in sequences:
        firsts.append(firsts[-1] + new)
    if case["kind"] == "append":
        # the rows that the qkv linear has just written
        qkv = _normal(g, (tokens, (heads + 2 * kv) * dim))
        state["q"], state["new_k"], state["new_v"] = qkv.split([heads * dim, kv * dim, kv * dim], dim=1)
        owner = torch.repeat_interleave(torch.arange(len(sequences), device=DEVICE), _ints([new for new, _ in sequences]), output_size=tokens)
        positions = torch.arange(tokens, device=DEVICE) - _ints(firsts[:-1])[owner] + lens[owner] - case["new"]
        state["positions"] = positions.to(torch.int32)
        state["slots"] = (table[owner, positions // page] * page + positions % page).to(torch.int32)
        r = case["rotary"] // 2
        angles = torch.arange(max(length for _, length in sequences), device=DEVICE, dtype=torch.float64)[:, None] * (
            THETA ** (-torch.arange(r, device=DEVICE, dtype=torch.float64) / r))[None, :]
        state["cos"], state["sin"] = angles.cos().float(), angles.sin().float()
        state["out"] = torch.empty((tokens, heads * dim), dtype=torch.float16, device=DEVICE)
        return state
    state["q"] = _normal(g, (tokens, heads * dim), 1.4)
    state["lens"], state["starts"] = lens, _ints(firsts)
    state["most_new"], state["most"] = max(new for new, _ in sequences), max(length for _, length in sequences)
    state["scale"] = 1.0 / math.sqrt(dim)
    state["out"] = torch.empty((tokens, heads * dim), dtype=torch.float16, device=DEVICE)
    return state


# ---- one pass ------------------------------------------------------------------------------------------------------------------

def _handles(s):
    """The binding, and what a program that uses it keeps beside its tensors: the description of its cache and a workspace."""
    from paper_2506_02024_amd import binding as nfp

    if "cache_handle" not in s and s["kind"] != "norm":
        s["cache_handle"] = nfp.KVCache(k=s["k"], v=s["v"], k_scale=s["k_scale"], v_scale=s["v_scale"])
        if s["kind"] != "append":
            need = nfp.paged_attention_workspace_size(s["q"].shape[0], s["heads"], s["cache_handle"], s["lens"].numel(), max_new=s["most_new"],
                                                      max_len=s["most"], window=s["window"], sinks=s["sinks"])
            s["workspace"] = nfp.new_workspace(need, DEVICE)
    return nfp


def _run_own(s):
    nfp = _handles(s)
    if s["kind"] == "norm":
        nfp.add_rms_norm(s["x"], s["weight"], EPS, residual=s["residual"], sum_out=s["sum"], out=s.get("y"), Xq=s.get("codes"),
                         scales=s.get("scales"))
        return _norm_outputs(s)
    if s["kind"] == "append":
        nfp.rope_append(s["q"], s["new_k"], s["new_v"], s["positions"], s["slots"], s["cache_handle"], s["cos"], s["sin"], out=s["out"])
        return _append_outputs(s)
    # (where every sequence has as many new tokens, the call needs no starts)
    return nfp.paged_attention(s["q"], s["cache_handle"], s["table"], s["lens"], starts=None if s["kind"] == "decode" else s["starts"],
                               max_new=s["most_new"], max_len=s["most"], scale=s["scale"], window=s["window"], sinks=s["sinks"],
                               out=s["out"], workspace=s["workspace"])


def _norm_outputs(s):
    got = {"sum": s["sum"]}
    if "y" in s:
        got["y"] = s["y"]
    if "codes" in s:
        got["codes"], got["scales"] = s["codes"].view(torch.float8_e4m3fn), s["scales"]
    return got


def _append_outputs(s):
    if s["cache"] == "fp16":
        return {"q": s["out"], "k": s["k"], "v": s["v"]}
    return {"q": s["out"], "k": s["k"].view(torch.float8_e4m3fn), "v": s["v"].view(torch.float8_e4m3fn)}


def _codes(x, scale):
    return (x / scale).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)


def _run_norm(s):
    h = (s["x"].float() + s["residual"].float()).half()
    s["sum"].copy_(h)
    h = h.float()
    y = h * torch.rsqrt(h.square().mean(dim=1, keepdim=True) + EPS) * s["weight"].float()
    if "y" in s:
        s["y"].copy_(y)
    if "codes" in s:
        amax = y.abs().amax(dim=1, keepdim=True)
        scale = torch.where(amax == 0, torch.ones_like(amax), amax / 448.0)
        s["codes"].copy_(_codes(y, scale))
        s["scales"].copy_(scale[:, 0])
    return _norm_outputs(s)


def _rotated(x, cos, sin, dim):
    """Rows of heads of `dim`; the first 2 r dims of a head are r pairs (i, i + r), r the width of the tables."""
    x = x.reshape(x.shape[0], -1, dim)
    r = cos.shape[1]
    a, b, rest = x[..., :r], x[..., r:2 * r], x[..., 2 * r:]
    c, s = cos[:, None, :], sin[:, None, :]
    return torch.cat([a * c - b * s, b * c + a * s, rest], dim=-1)


def _run_append(s):
    dim, kv, page = s["dim"], s["kv_heads"], s["page"]
    at = s["positions"].long()
    cos, sin = s["cos"][at], s["sin"][at]
    s["out"].copy_(_rotated(s["q"].float(), cos, sin, dim).flatten(1))
    k = _rotated(s["new_k"].float(), cos, sin, dim)
    v = s["new_v"].float().reshape(-1, kv, dim)
    if s["cache"] == "fp16":
        k, v = k.half(), v.half()
    else:
        k, v = _codes(k, s["k_scale"][None, :, None]), _codes(v, s["v_scale"][None, :, None])
    slots = s["slots"].long()
    where, block, token = slots // page, slots % page // 16, slots % 16
    e = s["k"].shape[-1]
    s["k"].permute(0, 2, 4, 1, 3, 5)[where, block, token] = k.reshape(-1, kv, dim // e, e)
    s["v"].permute(0, 2, 3, 5, 1, 4)[where, block, token // e, token % e] = v
    return _append_outputs(s)


def _rows(s, table, dtype):
    """Keys and values of the sequences of a table, as [sequence, head, token, dim] in `dtype`."""
    at = table.long().clamp(min=0)
    k = s["k"][at].permute(0, 2, 1, 3, 5, 4, 6)          # sequence, head, page, block, token, dims / e, e
    v = s["v"][at].permute(0, 2, 1, 3, 4, 6, 5)          # sequence, head, page, block, tokens / e, e, dim
    shape = (at.shape[0], s["kv_heads"], at.shape[1] * s["page"], s["dim"])
    k, v = k.reshape(shape), v.reshape(shape)
    if s["cache"] == "fp16":
        return k.to(dtype), v.to(dtype)
    return tuple(x.view(torch.float8_e4m3fn).to(dtype) * scale.to(dtype)[None, :, None, None]
                 for x, scale in ((k, s["k_scale"]), (v, s["v_scale"])))


def _run_attention(s):
    dim, kv, heads, new = s["dim"], s["kv_heads"], s["heads"], s["most_new"]
    lens, starts = s["lens"].long(), s["starts"].long()
    batch, tokens = lens.numel(), s["q"].shape[0]
    k, v = _rows(s, s["table"], torch.float32)
    # the sequences' new tokens, padded to as many for each
    i = torch.arange(new, device=DEVICE)[None, :]
    mine = starts[1:, None] - starts[:-1, None]
    row = (starts[:-1, None] + i).clamp(max=tokens - 1)
    q = s["q"].float()[row].reshape(batch, new, kv, heads // kv, dim).permute(0, 2, 3, 1, 4).reshape(batch, kv, -1, dim)
    t = torch.arange(k.shape[2], device=DEVICE)[None, None, :]
    pos = (lens[:, None] - mine + i)[:, :, None]
    seen = t <= pos
    if s["window"] > 0:
        seen &= (t > pos - s["window"]) | (t < s["sinks"])
    scores = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(s["scale"])
    scores = scores.reshape(batch, kv, heads // kv, new, -1).masked_fill_(~seen[:, None, None], -math.inf)
    top = scores.amax(dim=-1, keepdim=True).clamp_(min=-1e30)
    p = scores.sub_(top).exp_()
    total = p.sum(dim=-1, keepdim=True)
    o = torch.matmul(p.reshape(batch, kv, -1, p.shape[-1]), v).reshape(batch, kv, heads // kv, new, dim)
    o = torch.where(total > 0, o / total, torch.zeros_like(o)).permute(0, 3, 1, 2, 4).reshape(batch * new, heads * dim)
    # back to rows one after the other: the places of padding are the last to be taken
    back = torch.where(i < mine, row, tokens).reshape(-1)
    whole = torch.empty((tokens + 1, heads * dim), dtype=torch.float32, device=DEVICE)
    whole[back] = o
    s["out"].copy_(whole[:tokens])
    return s["out"]


def run(state):
    if own:
        return _run_own(state)
    if state["kind"] == "norm":
        return _run_norm(state)
    if state["kind"] == "append":
        return _run_append(state)
    return _run_attention(state)


# ---- the same in 64 bits -------------------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    wide = torch.float64
    if case["kind"] == "norm":
        total = (s["x"].to(wide) + s["residual"].to(wide))
        h = total.half().to(wide)                          # the sum is stored, and then used, in FP16
        y = h / (h.pow(2).sum(dim=1, keepdim=True) / case["hidden"] + EPS).sqrt() * s["weight"].to(wide)
        got = {"sum": total}
        if case["out"] != "e4m3":
            got["y"] = y
        if case["out"] != "fp16":
            scale = y.abs().max(dim=1, keepdim=True).values / 448.0
            got["codes"], got["scales"] = y / scale, scale[:, 0]
        return got
    dim, kv, heads, page = case["dim"], case["kv_heads"], case["heads"], case["page"]
    if case["kind"] == "append":
        r = case["rotary"] // 2
        at = s["positions"].long()

        def turned(x):
            x = x.to(wide).reshape(x.shape[0], -1, dim).clone()
            z = torch.complex(x[..., :r], x[..., r:2 * r]) * torch.complex(s["cos"][at].to(wide), s["sin"][at].to(wide))[:, None, :]
            x[..., :r], x[..., r:2 * r] = z.real, z.imag
            return x

        k, v = turned(s["new_k"]), s["new_v"].to(wide).reshape(-1, kv, dim)
        if case["cache"] == "fp16":
            whole_k, whole_v = s["k"].to(wide), s["v"].to(wide)
        else:
            whole_k, whole_v = (x.view(torch.float8_e4m3fn).to(wide) for x in (s["k"], s["v"]))
            k = (k / s["k_scale"].to(wide)[None, :, None]).clamp(-448.0, 448.0)
            v = (v / s["v_scale"].to(wide)[None, :, None]).clamp(-448.0, 448.0)
        # flat places of every value, written out from the storage's definition
        e = whole_k.shape[-1]
        slot, head, d = s["slots"].long()[:, None, None], torch.arange(kv, device=DEVICE)[None, :, None], torch.arange(dim, device=DEVICE)[None, None, :]
        block = ((slot // page) * kv + head) * (page // 16) + slot % page // 16
        token = slot % 16
        whole_k.view(-1)[((block * (dim // e) + d // e) * 16 + token) * e + d % e] = k
        whole_v.view(-1)[((block * (16 // e) + token // e) * dim + d) * e + token % e] = v
        return {"q": turned(s["q"]).flatten(1), "k": whole_k, "v": whole_v}
    out = torch.zeros((s["q"].shape[0], heads, dim), dtype=wide, device=DEVICE)
    first = 0
    for b, (new, length) in enumerate(_sequences(case)):
        # flat places of the sequence's keys and values, [head, token, dim]
        t = torch.arange(length, device=DEVICE)
        block = ((s["table"][b].long()[t // page][None, :, None] * kv + torch.arange(kv, device=DEVICE)[:, None, None]) * (page // 16)
                 + (t % page // 16)[None, :, None])
        e, d, token = s["k"].shape[-1], torch.arange(dim, device=DEVICE)[None, None, :], (t % 16)[None, :, None]
        keys = s["k"].reshape(-1)[((block * (dim // e) + d // e) * 16 + token) * e + d % e]
        values = s["v"].reshape(-1)[((block * (16 // e) + token // e) * dim + d) * e + token % e]
        if case["cache"] == "e4m3":
            keys, values = (x.view(torch.float8_e4m3fn).to(wide) * scale.to(wide)[:, None, None]
                            for x, scale in ((keys, s["k_scale"]), (values, s["v_scale"])))
        keys, values, t = keys.to(wide), values.to(wide), t[None, :]
        for lo in range(0, new, 2048):
            hi = min(new, lo + 2048)
            pos = torch.arange(length - new + lo, length - new + hi, device=DEVICE)[:, None]
            seen = t <= pos
            if case["window"] > 0:
                seen &= (pos - t < case["window"]) | (t < case["sinks"])
            for head in range(heads):
                at = head // (heads // kv)
                q = s["q"][first + lo:first + hi, head * dim:(head + 1) * dim].to(wide)
                scores = (q @ keys[at].t()) * s["scale"]
                p = torch.softmax(scores.masked_fill(~seen, -math.inf), dim=1)
                out[first + lo:first + hi, head] = p @ values[at]
        first += new
    return out.flatten(1)
