"""GPU: a decoder layer whose feed-forward half is one fused linear, or a mixture of experts with and without a shared one."""
import numpy as np
import pytest
import torch

import feed_forward_helpers as ff
from helpers import bits

pytestmark = pytest.mark.gpu
HIDDEN, HEADS, KV, DIM, FFN, PAGE, EPS, EXPERTS, EXPERT_FFN, TOP = 256, 4, 2, 64, 528, 16, 1e-5, 12, 96, 3


@pytest.fixture(scope="module")
def nfp():
    from paper_2506_02024_amd import binding

    return binding


def weights(g):
    make = lambda *s: ff.normal(g, *s, sigma=s[-1] ** -0.5)
    ones = torch.ones(HIDDEN, dtype=torch.float16, device="cuda:0")
    layer = dict(qkv=make((HEADS + 2 * KV) * DIM, HIDDEN), o=make(HIDDEN, HEADS * DIM), gate_up=make(2 * FFN, HIDDEN), down=make(HIDDEN, FFN), norm1=ones, norm2=ones)
    return layer, (make(EXPERTS, HIDDEN), make(EXPERTS, 2 * EXPERT_FFN, HIDDEN), make(EXPERTS, HIDDEN, EXPERT_FFN))


def inputs(nfp, g, tokens):
    cache = nfp.KVCache(tokens // PAGE + 2, PAGE, KV, DIM, device="cuda:0")
    ints = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda:0")
    pos = torch.arange(tokens, device="cuda:0", dtype=torch.int32)
    table = torch.arange(cache.pages, device="cuda:0", dtype=torch.int32)[None]
    return cache, pos, pos.clone(), table, ints([tokens])


def half(nfp, layer, w, mixture, x_in, mode):
    """The feed-forward half in 64 bits, from the residual stream behind the attention; the experts that the library's router chose."""
    h = x_in.double()
    x = h / torch.sqrt((h * h).mean(1, keepdim=True) + EPS)
    y = torch.zeros_like(h)
    if w is not None:
        gate, up = (x @ w["gate_up"].double().t().contiguous()).chunk(2, dim=1)
        y = (gate * torch.sigmoid(gate) * up) @ w["down"].double().t().contiguous()
    if mixture is not None:
        ids, share = nfp.moe_route(x.half(), mixture[0], TOP)
        for e in range(EXPERTS):
            part = (share.double() * (ids == e)).sum(1, keepdim=True)
            gate, up = (x @ mixture[1][e].double().t().contiguous()).chunk(2, dim=1)
            y += part * ((gate * torch.sigmoid(gate) * up) @ mixture[2][e].double().t().contiguous())
    return y


# FP16: half a dozen roundings of 2.1e-4 (2-norm); FP8: E4M3 operands, 2.6e-2 each, on the way through two linears (experts: weights alone)
@pytest.mark.parametrize("mode,bound", [(0, 2e-3), (1, 0.1)], ids=["fp16", "fp8"])
@pytest.mark.parametrize("kind", ["fused", "mixture", "shared"])
@pytest.mark.parametrize("tokens", [5, 150])
def test_layer(nfp, kind, mode, bound, tokens):
    from paper_2506_02024_amd.decoder_layer import DecoderLayer, Mixture, rotary_tables

    g = ff.generator(4)
    w, m = weights(g)
    mixture = None if kind == "fused" else Mixture(*m, TOP)
    own = dict(w, gate_up=None, down=None) if kind == "mixture" else w
    layer = DecoderLayer(heads=HEADS, kv_heads=KV, eps=EPS, fused=kind == "fused", mixture=mixture, **own)
    plain = DecoderLayer(heads=HEADS, kv_heads=KV, eps=EPS, **w)
    x, delta = ff.normal(g, tokens, HIDDEN), 0.3 * ff.normal(g, tokens, HIDDEN)
    cos, sin = rotary_tables(tokens, DIM)
    got = []
    for which in (layer, plain):
        cache, pos, slots, table, lens = inputs(nfp, g, tokens)
        stream = x.clone()
        got.append((which(delta.clone(), stream, mode, cache, pos, slots, table, lens, cos, sin), stream))
    (y, stream), (other, same) = got
    assert np.array_equal(bits(stream), bits(same))    # (up to here nothing differs)
    ref = half(nfp, layer, None if kind == "mixture" else w, None if kind == "fused" else m, stream, mode)
    assert (y.double() - ref).norm() <= bound * ref.norm()
    if kind == "fused":                                # torch's activation on float16: two roundings more
        assert (y.double() - ref).norm() <= (other.double() - ref).norm() * 1.05


@pytest.mark.parametrize("mode", [0, 1])
def test_replayed_decode_steps(nfp, mode):
    """A graph of a layer with a mixture and a shared expert, replayed, against the same calls made eagerly; the graph's workspace stays its own."""
    from paper_2506_02024_amd.decoder_layer import DecoderLayer, Mixture, rotary_tables

    g = ff.generator(5)
    w, m = weights(g)
    layer = DecoderLayer(heads=HEADS, kv_heads=KV, eps=EPS, mixture=Mixture(*m, TOP, scoring="sigmoid", bias=torch.zeros(EXPERTS, device="cuda:0"), factor=1.5), **w)
    batch, cos_sin = 6, rotary_tables(64, DIM)
    cache = nfp.KVCache(batch * 4, PAGE, KV, DIM, device="cuda:0")
    table = torch.arange(batch * 4, device="cuda:0", dtype=torch.int32).reshape(batch, 4)
    x, delta = ff.normal(g, batch, HIDDEN), ff.normal(g, batch, HIDDEN)
    lens = torch.full((batch,), 20, dtype=torch.int32, device="cuda:0")
    slots = (table[:, 1] * PAGE + 3).contiguous()
    ws = nfp.new_workspace(layer.workspace_size(batch, mode, cache, batch, 1, 64), "cuda:0")
    call = lambda c, s, ws: layer(delta, s, mode, c, lens - 1, slots, table, lens, *cos_sin, max_len=64, workspace=ws)
    stream = x.clone()
    call(cache, stream, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call(cache, stream, ws)
    for _ in range(3):
        x.normal_(generator=g)
        delta.normal_(generator=g)
        stream.copy_(x)
        eager = x.clone()
        again = call(nfp.KVCache(k=cache.k.clone(), v=cache.v.clone()), eager, None)
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(bits(out), bits(again)) and np.array_equal(bits(stream), bits(eager))
