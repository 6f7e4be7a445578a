"""A decoder layer's workspace: what a captured graph was given stays the graph's, whatever the layer is called with afterwards."""
import types
import weakref

import numpy as np
import pytest
import torch

from block_helpers import page_table
from helpers import bits


class Library:
    """Stands for the binding: computes nothing, and notes every workspace that is made, with what was going on, and used."""

    MODE_FP16, MODE_FP8 = 0, 1

    def __init__(self, monkeypatch):
        self.capturing, self.stream, self.made, self.used = False, 0, {}, []
        monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: self.capturing)
        monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: types.SimpleNamespace(cuda_stream=self.stream))

    def Layer(self, w, packed=False):
        return types.SimpleNamespace(shape=tuple(w.shape), _dims=tuple(w.shape), is_exception=False, upper=None)

    def gemm_workspace_size(self, M, N, K, mode):
        return 64 * M

    def paged_attention_workspace_size(self, tokens, heads, cache, batch, max_new=None, max_len=0, window=0, sinks=0):
        return 100 * tokens

    def new_workspace(self, nbytes, device):
        ws = torch.zeros(nbytes, dtype=torch.uint8)
        self.made[ws.data_ptr()] = self.capturing
        return ws

    def _use(self, workspace):
        self.used.append((weakref.ref(workspace), workspace.data_ptr(), self.capturing, self.stream))

    def add_rms_norm(self, X, weight, eps, residual=None, sum_out=None, out=None, Xq=None, scales=None):
        return X, None, None, sum_out

    def linear(self, X, layer, mode, workspace=None):
        self._use(workspace)
        return torch.zeros((X.shape[0], layer.shape[0]), dtype=torch.float16)

    def gemm_fp8_prequantized(self, Xq, scales, upper, workspace=None):
        self._use(workspace)
        return torch.zeros((Xq.shape[0], 256 if len(self.used) % 5 == 1 else 64), dtype=torch.float16)      # (qkv, gate/up)

    def rope_append(self, q, *rest, out=None):
        return q

    def paged_attention(self, q, *rest, window=0, sinks=0, workspace=None):
        self._use(workspace)
        return q


@pytest.fixture
def library(monkeypatch):
    from paper_2506_02024_amd import decoder_layer

    lib = Library(monkeypatch)
    monkeypatch.setattr(decoder_layer, "nfp", lib)
    w = lambda n, k: torch.zeros((n, k), dtype=torch.float16)
    layer = decoder_layer.DecoderLayer(w(256, 64), w(64, 128), w(64, 64), w(64, 32), None, None, 2, 1)
    cache = types.SimpleNamespace(head_dim=64, page_tokens=16)

    def call(tokens, capturing=False, stream=0, **kw):
        lib.capturing, lib.stream, first = capturing, stream, len(lib.used)
        x = torch.zeros((tokens, 64), dtype=torch.float16)
        layer(x, x.clone(), kw.pop("mode", 0), cache, None, None, torch.zeros((1, 2)), torch.zeros(1), None, None, **kw)
        assert len(lib.used) > first
        return lib.used[first:]
    lib.layer, lib.cache, lib.call = layer, cache, call
    return lib


@pytest.mark.parametrize("mode", [0, 1])
def test_what_a_capture_used_is_alive_after_a_larger_call(library, mode):
    library.call(16, mode=mode)                         # (the warm-up before a capture)
    captured = library.call(16, capturing=True, mode=mode)
    library.call(4000, mode=mode)                       # a prompt
    for ref, place, _, _ in captured:
        # memory of the graph itself, or a tensor that is still held
        assert library.made[place] or ref() is not None


def test_a_workspace_that_only_a_graph_clears_is_not_used_outside_it(library):
    library.call(4000, capturing=True)
    eager = library.call(16)
    assert all(not library.made[place] for _, place, _, _ in eager)


def test_two_streams_have_two(library):
    first, second = library.call(16, stream=1), library.call(16, stream=2)
    again = library.call(16, stream=1)
    places = [{place for _, place, _, _ in used} for used in (first, second, again)]
    assert not places[0] & places[1] and places[0] == places[2]


def test_a_workspace_that_is_passed(library):
    need = library.layer.workspace_size(300, 0, library.cache, 1, 300, 32)
    assert need == 100 * 300
    mine = torch.zeros(need, dtype=torch.uint8)
    for capturing in (False, True):
        assert {place for _, place, _, _ in library.call(300, capturing=capturing, workspace=mine)} == {mine.data_ptr()}
    library.used.clear()
    with pytest.raises(ValueError):
        library.call(301, workspace=mine)
    assert not library.used and not library.made        # nothing ran, nothing was made


HIDDEN, HEADS, KV, DIM, FFN, PAGE = 256, 8, 2, 64, 528, 16


@pytest.mark.gpu
@pytest.mark.parametrize("mode", [0, 1], ids=["fp16", "fp8"])
@pytest.mark.parametrize("passed", [False, True])
def test_a_larger_prompt_between_capture_and_replay(mode, passed):
    from paper_2506_02024_amd import binding as nfp
    from paper_2506_02024_amd.decoder_layer import DecoderLayer, rotary_tables

    g = torch.Generator(device="cuda:0")
    g.manual_seed(5)
    make = lambda n, k: torch.empty((n, k), dtype=torch.float16, device="cuda:0").normal_(0.0, 1.0 / k ** 0.5, generator=g)
    ones = torch.ones(HIDDEN, dtype=torch.float16, device="cuda:0")
    layer = DecoderLayer(make((HEADS + 2 * KV) * DIM, HIDDEN), make(HIDDEN, HEADS * DIM), make(2 * FFN, HIDDEN), make(HIDDEN, FFN), ones, ones, HEADS, KV)
    # four sequences of some thousand tokens, which are split over workgroups; the prompt is a fifth one's
    lens_host, prompt = [3000, 900, 2000, 50], 1500
    table_host = page_table(np.random.default_rng(1), [n + 8 for n in lens_host] + [prompt], PAGE, 480, columns=200)
    table = torch.from_numpy(table_host).to("cuda:0")
    k, v = nfp.KVCache(480, PAGE, KV, DIM, device="cuda:0").k, nfp.KVCache(480, PAGE, KV, DIM, device="cuda:0").v
    cache = nfp.KVCache(k=k.normal_(generator=g), v=v.normal_(generator=g))
    cos, sin = rotary_tables(3200, DIM)
    ints = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda:0")
    slots = lambda b, p: ints(table_host[b, p // PAGE] * PAGE + p % PAGE)
    static = dict(delta=torch.zeros((4, HIDDEN), dtype=torch.float16, device="cuda:0"), x=torch.zeros((4, HIDDEN), dtype=torch.float16, device="cuda:0"),
                  pos=ints([0] * 4), slots=ints([-1] * 4), lens=ints([1] * 4))
    size = layer.workspace_size(4, mode, cache, 4, 1, 3100)
    workspaces = [nfp.new_workspace(size, "cuda:0") if passed else None for _ in range(2)]
    decode = lambda s, c, ws: layer(s["delta"], s["x"], mode, c, s["pos"], s["slots"], table[:4], s["lens"], cos, sin, max_len=3100, workspace=ws)
    decode(static, cache, workspaces[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = decode(static, cache, workspaces[0])
    for step in range(4):
        # a prompt that needs far more room, then tensors that take what memory became free
        n = prompt - 100 * step
        x = torch.empty((n, HIDDEN), dtype=torch.float16, device="cuda:0").normal_(generator=g)
        layer(x, x.clone(), nfp.MODE_FP8, cache, ints(np.arange(n)), slots(np.full(n, 4), np.arange(n)), table[4:], ints([n]), cos, sin, max_len=prompt)
        taken = [torch.full((max(size, 1 << 20),), 0x5a, dtype=torch.uint8, device="cuda:0") for _ in range(8)]
        p = np.array(lens_host) + step
        x, d = (torch.empty((4, HIDDEN), dtype=torch.float16, device="cuda:0").normal_(generator=g) for _ in range(2))
        eager = dict(delta=d, x=x.clone(), pos=ints(p), slots=slots(np.arange(4), p), lens=ints(p + 1))
        again = decode(eager, nfp.KVCache(k=cache.k.clone(), v=cache.v.clone()), workspaces[1])
        for name in static:
            static[name].copy_(x if name == "x" else eager[name])
        graph.replay()
        assert np.array_equal(bits(out), bits(again)) and np.array_equal(bits(static["x"]), bits(eager["x"]))
        assert all(bool((t == 0x5a).all()) for t in taken)
        del taken
    for ws in workspaces:
        if ws is not None:
            assert not ws[:nfp.WORKSPACE_COUNTER_BYTES].any()
