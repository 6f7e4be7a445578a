"""One decoder layer of a served language model, from the library's calls as a serving program makes them: norm, the four linears over
byte planes, rotary positions and cache write, attention over the paged cache, in FP16 or FP8 mode per step.

    python -m paper_2506_02024_amd.decoder_layer        a prompt in two chunks, then decode steps from a graph, timed
"""
import time

import torch

from . import binding as nfp


class DecoderLayer:
    """The layer's weights (float16, on the GPU): qkv [(heads + 2 kv_heads) head_dim, hidden], o [hidden, heads head_dim], gate_up [2 ffn,
    hidden] (gate rows first), down [hidden, ffn], and the two norms' [hidden].  The linears become planes here."""

    def __init__(self, qkv, o, gate_up, down, norm1, norm2, heads, kv_heads, eps=1e-5, packed=False):
        self.linears = {name: nfp.Layer(w, packed=packed) for name, w in (("qkv", qkv), ("o", o), ("gate_up", gate_up), ("down", down))}
        self.norm1, self.norm2, self.heads, self.kv_heads, self.eps = norm1, norm2, heads, kv_heads, eps
        self.workspace = None

    def _room(self, need, device):
        if self.workspace is None or self.workspace.numel() < need:
            self.workspace = nfp.new_workspace(need, device)
        return self.workspace

    def _linear(self, name, x, mode):
        layer = self.linears[name]
        need = nfp.gemm_workspace_size(x.shape[0], layer.shape[0], layer.shape[1], nfp.MODE_FP16 if layer.is_exception else mode)
        return nfp.linear(x, layer, mode, workspace=self._room(need, x.device))

    def _norm_linear(self, name, delta, stream, weight, mode):
        """The linear of the norm of stream + delta; the sum stays in stream.  In FP8 mode the norm writes the codes that the linear
        multiplies; a layer that keeps its FP16 weights takes the norm in FP16 in both modes."""
        layer = self.linears[name]
        if mode == nfp.MODE_FP16 or layer.is_exception:
            x, _, _, _ = nfp.add_rms_norm(delta, weight, self.eps, residual=stream, sum_out=stream)
            return self._linear(name, x, mode)
        codes = torch.empty(delta.shape, dtype=torch.uint8, device=delta.device)
        scales = torch.empty(delta.shape[0], dtype=torch.float32, device=delta.device)
        nfp.add_rms_norm(delta, weight, self.eps, residual=stream, sum_out=stream, Xq=codes, scales=scales)
        need = nfp.gemm_workspace_size(delta.shape[0], *layer.shape, mode)
        return nfp.gemm_fp8_prequantized(codes, scales, layer.upper, workspace=self._room(need, delta.device))

    def __call__(self, delta, stream, mode, cache, positions, slots, table, lens, cos, sin, starts=None, max_new=None, max_len=None,
                 window=0, sinks=0):
        """Adds delta (the output of the layer before, float16 [tokens, hidden]) to stream in place and returns this layer's own delta, which
        the next layer (or the last norm) adds.  The other arguments are those of rope_append and paged_attention."""
        q_cols, kv_cols = self.heads * cache.head_dim, self.kv_heads * cache.head_dim
        q, k, v = self._norm_linear("qkv", delta, stream, self.norm1, mode).split([q_cols, kv_cols, kv_cols], dim=1)
        q = nfp.rope_append(q, k, v, positions, slots, cache, cos, sin, out=q)
        per = delta.shape[0] // max(lens.shape[0], 1) if starts is None else delta.shape[0]
        most_new, most = per if max_new is None else max_new, table.shape[1] * cache.page_tokens if max_len is None else max_len
        need = nfp.paged_attention_workspace_size(q.shape[0], self.heads, cache, lens.shape[0], most_new, most, window, sinks)
        o = nfp.paged_attention(q, cache, table, lens, starts, most_new, most, window=window, sinks=sinks, workspace=self._room(need, q.device))
        delta = self._linear("o", o, mode)
        gate, up = self._norm_linear("gate_up", delta, stream, self.norm2, mode).chunk(2, dim=1)
        return self._linear("down", torch.nn.functional.silu(gate) * up, mode)


def rotary_tables(positions, head_dim, theta=500000.0, device="cuda:0"):
    """(cos, sin) float32 [positions, head_dim / 2]."""
    angle = torch.arange(positions, dtype=torch.float64, device=device)[:, None] * theta ** (
        -torch.arange(head_dim // 2, dtype=torch.float64, device=device) / (head_dim // 2))
    return angle.cos().float(), angle.sin().float()


def main(hidden=4096, heads=32, kv_heads=8, head_dim=128, ffn=14336, prompt=1500, batch=16, steps=20, page=64):
    g = torch.Generator(device="cuda:0")
    g.manual_seed(0)
    w = lambda n, k: torch.empty((n, k), dtype=torch.float16, device="cuda:0").normal_(0.0, 0.02, generator=g)
    ones = torch.ones(hidden, dtype=torch.float16, device="cuda:0")
    layer = DecoderLayer(w((heads + 2 * kv_heads) * head_dim, hidden), w(hidden, heads * head_dim), w(2 * ffn, hidden), w(hidden, ffn),
                         ones, ones, heads, kv_heads)
    columns = -(-(prompt + 2 * (steps + 4)) // page)
    cache = nfp.KVCache(batch * columns, page, kv_heads, head_dim, device="cuda:0")
    table = torch.randperm(batch * columns, generator=g, device="cuda:0").to(torch.int32).reshape(batch, columns)
    cos, sin = rotary_tables(columns * page, head_dim)
    at = torch.arange(batch, device="cuda:0")

    def slots_of(owner, position):
        return (table[owner, position // page] * page + position % page).to(torch.int32)

    # every sequence's prompt in two chunks, one call for all sequences; twice, since first calls load kernels and allocate (a cache's slots may be written again)
    for lo, hi in ((0, prompt * 2 // 3), (prompt * 2 // 3, prompt)):
        n = hi - lo
        x = torch.empty((batch * n, hidden), dtype=torch.float16, device="cuda:0").normal_(generator=g)
        position = torch.arange(lo, hi, device="cuda:0").repeat(batch)
        lens = torch.full((batch,), hi, dtype=torch.int32, device="cuda:0")
        mode = nfp.select_mode(x.shape[0])                # (many tokens: FP8 mode)
        for _ in range(2):
            again = x.clone()
            torch.cuda.synchronize()
            began = time.perf_counter()
            layer(torch.zeros_like(x), again, mode, cache, position.to(torch.int32), slots_of(at.repeat_interleave(n), position), table, lens, cos, sin, max_len=hi)
            torch.cuda.synchronize()
        print("prompt tokens %d ... %d of %d sequences: %.2f ms" % (lo, hi - 1, batch, 1e3 * (time.perf_counter() - began)))
    # decode steps: lengths and slots live on the GPU, so that one captured graph serves all steps
    x, delta = torch.empty((batch, hidden), dtype=torch.float16, device="cuda:0").normal_(generator=g), torch.zeros((batch, hidden), dtype=torch.float16, device="cuda:0")
    lens = torch.full((batch,), prompt, dtype=torch.int32, device="cuda:0")
    for mode, name in ((nfp.MODE_FP16, "FP16"), (nfp.MODE_FP8, "FP8")):
        def step():
            position = lens.long()
            lens.add_(1)
            return layer(delta, x, mode, cache, position.to(torch.int32), slots_of(at, position), table, lens, cos, sin, max_len=columns * page)

        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        torch.cuda.synchronize()
        began = time.perf_counter()
        for _ in range(steps):
            graph.replay()
        torch.cuda.synchronize()
        print("decode, %s mode, %d sequences of %d tokens: %.1f us a step" % (name, batch, int(lens[0]), 1e6 * (time.perf_counter() - began) / steps))


if __name__ == "__main__":
    main()
