"""One decoder layer of a served language model, from the library's calls as a serving program makes them: norm, the four linears over
byte planes, rotary positions and cache write, attention over the paged cache, in FP16 or FP8 mode per step.

    python -m paper_2506_02024_amd.decoder_layer        a prompt in two chunks, then decode steps from a graph, timed
"""
import time

import torch

from . import binding as nfp


class Mixture:
    """A mixture of experts in the place of a layer's feed-forward: router [experts, hidden], gate_up [experts, 2 ffn, hidden] (gate rows first), down [experts,
    hidden, ffn], float16 on the GPU; the experts become planes here.  The other arguments are those of moe_route."""

    def __init__(self, router, gate_up, down, top_k, scoring="softmax", renormalize=True, bias=None, factor=1.0):
        self.router, self.experts, self.top_k = router, nfp.Experts(gate_up, down, nfp.ACT_SILU), top_k
        self.choice = dict(scoring=scoring, renormalize=renormalize, bias=bias, factor=factor)

    def workspace_size(self, tokens):
        return max(nfp.moe_route_workspace_size(tokens, *self.router.shape),
                   nfp.moe_workspace_size(min(tokens, nfp.MOE_MOST_TOKENS), self.experts, self.top_k))

    def __call__(self, x, mode, residual, workspace):
        """The experts' weighted sum for the rows of x, added to residual in place if there is one.  More tokens than a call takes (a prompt) go through the
        experts in as many calls."""
        ids, weights = nfp.moe_route(x, self.router, self.top_k, workspace=workspace, **self.choice)
        out = torch.empty_like(x) if residual is None else residual
        for lo in range(0, x.shape[0], nfp.MOE_MOST_TOKENS):
            part = slice(lo, lo + nfp.MOE_MOST_TOKENS)
            nfp.moe(x[part], self.experts, ids[part], weights[part], mode, residual=None if residual is None else residual[part], out=out[part],
                    workspace=workspace)
        return out


class DecoderLayer:
    """The layer's weights (float16, on the GPU): qkv [(heads + 2 kv_heads) head_dim, hidden], o [hidden, heads head_dim], gate_up [2 ffn,
    hidden] (gate rows first), down [hidden, ffn], and the two norms' [hidden].  The linears become planes here.

    fused: the gate's activation and its product with the up projection in the gate_up linear's epilogue, in 32 bits, instead of torch's calls on
    float16.  mixture: a Mixture, which is added to what gate_up and down (a shared expert, fused) give, or is all there is if they are None.

    Calls that may overlap in time need workspaces of their own, and a captured graph needs one that stays: a program that captures calls
    or issues them on several streams makes one for each graph and stream, of the largest workspace_size among its calls (a smaller batch can need more
    than a larger one, where it splits K or a sequence into more parts), and passes it (all layers of a model can share it).  A call that is given none takes the layer's own, of which there is one for every stream, and while a graph is
    captured one from that graph's memory, which the graph clears in every replay (3 us a layer)."""

    def __init__(self, qkv, o, gate_up, down, norm1, norm2, heads, kv_heads, eps=1e-5, packed=False, fused=False, mixture=None):
        self.fused, self.mixture = fused or mixture is not None, mixture
        if self.fused and gate_up is not None:
            gate_up = nfp.interleave_gate_up(gate_up)
        self.linears = {name: nfp.Layer(w, packed=packed) for name, w in (("qkv", qkv), ("o", o), ("gate_up", gate_up), ("down", down))
                        if w is not None}
        self.norm1, self.norm2, self.heads, self.kv_heads, self.eps = norm1, norm2, heads, kv_heads, eps
        self._own = {}                                  # stream -> workspace; never one that a graph has seen

    def workspace_size(self, tokens, mode, cache, batch, max_new, max_len, window=0, sinks=0):
        """Bytes of workspace that a call of so many new tokens needs (nfp.new_workspace makes one)."""
        need = [nfp.gemm_workspace_size(tokens, *layer.shape, nfp.MODE_FP16 if layer.is_exception else mode) for layer in self.linears.values()]
        if self.mixture is not None:
            need.append(self.mixture.workspace_size(tokens))
        return max(need + [nfp.paged_attention_workspace_size(tokens, self.heads, cache, batch, max_new, max_len, window, sinks)])

    def _room(self, need, device):
        if torch.cuda.is_current_stream_capturing():
            return nfp.new_workspace(need, device)
        stream = torch.cuda.current_stream(device).cuda_stream
        if stream not in self._own or self._own[stream].numel() < need:
            # (the one before was made on this stream and used by nothing but eager calls on it: what takes its memory next comes after them)
            self._own[stream] = nfp.new_workspace(need, device)
        return self._own[stream]

    def _norm_linear(self, name, delta, stream, weight, mode, workspace):
        """The linear of the norm of stream + delta; the sum stays in stream.  In FP8 mode the norm writes the codes that the linear
        multiplies; a layer that keeps its FP16 weights takes the norm in FP16 in both modes."""
        layer = self.linears[name]
        if mode == nfp.MODE_FP16 or layer.is_exception:
            x, _, _, _ = nfp.add_rms_norm(delta, weight, self.eps, residual=stream, sum_out=stream)
            return nfp.linear(x, layer, mode, workspace=workspace)
        codes = torch.empty(delta.shape, dtype=torch.uint8, device=delta.device)
        scales = torch.empty(delta.shape[0], dtype=torch.float32, device=delta.device)
        nfp.add_rms_norm(delta, weight, self.eps, residual=stream, sum_out=stream, Xq=codes, scales=scales)
        return nfp.gemm_fp8_prequantized(codes, scales, layer.upper, workspace=workspace)

    def _feed_forward(self, delta, stream, mode, workspace):
        """Norm, gate and up with the activation, down; the mixture on top.  The norm writes the codes that gate_up multiplies in FP8 mode, and float16 where
        somebody reads it."""
        up = self.linears.get("gate_up")
        coded = up is not None and mode == nfp.MODE_FP8 and not up.is_exception
        x = codes = scales = y = None
        if coded:
            codes = torch.empty(delta.shape, dtype=torch.uint8, device=delta.device)
            scales = torch.empty(delta.shape[0], dtype=torch.float32, device=delta.device)
        if self.mixture is not None or not coded:
            x = torch.empty_like(delta)
        nfp.add_rms_norm(delta, self.norm2, self.eps, residual=stream, sum_out=stream, out=x, Xq=codes, scales=scales)
        if up is not None:
            h = nfp.linear_fused(codes if coded else x, up, mode, activation=nfp.ACT_SILU, gated=True, scales=scales, workspace=workspace)
            y = nfp.linear(h, self.linears["down"], mode, workspace=workspace)
        return y if self.mixture is None else self.mixture(x, mode, y, workspace)

    def __call__(self, delta, stream, mode, cache, positions, slots, table, lens, cos, sin, starts=None, max_new=None, max_len=None,
                 window=0, sinks=0, workspace=None):
        """Adds delta (the output of the layer before, float16 [tokens, hidden]) to stream in place and returns this layer's own delta, which
        the next layer (or the last norm) adds.  workspace: see the class.  The other arguments are those of rope_append and paged_attention."""
        per = delta.shape[0] // max(lens.shape[0], 1) if starts is None else delta.shape[0]
        most_new, most = per if max_new is None else max_new, table.shape[1] * cache.page_tokens if max_len is None else max_len
        need = self.workspace_size(delta.shape[0], mode, cache, lens.shape[0], most_new, most, window, sinks)
        if workspace is None:
            workspace = self._room(need, delta.device)
        elif workspace.numel() < need:
            raise ValueError("this call needs a workspace of %d bytes, not %d" % (need, workspace.numel()))
        q_cols, kv_cols = self.heads * cache.head_dim, self.kv_heads * cache.head_dim
        q, k, v = self._norm_linear("qkv", delta, stream, self.norm1, mode, workspace).split([q_cols, kv_cols, kv_cols], dim=1)
        q = nfp.rope_append(q, k, v, positions, slots, cache, cos, sin, out=q)
        o = nfp.paged_attention(q, cache, table, lens, starts, most_new, most, window=window, sinks=sinks, workspace=workspace)
        delta = nfp.linear(o, self.linears["o"], mode, workspace=workspace)
        if self.fused:
            return self._feed_forward(delta, stream, mode, workspace)
        gate, up = self._norm_linear("gate_up", delta, stream, self.norm2, mode, workspace).chunk(2, dim=1)
        return nfp.linear(torch.nn.functional.silu(gate) * up, self.linears["down"], mode, workspace=workspace)


def rotary_tables(positions, head_dim, theta=500000.0, device="cuda:0"):
    """(cos, sin) float32 [positions, head_dim / 2]."""
    angle = torch.arange(positions, dtype=torch.float64, device=device)[:, None] * theta ** (
        -torch.arange(head_dim // 2, dtype=torch.float64, device=device) / (head_dim // 2))
    return angle.cos().float(), angle.sin().float()


def main(hidden=4096, heads=32, kv_heads=8, head_dim=128, ffn=14336, prompt=1500, batch=16, steps=20, page=64, experts=32, expert_ffn=1408, top_k=4):
    g = torch.Generator(device="cuda:0")
    g.manual_seed(0)
    w = lambda *shape: torch.empty(shape, dtype=torch.float16, device="cuda:0").normal_(0.0, 0.02, generator=g)
    ones = torch.ones(hidden, dtype=torch.float16, device="cuda:0")
    weights = (w((heads + 2 * kv_heads) * head_dim, hidden), w(hidden, heads * head_dim), w(2 * ffn, hidden), w(hidden, ffn), ones, ones, heads, kv_heads)
    mixture = Mixture(w(experts, hidden), w(experts, 2 * expert_ffn, hidden), w(experts, hidden, expert_ffn), top_k)
    for what, layer in (("activation by torch", DecoderLayer(*weights)), ("activation in the linear", DecoderLayer(*weights, fused=True)),
                        ("%d of %d experts of %d" % (top_k, experts, expert_ffn), DecoderLayer(*weights[:2], None, None, *weights[4:], mixture=mixture))):
        print(what)
        run(layer, g, hidden, head_dim, prompt, batch, steps, page)


def run(layer, g, hidden, head_dim, prompt, batch, steps, page):
    kv_heads = layer.kv_heads
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
        workspace = nfp.new_workspace(layer.workspace_size(batch, mode, cache, batch, 1, columns * page), "cuda:0")     # (the graph's)

        def step():
            position = lens.long()
            lens.add_(1)
            return layer(delta, x, mode, cache, position.to(torch.int32), slots_of(at, position), table, lens, cos, sin, max_len=columns * page,
                         workspace=workspace)

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
