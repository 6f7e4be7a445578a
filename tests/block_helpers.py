"""Plain 64-bit forms of what stands around the linears, and a paged cache written out from its definition."""
import numpy as np
import torch


def blocks_of(rows, fp8):
    """(keys, values) storage blocks of [blocks, 16 tokens, D] rows, written out from the storage's definition:
    [D / E][16][E] and [16 / E][D][E] per block."""
    n, _, d = rows.shape
    e = 16 if fp8 else 8
    k = rows.reshape(n, 16, d // e, e).transpose(0, 2, 1, 3)
    v = rows.reshape(n, 16 // e, e, d).transpose(0, 1, 3, 2)
    return np.ascontiguousarray(k), np.ascontiguousarray(v)


class HostCache:
    """Keys and values as rows [pages, page tokens, kv heads, D] on the host, FP16 values or E4M3 codes."""

    def __init__(self, pages, page, kv, d, fp8, seed=0, fill=None):
        rng = np.random.default_rng(seed)
        self.shape, self.page, self.fp8, self.d, self.kv = (pages, page, kv, d), page, fp8, d, kv
        if fp8:
            make = lambda: torch.from_numpy(rng.standard_normal(self.shape, dtype=np.float32) * 60).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).numpy().copy()
            self.k_scale, self.v_scale = ((rng.uniform(0.5, 2.0, kv) / 60).astype(np.float32) for _ in range(2))
        else:
            make = lambda: rng.standard_normal(self.shape, dtype=np.float32).astype(np.float16)
            self.k_scale = self.v_scale = None
        self.k, self.v = make(), make()
        if fill is not None:                               # memory that nothing was written to
            for x in (self.k, self.v):
                x[...] = 0x7f if fp8 else np.float16(fill)

    def wide(self, which):
        x = getattr(self, which)
        if not self.fp8:
            return x.astype(np.float64)
        scale = getattr(self, which + "_scale").astype(np.float64)
        return torch.from_numpy(x).view(torch.float8_e4m3fn).double().numpy() * scale[None, None, :, None]

    def storage(self):
        pages, page, kv, d = self.shape
        got = []
        for i, x in enumerate((self.k, self.v)):
            rows = x.transpose(0, 2, 1, 3).reshape(pages * kv * page // 16, 16, d)
            b = blocks_of(rows, self.fp8)[i]
            got.append(b.reshape((pages, kv, page // 16) + b.shape[1:]))
        return got

    def to_device(self, nfp, device="cuda:0"):
        k, v = (torch.from_numpy(x).to(device) for x in self.storage())
        scales = [None if s is None else torch.from_numpy(s).to(device) for s in (self.k_scale, self.v_scale)]
        return nfp.KVCache(k=k, v=v, k_scale=scales[0], v_scale=scales[1])


def attention_ref(q, cache, table, lens, news, heads, scale, window=0, sinks=0):
    """(o, a): outputs [tokens, heads, D] in 64 bits and a = sum p |v| / sum p, the size against which the rounding of the
    probabilities counts.  q: float16 [tokens, heads * D]; a new token that sees nothing gives zero."""
    d, kv, page = cache.d, cache.kv, cache.page
    k, v = cache.wide("k"), cache.wide("v")
    q = q.astype(np.float64).reshape(len(q), heads, d)
    o, a = np.zeros_like(q), np.zeros_like(q)
    first = 0
    for b, new in enumerate(news):
        for i in range(new):
            pos = lens[b] - new + i
            t = np.arange(max(0, pos + 1))
            if window > 0:
                t = t[(t > pos - window) | (t < sinks)]
            if len(t):
                at = table[b][t // page], t % page
                for h in range(heads):
                    g = h // (heads // kv)
                    s = (k[at[0], at[1], g] @ q[first + i, h]) * scale
                    p = np.exp(s - s.max())
                    p /= p.sum()
                    o[first + i, h] = p @ v[at[0], at[1], g]
                    a[first + i, h] = p @ np.abs(v[at[0], at[1], g])
        first += new
    return o, a


def assert_attention_close(got, ref, a, what=""):
    """An FP16 output (half a unit: 2^-11) of sums whose probabilities are rounded to FP16 (2^-11 of their size each, and as
    much again for everything that is held in 32 bits: scores, exponentials, sums)."""
    got = got.detach().cpu().numpy().astype(np.float64).reshape(ref.shape)
    assert np.all(np.isfinite(got)), what + ": not finite"
    bound = 2.0 ** -11 * np.abs(ref) + 2.0 ** -10 * a + 2.0 ** -24
    worst = np.max(np.abs(got - ref) / bound)
    assert worst <= 1.0, "%s: %g of the bound" % (what, worst)


def page_table(rng, lens, page, pages, spare=0, columns=None):
    """A table of pages in any order for sequences of these lengths; entries that no sequence needs are -1."""
    need = [-(-n // page) for n in lens]
    order = rng.permutation(pages)[: sum(need)]
    assert sum(need) + spare <= pages
    table = np.full((len(lens), columns or max(1, max(need))), -1, dtype=np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table
