"""GPU: rotary positions and the write into the paged cache against a plain form in 64 bits."""
import numpy as np
import pytest
import torch

from block_helpers import HostCache
from helpers import bits

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def nfp():
    from paper_2506_02024_amd import binding

    return binding


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda:0")


def _tables(n, rotary):
    angle = np.arange(n)[:, None] * (10000.0 ** (-np.arange(rotary // 2) / max(1, rotary // 2)))[None, :]
    return np.cos(angle).astype(np.float32), np.sin(angle).astype(np.float32)


def _turn(x, cos, sin):
    """[M, heads, D] in 64 bits, and the size of the terms of every value."""
    x = x.astype(np.float64)
    r = cos.shape[1]
    out, size = x.copy(), np.zeros_like(x)
    c, s = cos.astype(np.float64)[:, None], sin.astype(np.float64)[:, None]
    a, b = x[..., :r], x[..., r:2 * r]
    out[..., :r], out[..., r:2 * r] = a * c - b * s, b * c + a * s
    size[..., :r] = size[..., r:2 * r] = np.abs(a) + np.abs(b)
    return out, size


def _check(nfp, slots, heads, kv, d, page, fp8, rotary, pages=None, seed=0, in_place=False):
    rng = np.random.default_rng(seed)
    M = len(slots)
    slots = np.asarray(slots, dtype=np.int32)
    pages = pages or int(slots.max()) // page + 2
    qkv = (rng.standard_normal((M, (heads + 2 * kv) * d)) * 2).astype(np.float16)
    positions = rng.integers(0, 500, M).astype(np.int32)
    cos, sin = _tables(500, rotary)
    cache = HostCache(pages, page, kv, d, fp8, seed)
    dev = cache.to_device(nfp)
    rows = _dev(qkv)
    q, k, v = rows.split([heads * d, kv * d, kv * d], dim=1)
    tables = dict(cos=_dev(cos), sin=_dev(sin)) if rotary else {}
    out = nfp.rope_append(q, k, v, _dev(positions), _dev(slots), dev, out=q if in_place else None, **tables)
    # the queries: FP16 of two products in 32 bits
    host = qkv.reshape(M, heads + 2 * kv, d)
    want, size = _turn(host[:, :heads], cos[positions], sin[positions]) if rotary else (host[:, :heads].astype(np.float64), 0.0)
    got = out.cpu().numpy().astype(np.float64).reshape(want.shape)
    assert np.all(np.abs(got - want) <= 2.0 ** -11 * np.abs(want) + 2.0 ** -22 * size + 2.0 ** -25)
    if not in_place:
        assert np.array_equal(bits(rows), qkv.view(np.uint16))
    # the cache: what was written, and nothing else
    keys, size = _turn(host[:, heads:heads + kv], cos[positions], sin[positions]) if rotary else (host[:, heads:heads + kv].astype(np.float64), np.zeros((M, kv, d)))
    values = host[:, heads + kv:]
    ok = (slots >= 0) & (slots < pages * page)
    at = slots[ok] // page, slots[ok] % page
    raw = {"k": cache.k.copy(), "v": cache.v.copy()}
    new = {}
    for name, store, index in (("k", dev.k, 0), ("v", dev.v, 1)):
        flat = store.cpu().numpy()
        e = 16 if fp8 else 8
        if name == "k":
            back = flat.transpose(0, 2, 4, 1, 3, 5).reshape(pages, page, kv, d)
        else:
            back = flat.transpose(0, 2, 3, 5, 1, 4).reshape(pages, page, kv, d)
        new[name] = back[at]
        untouched = np.ones((pages, page), dtype=bool)
        untouched[at] = False
        assert np.array_equal(back[untouched].view(np.uint8), raw[name][untouched].view(np.uint8)), name
    if fp8:
        for got, want, size, scale in ((new["k"], keys[ok], size[ok], cache.k_scale), (new["v"], values[ok].astype(np.float64), 0.0, cache.v_scale)):
            want = want / scale.astype(np.float64)[None, :, None]
            size = size / scale.astype(np.float64)[None, :, None]
            got = torch.from_numpy(got.copy()).view(torch.float8_e4m3fn).double().numpy()
            want = np.clip(want, -448, 448)
            assert np.all(np.abs(got - want) <= (2.0 ** -4 + 2.0 ** -20) * np.abs(want) + 2.0 ** -22 * size + 2.0 ** -10 * 1.001)
    else:
        assert np.array_equal(new["v"].view(np.uint16), values[ok].view(np.uint16))
        assert np.all(np.abs(new["k"].astype(np.float64) - keys[ok]) <= 2.0 ** -11 * np.abs(keys[ok]) + 2.0 ** -22 * size[ok] + 2.0 ** -25)


@pytest.mark.parametrize("fp8", [False, True], ids=["fp16", "e4m3"])
@pytest.mark.parametrize("d,rotary", [(64, 64), (96, 96), (128, 128), (256, 256), (128, 64), (96, 32), (256, 16), (64, 0), (128, 0), (256, 0)])
def test_dims(nfp, d, rotary, fp8):
    _check(nfp, [0, 5, 63, 64, 200, 17, 18], 6, 2, d, 16, fp8, rotary)


@pytest.mark.parametrize("fp8", [False, True], ids=["fp16", "e4m3"])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("start,count", [(0, 1), (0, 100), (5, 77), (13, 300), (16, 16), (8, 8), (250, 40)])
def test_runs_of_slots(nfp, start, count, page, fp8):
    _check(nfp, np.arange(start, start + count), 4, 1, 64, page, fp8, 64, seed=start)


@pytest.mark.parametrize("fp8", [False, True], ids=["fp16", "e4m3"])
def test_slots_in_any_order_and_padding(nfp, fp8):
    rng = np.random.default_rng(3)
    slots = rng.permutation(640)[:333].astype(np.int64)
    slots[::7] = -1
    slots[3] = 640                                      # the first place behind the cache
    slots[4] = 2 ** 31 - 1
    slots[5] = -2 ** 31
    _check(nfp, slots, 8, 2, 128, 64, fp8, 128, pages=10)
    # pieces of sequences one behind the other
    _check(nfp, np.concatenate([np.arange(100, 117), np.arange(33, 64), np.arange(320, 500), [7]]), 8, 2, 128, 32, fp8, 128)


def test_queries_in_place(nfp):
    _check(nfp, [4, 9, 100], 4, 2, 128, 16, False, 128, in_place=True)


def test_values_beyond_the_codes_saturate(nfp):
    cache = nfp.KVCache(1, 16, 1, 64, torch.uint8, "cuda:0")
    x = torch.zeros((3, 64), dtype=torch.float16, device="cuda:0")
    x[0], x[1], x[2] = 60000, float("-inf"), float("nan")
    nfp.rope_append(x, x, x, None, torch.arange(3, dtype=torch.int32, device="cuda:0"), cache)
    for rows in (cache.keys().reshape(16, 64), cache.values().reshape(16, 64)):
        assert torch.all(rows[0] == 0x7e) and torch.all(rows[1] == 0xfe) and torch.all(rows[2] & 0x7f == 0x7f)


def test_positions_outside_the_tables_give_nan(nfp):
    cache = nfp.KVCache(1, 16, 1, 64, device="cuda:0")
    cos, sin = (_dev(t) for t in _tables(10, 64))
    x = torch.ones((4, 64), dtype=torch.float16, device="cuda:0")
    out = nfp.rope_append(x, x, x, _dev(np.array([0, 9, 10, -1], dtype=np.int32)), _dev(np.arange(4, dtype=np.int32)), cache, cos, sin)
    assert torch.isfinite(out[:2]).all() and torch.isnan(out[2:]).all()
    keys = cache.keys().reshape(16, 64)
    assert torch.isfinite(keys[:2]).all() and torch.isnan(keys[2:4]).all()


def test_a_cache_whose_offsets_pass_32_bits(nfp):
    # 9 GB of values: the last page starts past 2^32 elements
    pages, page, kv, d = 140000, 256, 1, 128
    cache = nfp.KVCache(k=torch.empty((pages, kv, 16, d // 8, 16, 8), dtype=torch.float16, device="cuda:0"),
                        v=torch.empty((pages, kv, 16, 2, d, 8), dtype=torch.float16, device="cuda:0"))
    rng = np.random.default_rng(0)
    M = 300
    x = rng.standard_normal((M, d)).astype(np.float16)
    at = np.arange(M)
    table = np.array([[pages - 1, pages - 3]], dtype=np.int32)
    slots = (table[0][at // page].astype(np.int64) * page + at % page).astype(np.int32)
    xd = _dev(x)
    nfp.rope_append(xd, xd, xd, None, _dev(slots), cache)
    for view in (cache.keys(), cache.values()):
        rows = torch.stack([view[int(p)].reshape(page, d) for p in table[0]]).reshape(2 * page, d)[:M]
        assert np.array_equal(bits(rows), x.view(np.uint16))
    got = nfp.paged_attention(xd[-1:], cache, _dev(table), _dev(np.array([M], dtype=np.int32)))
    s = x.astype(np.float64) @ x[-1].astype(np.float64) * d ** -0.5
    p = np.exp(s - s.max())
    p /= p.sum()
    assert np.all(np.abs(got.cpu().numpy()[0] - p @ x.astype(np.float64)) <= 2.0 ** -9 * (p @ np.abs(x.astype(np.float64))) + 2.0 ** -24)


def test_refusals(nfp):
    cache = nfp.KVCache(2, 16, 2, 64, device="cuda:0")
    q, k = torch.zeros((3, 256), dtype=torch.float16, device="cuda:0"), torch.zeros((3, 128), dtype=torch.float16, device="cuda:0")
    at = torch.arange(3, dtype=torch.int32, device="cuda:0")
    cos = torch.zeros((8, 32), dtype=torch.float32, device="cuda:0")
    nfp.rope_append(q, k, k, at, at, cache, cos, cos)
    with pytest.raises(nfp.NestedFPError) as e:
        nfp.rope_append(q[:, :192], k, k, at, at, cache, cos, cos)        # 3 heads over 2
    assert e.value.status == nfp.ERR_SHAPE
    with pytest.raises(nfp.NestedFPError) as e:
        nfp.rope_append(q, k, k, at, at, cache, cos[:, :20].contiguous(), cos[:, :20].contiguous())
    assert e.value.status == nfp.ERR_SHAPE
    for bad in (dict(v=k[:, :64]), dict(k=k.float()), dict(slots=at.long()), dict(positions=at[:2]), dict(sin=None), dict(q=q[:2])):
        args = dict(q=q, k=k, v=k, positions=at, slots=at, cache=cache, cos=cos, sin=cos)
        with pytest.raises(ValueError):
            nfp.rope_append(**dict(args, **bad))
