"""CPU: what stands around the linears rejects bad arguments before it touches a device, and its workspace stays bounded."""
import ctypes

import pytest

OK, ARG, SHAPE, WORKSPACE = 0, 1, 2, 4
FAKE = 0x10000                                             # aligned, never dereferenced


@pytest.fixture(scope="module")
def nfp():
    from paper_2506_02024_amd import binding, build

    if build.is_stale():
        build.build_library()
    binding.lib()
    return binding


def _cache(nfp, pages=8, page=16, kv=2, d=64, kind=0, k=FAKE, v=FAKE):
    return nfp._CacheStruct(pages, page, kv, d, kind, k, v, None, None)


def test_norm(nfp):
    def call(X=FAKE, M=4, K=64, ldx=64, R=FAKE, ldr=64, w=FAKE, eps=1e-5, s=FAKE, lds=64, Y=FAKE, ldy=64, Xq=FAKE, scales=FAKE):
        return nfp.lib().nestedfp_add_rms_norm(X, M, K, ldx, R, ldr, w, eps, s, lds, Y, ldy, Xq, scales, None)

    assert call(M=0) == OK
    for bad in (dict(X=0), dict(w=0), dict(Y=0, Xq=0), dict(scales=0), dict(M=-1), dict(K=0), dict(eps=-1.0), dict(eps=float("nan"))):
        assert call(**bad) == ARG, bad
    for bad in (dict(K=40), dict(ldx=56), dict(ldr=68), dict(lds=8), dict(ldy=60), dict(X=FAKE + 8), dict(R=FAKE + 2), dict(Xq=FAKE + 4),
                dict(scales=FAKE + 2), dict(w=FAKE + 8), dict(K=(1 << 21) + 16, ldx=1 << 22)):
        assert call(**bad) == SHAPE, bad


def test_cache_descriptions(nfp):
    size = nfp.lib().nestedfp_kv_cache_bytes
    assert size(ctypes.byref(_cache(nfp))) == 8 * 16 * 2 * 64 * 2
    assert size(ctypes.byref(_cache(nfp, kind=1))) == 8 * 16 * 2 * 64
    assert size(None) == 0
    for bad in (dict(page=8), dict(page=24), dict(page=512), dict(d=80), dict(d=0), dict(kv=0), dict(pages=-1), dict(kind=2), dict(pages=1 << 28),
                dict(pages=1 << 22, page=256, kv=32)):
        assert size(ctypes.byref(_cache(nfp, **bad))) == 0, bad
    assert size(ctypes.byref(_cache(nfp, pages=1 << 22, page=256, kv=16, d=256))) == (1 << 30) * 16 * 256 * 2


def test_append(nfp):
    def call(Q=FAKE, ldq=256, K=FAKE, ldk=128, V=FAKE, ldv=128, M=3, heads=4, cos=FAKE, sin=FAKE, known=10, rotary=64, positions=FAKE,
             slots=FAKE, out=FAKE, ldo=256, cache=None, **kw):
        c = _cache(nfp, **kw) if cache is None else cache
        return nfp.lib().nestedfp_rope_append(Q, ldq, K, ldk, V, ldv, M, heads, cos, sin, known, rotary, positions, slots, out, ldo,
                                              ctypes.byref(c) if c else None, None)

    assert call(M=0) == OK
    for bad in (dict(Q=0), dict(K=0), dict(V=0), dict(out=0), dict(slots=0), dict(cos=0), dict(positions=0), dict(M=-1), dict(heads=0), dict(rotary=-16),
                dict(cache=False), dict(k=0), dict(kind=5)):
        assert call(**bad) == ARG, bad
    for bad in (dict(heads=3), dict(ldq=248), dict(ldk=132), dict(ldv=120), dict(ldo=0), dict(rotary=24), dict(rotary=80), dict(Q=FAKE + 8),
                dict(slots=FAKE + 2), dict(page=20), dict(d=48), dict(v=FAKE + 8)):
        assert call(**bad) == SHAPE, bad


def test_attention(nfp):
    def call(Q=FAKE, tokens=4, ldq=256, heads=4, table=FAKE, ld=10, cols=10, lens=FAKE, batch=4, starts=0, max_new=1, max_len=160, scale=0.1,
             window=0, sinks=0, O=FAKE, ldo=256, ws=FAKE, n=1 << 24, cache=None, **kw):
        c = _cache(nfp, **kw) if cache is None else cache
        return nfp.lib().nestedfp_paged_attention(Q, tokens, ldq, heads, ctypes.byref(c) if c else None, table, ld, cols, lens, batch, starts or None,
                                                  max_new, max_len, scale, window, sinks, O, ldo, ws, n, None)

    assert call(tokens=0) == OK
    for bad in (dict(Q=0), dict(O=0), dict(lens=0), dict(table=0), dict(tokens=-1), dict(batch=-1), dict(batch=0), dict(heads=0), dict(max_new=0),
                dict(max_len=-1), dict(window=-1), dict(sinks=-1), dict(scale=float("nan")), dict(scale=float("inf")), dict(ld=9), dict(cols=-1),
                dict(tokens=5), dict(tokens=8), dict(cache=False), dict(k=0)):
        assert call(**bad) == ARG, bad
    for bad in (dict(heads=5), dict(ldq=200), dict(ldo=260), dict(Q=FAKE + 8), dict(O=FAKE + 4), dict(lens=FAKE + 1), dict(table=FAKE + 2),
                dict(max_len=1 << 31), dict(d=72), dict(page=40)):
        assert call(**bad) == SHAPE, bad
    # long sequences of a small batch are split over workgroups: a workspace is asked for
    assert call(max_len=100000, ws=0) == WORKSPACE
    assert call(max_len=100000, n=16384) == WORKSPACE
    assert call(max_len=100000, ws=FAKE + 4) == WORKSPACE


def test_attention_workspace_does_not_grow_with_the_cache(nfp):
    size = nfp.lib().nestedfp_paged_attention_workspace_size
    most = 0
    for d in (64, 96, 128, 256):
        for kind in (0, 1):
            for kv, heads in ((1, 1), (1, 71), (8, 32), (8, 64), (10, 40), (32, 32)):
                c = _cache(nfp, pages=1 << 20, kv=kv, d=d, kind=kind)
                for batch in (1, 7, 64, 600):
                    for new in (1, 4, 100):
                        for length in (1, 1000, 131072, 10000000):
                            for window in (0, 4096):
                                most = max(most, size(batch * new, batch, heads, ctypes.byref(c), new, length, window, 4))
    assert 16384 < most <= 512 << 20
    assert size(0, 4, 4, ctypes.byref(_cache(nfp)), 1, 100, 0, 0) == 0
    assert size(4, 4, 5, ctypes.byref(_cache(nfp)), 1, 100, 0, 0) == 0
    assert size(4, 4, 4, None, 1, 100, 0, 0) == 0
    assert size(4, 4, 4, ctypes.byref(_cache(nfp)), 1, 16, 0, 0) == 0          # nothing to split


@pytest.mark.gpu
def test_the_binding_refuses_what_is_not_on_the_gpu(nfp):
    import torch

    x, w = torch.zeros((4, 64), dtype=torch.float16), torch.ones(64, dtype=torch.float16)
    at = torch.zeros(4, dtype=torch.int32)
    cache = nfp.KVCache(2, 16, 1, 64, device="cpu")
    for call in (lambda: nfp.add_rms_norm(x, w), lambda: nfp.rope_append(x, x, x, at, at, cache),
                 lambda: nfp.paged_attention(x, cache, at.reshape(4, 1), at, workspace=torch.zeros(16, dtype=torch.uint8)),
                 lambda: nfp.add_rms_norm(x, None, out=x)):
        with pytest.raises(ValueError):
            call()


def test_keys_and_values_of_a_cache_as_views(nfp):
    import torch

    from block_helpers import HostCache

    with pytest.raises(ValueError):
        nfp.KVCache(k=torch.zeros((2, 1, 1, 8, 16, 8), dtype=torch.float16), v=torch.zeros((2, 1, 1, 2, 64, 4), dtype=torch.float16))
    with pytest.raises(ValueError):
        nfp.KVCache(2, 16, 1, 64, device="cpu", k_scale=torch.ones(2))
    for fp8 in (False, True):
        host = HostCache(3, 64, 2, 96, fp8, seed=4)
        k, v = (torch.from_numpy(a) for a in host.storage())
        cache = nfp.KVCache(k=k, v=v)
        for view, rows in ((cache.keys(), host.k), (cache.values(), host.v)):
            assert (view.reshape(rows.shape).numpy().view("uint8") == rows.view("uint8")).all()
