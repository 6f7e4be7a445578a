"""What a cache's storage may be: the calls refuse one in host memory before anything is launched."""
import pytest
import torch


@pytest.fixture(scope="module")
def nfp():
    from paper_2506_02024_amd import binding, build

    if build.is_stale():
        build.build_library()
    binding.lib()
    return binding


@pytest.mark.parametrize("dtype", [torch.float16, torch.uint8])
def test_the_calls_refuse_a_cache_in_host_memory(nfp, dtype):
    # (the compiled calls themselves, which need no stream: the cache is looked at before the other arguments)
    cache = nfp.KVCache(2, 16, 1, 64, dtype, device="cpu")
    x, at = torch.zeros((4, 64), dtype=torch.float16), torch.zeros(4, dtype=torch.int32)
    calls = nfp._marshalled()
    with pytest.raises(ValueError, match="cache must be on the GPU"):
        calls.rope_append(x, x, x, at, at, cache._at, None, None, x.clone(), 0)
    with pytest.raises(ValueError, match="cache must be on the GPU"):
        calls.paged_attention(x, cache._at, at.reshape(4, 1), at, None, 1, 16, 0.125, 0, 0, x.clone(), torch.zeros(16, dtype=torch.uint8), 0)


def test_storage_on_two_devices_is_refused(nfp):
    meta = torch.ones(1, device="meta")
    for bad in (dict(k_scale=meta), dict(v_scale=meta)):
        with pytest.raises(ValueError, match="one device"):
            nfp.KVCache(2, 16, 1, 64, torch.uint8, device="cpu", **bad)
    k, v = torch.zeros((2, 1, 1, 8, 16, 8), dtype=torch.float16), torch.zeros((2, 1, 1, 2, 64, 8), dtype=torch.float16, device="meta")
    with pytest.raises(ValueError, match="one device"):
        nfp.KVCache(k=k, v=v)


@pytest.mark.gpu
def test_only_the_cache_is_in_host_memory(nfp):
    cache = nfp.KVCache(2, 16, 1, 64, device="cpu")
    x, at = torch.zeros((4, 64), dtype=torch.float16, device="cuda:0"), torch.zeros(4, dtype=torch.int32, device="cuda:0")
    with pytest.raises(ValueError, match="cache must be on the GPU"):
        nfp.rope_append(x, x, x, None, at, cache)
    with pytest.raises(ValueError, match="cache must be on the GPU"):
        nfp.paged_attention(x, cache, at.reshape(4, 1), at)
    with pytest.raises(ValueError, match="one device"):
        nfp.KVCache(2, 16, 1, 64, torch.uint8, device="cuda:0", k_scale=torch.ones(1))


@pytest.mark.gpu
def test_storage_is_made_on_the_gpu(nfp):
    cache = nfp.KVCache(2, 16, 1, 64)
    assert cache.k.is_cuda and cache.v.is_cuda and cache._at


def test_scales_of_an_fp16_cache_are_refused(nfp):
    import ctypes

    for name in ("k_scale", "v_scale"):
        with pytest.raises(ValueError, match="E4M3"):
            nfp.KVCache(2, 16, 1, 64, device="cpu", **{name: torch.ones(1)})
        assert getattr(nfp.KVCache(2, 16, 1, 64, torch.uint8, device="cpu", **{name: torch.ones(1)}), name) is not None
    fake = 0x10000                                     # aligned, never dereferenced
    for kind, status in ((nfp.CACHE_FP16, nfp.ERR_ARG), (nfp.CACHE_E4M3, nfp.ERR_WORKSPACE)):
        for scales in ((fake, None), (None, fake)):
            c = nfp._CacheStruct(8, 16, 2, 64, kind, fake, fake, *scales)
            assert nfp.lib().nestedfp_paged_attention(fake, 4, 256, 4, ctypes.byref(c), fake, 10, 10, fake, 4, None, 1, 100000, 0.1, 0, 0, fake, 256,
                                                      None, 0, None) == status
            if kind == nfp.CACHE_FP16:
                assert nfp.lib().nestedfp_rope_append(fake, 256, fake, 128, fake, 128, 3, 4, fake, fake, 10, 64, fake, fake, fake, 256,
                                                      ctypes.byref(c), None) == nfp.ERR_ARG
