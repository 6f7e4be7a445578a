"""The workspace of ragged batches stays bounded, and tiles that there is no room to split are worked out whole."""
import ctypes

import numpy as np
import pytest

MOST = (256 << 20) + 16384                             # parts, and the counters in front of them


@pytest.fixture(scope="module")
def nfp():
    from paper_2506_02024_amd import binding, build

    if build.is_stale():
        build.build_library()
    binding.lib()
    return binding


def test_ragged_workspaces_are_bounded(nfp):
    size = nfp.lib().nestedfp_paged_attention_workspace_size
    most = 0
    for d in (64, 96, 128, 256):
        for kv, heads in ((1, 1), (1, 8), (1, 71), (2, 16), (8, 32), (8, 64), (10, 10), (10, 40), (32, 32)):
            c = nfp._CacheStruct(1 << 20, 16, kv, d, 0, 0x10000, 0x10000, None, None)
            for batch in (2, 7, 64, 256, 600, 1000):
                for tokens in (batch + 1, batch + 33, batch + 600, 4 * batch + 7, 8192 + batch, 100000):
                    for max_new in (2, 9, 100, 512, tokens):
                        for length in (1000, 131072, 10000000):
                            most = max(most, size(tokens, batch, heads, ctypes.byref(c), min(max_new, tokens), length, 0, 0))
    assert 16384 < most <= MOST


@pytest.mark.gpu
@pytest.mark.parametrize("waves", [4, 8])
@pytest.mark.parametrize("fp8", [False, True], ids=["fp16", "e4m3"])
@pytest.mark.parametrize("most", [1 << 12, 1 << 16, 1 << 20, 1 << 22])
def test_more_tiles_than_there_is_room_for(nfp, most, waves, fp8):
    # parts of 256 tokens for sequences of up to `most`: there is room for all tiles' parts, for those of a few tiles, for none
    import torch

    from block_helpers import assert_attention_close, attention_ref
    from test_paged_attention_gpu import _case, _dev

    # (36 query heads to a key/value head: no sequence is the streaming kernel's)
    news, heads = [1] * 40, 36
    news[20], news[37] = 2, 30
    lens = [max(n, 20 + 61 * i % 900) for i, n in enumerate(news)]
    cache, table, q = _case(lens, news, heads, 1, 64, 16, fp8)
    ref, a = attention_ref(q, cache, table, lens, news, heads, 0.125)
    dev, starts = cache.to_device(nfp), np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
    nfp.tune("attn_waves", waves)
    nfp.tune("attn_chunk", 256)
    try:
        size = nfp.paged_attention_workspace_size(len(q), heads, dev, 40, max_new=30, max_len=most)
        assert size <= MOST and (size == 0) == (most == 1 << 22 or most == 1 << 20 and waves == 8)
        # (guarded: what lies behind the workspace stays as it was)
        room = torch.full((size + (1 << 20),), 0x5a, dtype=torch.uint8, device="cuda:0")
        room[:min(size, nfp.WORKSPACE_COUNTER_BYTES)] = 0
        got = nfp.paged_attention(_dev(q), dev, _dev(table), _dev(np.asarray(lens, dtype=np.int32)), _dev(starts), max_new=30, max_len=most,
                                  workspace=room[:size])
        assert_attention_close(got, ref, a, "%d waves, up to %d tokens" % (waves, most))
        assert bool((room[size:] == 0x5a).all()) and not room[:min(size, nfp.WORKSPACE_COUNTER_BYTES)].any()
    finally:
        nfp.tune("attn_waves", -1)
        nfp.tune("attn_chunk", -1)
