"""GPU: scales of an E4M3 cache that are not ordinary numbers, by both kernels of the attention."""
import numpy as np
import pytest
import torch

from block_helpers import assert_attention_close, attention_ref
from test_paged_attention_gpu import _case, _dev, _run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def nfp():
    from paper_2506_02024_amd import binding

    return binding


@pytest.fixture(params=[0, 1], ids=["streaming", "tiles"])
def kernel(nfp, request):
    nfp.tune("attn_tiles", request.param)
    yield request.param
    nfp.tune("attn_tiles", -1)


@pytest.mark.parametrize("which", ["k_scale", "v_scale"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("chunk", [-1, 256])
def test_a_scale_that_is_nan_reaches_its_head_and_no_other(nfp, kernel, chunk, d, which):
    lens, news, heads, kv = [900, 3, 40, 300], [5, 5, 5, 5], 6, 3          # (two of the second sequence's new tokens see nothing)
    cache, table, q = _case(lens, news, heads, kv, d, 32, True, seed=d)
    ref, a = attention_ref(q, cache, table, lens, news, heads, d ** -0.5)
    getattr(cache, which)[1] = np.nan
    nfp.tune("attn_chunk", chunk)
    try:
        got = _run(nfp, cache, table, q, lens, news).float().cpu().numpy().reshape(-1, heads, d)
    finally:
        nfp.tune("attn_chunk", -1)
    sees = np.ones(20, dtype=bool)
    sees[5:7] = False
    assert np.isnan(got[sees, 2:4]).all() and not got[~sees].any()
    others = [0, 1, 4, 5]
    assert_attention_close(torch.from_numpy(got[:, others]), ref[:, others], a[:, others])


@pytest.mark.parametrize("scale", [0.0, -1.0])
def test_a_scale_of_zero_and_a_negative_one(nfp, kernel, scale):
    lens, news, heads, kv, d = [500, 40], [4, 4], 4, 2, 128
    cache, table, q = _case(lens, news, heads, kv, d, 32, True)
    cache.k_scale[1] *= np.float32(scale)
    ref, a = attention_ref(q, cache, table, lens, news, heads, d ** -0.5)
    assert_attention_close(_run(nfp, cache, table, q, lens, news), ref, a)
