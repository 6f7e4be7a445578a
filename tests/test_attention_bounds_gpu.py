"""GPU: new tokens past the bound that the caller gave, and past the end of Q, lose their output and move nobody's position."""
import numpy as np
import pytest
import torch

from block_helpers import assert_attention_close, attention_ref
from test_paged_attention_gpu import _case, _dev

pytestmark = pytest.mark.gpu
MARK = 7.0                                             # no output is as large: values are normal, outputs their averages


@pytest.fixture(scope="module")
def nfp():
    from paper_2506_02024_amd import binding

    return binding


def _check(nfp, lens, news, tokens, max_new, window, sinks, fp8, d, heads=8, kv=2):
    cache, table, q = _case(lens, news, heads, kv, d, 32, fp8, seed=max_new)
    ref, a = attention_ref(q, cache, table, lens, news, heads, d ** -0.5, window, sinks)
    starts = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
    out = torch.full((tokens, heads * d), MARK, dtype=torch.float16, device="cuda:0")
    nfp.paged_attention(_dev(q[:tokens]), cache.to_device(nfp), _dev(table), _dev(np.asarray(lens, dtype=np.int32)), _dev(starts),
                        max_new=max_new, max_len=max(lens), window=window, sinks=sinks, out=out)
    place = np.concatenate([np.arange(n) for n in news])[:tokens]
    has = place < max_new
    assert has.any() and (out.cpu().numpy()[~has] == MARK).all()
    assert_attention_close(out[torch.from_numpy(has).to("cuda:0")], ref[:tokens][has], a[:tokens][has])


@pytest.mark.parametrize("fp8", [False, True], ids=["fp16", "e4m3"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 3)])
# rows of a sequence: 4 max_new; up to 32 (16 at 256 dims) they are the streaming kernel's, others the tile kernel's
@pytest.mark.parametrize("news,lens,max_new", [([10, 3, 8], [100, 3, 400], 4), ([10, 3, 8], [100, 3, 400], 8), ([150, 1, 90, 0], [150, 40, 700, 9], 60),
                                               ([12, 400], [40, 1300], 100), ([9], [9], 1)])
def test_more_new_tokens_than_the_bound(nfp, news, lens, max_new, window, sinks, d, fp8):
    _check(nfp, lens, news, sum(news), max_new, window, sinks, fp8, d)


@pytest.mark.parametrize("d", [64, 256])
@pytest.mark.parametrize("news,lens,missing", [([2, 6], [33, 250], 3), ([50, 80], [50, 600], 45), ([1, 1, 70], [5, 90, 70], 1)])
def test_new_tokens_past_the_end_of_q(nfp, news, lens, missing, d):
    _check(nfp, lens, news, sum(news) - missing, max(news), 0, 0, False, d)
    _check(nfp, lens, news, sum(news) - missing, max(news) - missing, 16, 2, False, d)


def test_a_bound_below_the_rows_that_see_nothing(nfp):
    # five tokens of which two are in the cache: the first three new tokens see nothing, with or without a bound
    lens, news = [2, 60], [5, 40]
    cache, table, q = _case(lens, news, 4, 2, 64, 16, False)
    ref, a = attention_ref(q, cache, table, lens, news, 4, 0.125)
    for max_new in (4, 40):
        out = torch.full((45, 256), MARK, dtype=torch.float16, device="cuda:0")
        nfp.paged_attention(_dev(q), cache.to_device(nfp), _dev(table), _dev(np.array(lens, dtype=np.int32)), _dev(np.array([0, 5, 45], dtype=np.int32)),
                            max_new=max_new, max_len=60, out=out)
        assert not out[:3].any()
        assert_attention_close(out[:4], ref[:4], a[:4])
        assert_attention_close(out[5:5 + max_new], ref[5:5 + max_new], a[5:5 + max_new])
