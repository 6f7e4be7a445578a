"""GPU: attention of prompt chunks over a paged cache (tiles of many rows) against a plain form in 64 bits."""
import numpy as np
import pytest
import torch

from helpers import bits
from test_paged_attention_gpu import _case, _dev, _run
from block_helpers import assert_attention_close, attention_ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def nfp():
    from paper_2506_02024_amd import binding

    return binding


@pytest.fixture
def knobs(nfp):
    def pin(**kw):
        for name, value in kw.items():
            nfp.tune(name, value)
    yield pin
    nfp.tune("attn_chunk", -1)
    nfp.tune("attn_tiles", -1)


def _check(nfp, lens, news, heads, kv, d, page, fp8, window=0, sinks=0, seed=0, **kw):
    cache, table, q = _case(lens, news, heads, kv, d, page, fp8, seed)
    got = _run(nfp, cache, table, q, lens, news, window=window, sinks=sinks, **kw)
    ref, a = attention_ref(q, cache, table, lens, news, heads, d ** -0.5, window, sinks)
    assert_attention_close(got, ref, a, "%r" % ((lens, news, heads, kv, d, page, fp8, window, sinks),))


@pytest.mark.parametrize("fp8", [False, True], ids=["fp16", "e4m3"])
@pytest.mark.parametrize("d", [64, 96, 128, 256])
@pytest.mark.parametrize("heads,kv,new,context", [(4, 1, 33, 0), (4, 2, 130, 0), (3, 1, 100, 77), (2, 2, 257, 30), (5, 1, 64, 500), (8, 1, 19, 1)])
def test_one_chunk(nfp, heads, kv, new, context, d, fp8):
    _check(nfp, [new + context], [new], heads, kv, d, 16, fp8, seed=new)


@pytest.mark.parametrize("fp8", [False, True], ids=["fp16", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 64, 256])
def test_chunks_beside_decoding_sequences(nfp, page, d, fp8):
    news = [1, 1, 150, 0, 7, 70, 1, 8, 9, 2]
    lens = [1, 300, 150, 44, 7, 400, 17, 100, 9, 65]
    _check(nfp, lens, news, 8, 2, d, page, fp8)


@pytest.mark.parametrize("fp8", [False, True], ids=["fp16", "e4m3"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 3), (16, 4), (63, 0), (100, 17), (64, 64), (200, 1000), (5000, 4)])
def test_window_and_sinks(nfp, knobs, window, sinks, fp8):
    news, lens = [140, 1, 90], [140, 333, 640]
    for chunk in (-1, 256):
        knobs(attn_chunk=chunk)
        _check(nfp, lens, news, 4, 2, 128, 32, fp8, window, sinks)


@pytest.mark.parametrize("fp8", [False, True], ids=["fp16", "e4m3"])
@pytest.mark.parametrize("d", [64, 96, 128, 256])
@pytest.mark.parametrize("chunk", [256, 512, 100000])
def test_split_over_workgroups(nfp, knobs, chunk, d, fp8):
    news, lens = [70, 1, 300, 40], [1500, 700, 300, 41]
    knobs(attn_chunk=chunk)
    cache, table, q = _case(lens, news, 4, 2, d, 64, fp8, 1)
    ref, a = attention_ref(q, cache, table, lens, news, 4, d ** -0.5)
    first = _run(nfp, cache, table, q, lens, news)
    assert_attention_close(first, ref, a)
    for _ in range(2):                                     # (the counters are left as they were found)
        assert np.array_equal(bits(first), bits(_run(nfp, cache, table, q, lens, news)))


@pytest.mark.parametrize("fp8", [False, True], ids=["fp16", "e4m3"])
@pytest.mark.parametrize("d", [64, 96, 128, 256])
def test_few_rows_by_tiles_and_many_by_the_streaming_kernel(nfp, knobs, d, fp8):
    for tiles, lens, news in ((1, [1, 2, 15, 16, 17, 33, 64, 100, 257, 700], [1] * 10), (1, [0, 5, 2, 40], [3] * 4), (0, [90, 300], [90, 40])):
        knobs(attn_tiles=tiles)
        _check(nfp, lens, news, 8, 2, d, 16, fp8)


def test_rows_that_see_nothing(nfp):
    # lengths below the new tokens: the first rows see nothing and give zeros
    lens, news = [0, 50, 100], [60, 60, 60]
    cache, table, q = _case(lens, news, 4, 2, 128, 16, False)
    got = _run(nfp, cache, table, q, lens, news)
    ref, a = attention_ref(q, cache, table, lens, news, 4, 128 ** -0.5)
    assert_attention_close(got, ref, a)
    assert not got[:70].any() and got[70].any()


def test_an_entry_outside_the_cache_gives_nan_where_it_is_seen(nfp):
    lens, news = [200, 200], [100, 100]
    cache, table, q = _case(lens, news, 4, 2, 64, 16, False)
    ref, a = attention_ref(q, cache, table, lens, news, 4, 0.125)
    table[1, 9] = 1 << 30                                  # tokens 144 ... 159, new tokens 44 ... 59 of the second sequence
    got = _run(nfp, cache, table, q, lens, news)
    assert torch.isnan(got[144:]).all()
    assert_attention_close(got[:144], ref[:144], a[:144])


@pytest.mark.parametrize("fp8", [False, True], ids=["fp16", "e4m3"])
@pytest.mark.parametrize("d", [64, 96, 128, 256])
def test_a_value_that_is_not_finite_reaches_no_row_before_it(nfp, knobs, d, fp8):
    lens, news = [600, 600], [200, 200]
    cache, table, q = _case(lens, news, 4, 2, d, 32, fp8)
    ref, a = attention_ref(q, cache, table, lens, news, 4, d ** -0.5)
    for t in (450, 455):
        cache.v[table[1, t // 32], t % 32, 0, 7] = 0x7f if fp8 else np.float16(np.inf)
        cache.v[table[1, t // 32], t % 32, 1, d - 1] = 0xff if fp8 else np.float16(-np.inf)
    for chunk in (-1, 256):
        knobs(attn_chunk=chunk)
        got = _run(nfp, cache, table, q, lens, news)
        assert_attention_close(got[:250], ref[:250], a[:250])
        later = got[250:].float().cpu().numpy().reshape(-1, 4, d)
        hit = (lambda x, sign: np.isnan(x)) if fp8 else (lambda x, sign: x == sign * np.inf)
        assert hit(later[:, :2, 7], 1).all() and hit(later[:, 2:, d - 1], -1).all()
        later[:, :2, 7] = later[:, 2:, d - 1] = 0
        want = ref[250:].copy()
        want[:, :2, 7] = want[:, 2:, d - 1] = 0
        assert_attention_close(torch.from_numpy(later), want, a[250:])


def test_scores_that_grow_along_the_sequence(nfp):
    # every tile of tokens has larger scores than the one before: the sums are rescaled all the way
    lens, news, d = [900], [300], 128
    cache, table, q = _case(lens, news, 4, 1, d, 16, False)
    q[:] = np.abs(q)
    t = np.arange(900)
    cache.k[table[0, t // 16], t % 16, 0] = (np.abs(cache.k[table[0, t // 16], t % 16, 0]) * (t[:, None] / 900)).astype(np.float16)
    got = _run(nfp, cache, table, q, lens, news)
    ref, a = attention_ref(q, cache, table, lens, news, 4, d ** -0.5)
    assert_attention_close(got, ref, a)


def test_negative_scale(nfp):
    lens, news = [300], [120]
    cache, table, q = _case(lens, news, 4, 2, 64, 16, False)
    ref, a = attention_ref(q, cache, table, lens, news, 4, -0.3)
    assert_attention_close(_run(nfp, cache, table, q, lens, news, scale=-0.3), ref, a)
    ref, a = attention_ref(q, cache, table, lens, news, 4, 0.0)
    assert_attention_close(_run(nfp, cache, table, q, lens, news, scale=0.0), ref, a)


def test_strided_rows_and_the_same_bits_on_another_stream(nfp):
    lens, news, d = [400, 90], [200, 90], 128
    cache, table, q = _case(lens, news, 8, 2, d, 32, False)
    ref, a = attention_ref(q, cache, table, lens, news, 8, d ** -0.5)
    dev, td, ld = cache.to_device(nfp), _dev(table), _dev(np.asarray(lens, dtype=np.int32))
    starts = _dev(np.array([0, 200, 290], dtype=np.int32))
    wide = torch.full((290, 8 * d + 512), float("nan"), dtype=torch.float16, device="cuda:0")
    wide[:, 256:256 + 8 * d] = _dev(q)
    out = torch.zeros((290, 8 * d + 64), dtype=torch.float16, device="cuda:0")
    call = lambda o: nfp.paged_attention(wide[:, 256:256 + 8 * d], dev, td, ld, starts, max_new=200, max_len=400, out=o)
    call(out[:, 64:])
    assert_attention_close(out[:, 64:], ref, a)
    assert not out[:, :64].any()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        again = call(torch.empty((290, 8 * d), dtype=torch.float16, device="cuda:0"))
    side.synchronize()
    assert np.array_equal(bits(again), bits(out[:, 64:]))


@pytest.mark.parametrize("news", [1, 3, 40])
def test_a_bound_on_new_tokens_that_is_not_reached(nfp, news):
    # the launch is sized for chunks of 100 tokens, every sequence has fewer: each row is worked out once
    lens = [300, 77, news]
    cache, table, q = _case(lens, [news] * 3, 8, 2, 128, 32, False)
    ref, a = attention_ref(q, cache, table, lens, [news] * 3, 8, 128 ** -0.5)
    dev, td, ld = cache.to_device(nfp), _dev(table), _dev(np.asarray(lens, dtype=np.int32))
    first = nfp.paged_attention(_dev(q), dev, td, ld, max_new=100, max_len=300)
    assert_attention_close(first, ref, a)
    for _ in range(5):
        assert np.array_equal(bits(first), bits(nfp.paged_attention(_dev(q), dev, td, ld, max_new=100, max_len=300)))


@pytest.fixture(params=[4, 8])
def waves(nfp, request):
    nfp.tune("attn_waves", request.param)
    yield request.param
    nfp.tune("attn_waves", -1)


@pytest.mark.parametrize("fp8", [False, True], ids=["fp16", "e4m3"])
@pytest.mark.parametrize("d", [64, 96, 128, 256])
@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 17)])
@pytest.mark.parametrize("chunk", [-1, 256])
def test_both_heights_of_a_tile(nfp, knobs, waves, chunk, window, sinks, d, fp8):
    knobs(attn_chunk=chunk)
    _check(nfp, [1300, 333, 95, 270], [70, 1, 95, 260], 4, 2, d, 32, fp8, window, sinks, seed=2)


@pytest.mark.parametrize("fp8", [False, True], ids=["fp16", "e4m3"])
@pytest.mark.parametrize("d", [64, 96, 128, 256])
def test_parts_of_many_tiles(nfp, knobs, waves, d, fp8):
    # lengths that end in every part, tiles of one part among them
    knobs(attn_chunk=256)
    _check(nfp, [40 + 151 * i for i in range(10)], [40] * 10, 8, 8, d, 64, fp8, seed=3)


@pytest.mark.parametrize("fp8", [False, True], ids=["fp16", "e4m3"])
def test_values_that_are_not_finite_at_256_dims(nfp, waves, fp8):
    lens, news, d = [400, 400], [150, 150], 256
    cache, table, q = _case(lens, news, 4, 2, d, 32, fp8)
    ref, a = attention_ref(q, cache, table, lens, news, 4, d ** -0.5)
    cache.v[table[1, 340 // 32], 340 % 32, 1, d - 1] = 0xff if fp8 else np.float16(-np.inf)
    got = _run(nfp, cache, table, q, lens, news)
    assert_attention_close(got[:240], ref[:240], a[:240])
    later = got[240:].float().cpu().numpy().reshape(-1, 4, d)
    assert (np.isnan(later[:, 2:, d - 1]) if fp8 else later[:, 2:, d - 1] == -np.inf).all()
    later[:, 2:, d - 1] = 0
    want = ref[240:].copy()
    want[:, 2:, d - 1] = 0
    assert_attention_close(torch.from_numpy(later), want, a[240:])
