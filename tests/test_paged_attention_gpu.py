"""GPU: attention of new tokens over a paged cache against a plain form in 64 bits."""
import numpy as np
import pytest
import torch

from block_helpers import HostCache, assert_attention_close, attention_ref, page_table
from helpers import bits

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def nfp():
    from paper_2506_02024_amd import binding

    return binding


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda:0")


def _case(lens, news, heads, kv, d, page, fp8, seed=0, **kw):
    rng = np.random.default_rng(1000 + seed)
    pages = sum(-(-n // page) for n in lens) + 2
    cache = HostCache(pages, page, kv, d, fp8, seed)
    table = page_table(rng, lens, page, pages)
    # what no sequence holds: other pages, and the rest of the last ones
    held = np.zeros((pages, page), dtype=bool)
    for b, n in enumerate(lens):
        for t in range(n):
            held[table[b, t // page], t % page] = True
    for x in (cache.k, cache.v):
        x[~held] = 0x7f if fp8 else np.float16(np.nan)
    q = (rng.standard_normal((sum(news), heads * d)) * 1.4).astype(np.float16)
    return cache, table, q


def _run(nfp, cache, table, q, lens, news, **kw):
    uniform = len(set(news)) == 1 and not kw.pop("with_starts", False)
    starts = None if uniform else _dev(np.concatenate([[0], np.cumsum(news)]).astype(np.int32))
    return nfp.paged_attention(_dev(q), cache.to_device(nfp), _dev(table), _dev(np.asarray(lens, dtype=np.int32)), starts=starts,
                               max_new=max(news), max_len=max(max(lens), 1), **kw)


def _check(nfp, lens, news, heads, kv, d, page, fp8, window=0, sinks=0, seed=0, scale=None, **kw):
    cache, table, q = _case(lens, news, heads, kv, d, page, fp8, seed)
    got = _run(nfp, cache, table, q, lens, news, window=window, sinks=sinks, scale=scale, **kw)
    ref, a = attention_ref(q, cache, table, lens, news, heads, d ** -0.5 if scale is None else scale, window, sinks)
    assert_attention_close(got, ref, a, "%r" % ((lens, news, heads, kv, d, page, fp8, window, sinks),))
    return got


@pytest.fixture
def chunks_of(nfp):
    """Sets how many tokens of the cache a workgroup takes."""
    def pin(tokens):
        nfp.tune("attn_chunk", tokens)
    yield pin
    nfp.tune("attn_chunk", -1)


LENS = [1, 2, 15, 16, 17, 31, 33, 64, 100, 129, 257, 700]


@pytest.mark.parametrize("fp8", [False, True], ids=["fp16", "e4m3"])
@pytest.mark.parametrize("d", [64, 96, 128, 256])
@pytest.mark.parametrize("heads,kv,page", [(4, 1, 16), (6, 2, 64)])
def test_one_token_per_sequence(nfp, heads, kv, page, d, fp8):
    _check(nfp, LENS, [1] * len(LENS), heads, kv, d, page, fp8)


@pytest.mark.parametrize("fp8", [False, True], ids=["fp16", "e4m3"])
@pytest.mark.parametrize("heads,kv,news", [(16, 1, 1), (20, 1, 1), (71, 1, 1), (3, 3, 1), (14, 2, 5), (8, 2, 4), (40, 10, 3), (2, 2, 17)])
def test_groups_and_drafted_tokens(nfp, heads, kv, news, fp8):
    _check(nfp, [news, 30, 300, news + 1], [news] * 4, heads, kv, 128, 32, fp8, seed=heads)


@pytest.mark.parametrize("fp8", [False, True], ids=["fp16", "e4m3"])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_pages(nfp, page, fp8):
    _check(nfp, [1, page - 1, page, page + 1, 3 * page + 7], [1] * 5, 4, 2, 64, page, fp8)


@pytest.mark.parametrize("fp8", [False, True], ids=["fp16", "e4m3"])
@pytest.mark.parametrize("d", [64, 96, 128, 256])
@pytest.mark.parametrize("news", [1, 3])
def test_sequences_split_over_workgroups(nfp, chunks_of, news, d, fp8):
    lens = [3, 127, 128, 129, 500, 1000, 2049]
    cache, table, q = _case(lens, [news] * len(lens), 8, 2, d, 64, fp8, 5)
    ref, a = attention_ref(q, cache, table, lens, [news] * len(lens), 8, d ** -0.5)
    for tokens in (128, 384, 100000):
        chunks_of(tokens)
        for _ in range(2):                             # (the counters are left as they were found)
            assert_attention_close(_run(nfp, cache, table, q, lens, [news] * len(lens)), ref, a, "%d tokens per workgroup" % tokens)


@pytest.mark.parametrize("fp8", [False, True], ids=["fp16", "e4m3"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 4), (100, 0), (100, 17), (64, 64), (250, 1000), (5000, 4)])
@pytest.mark.parametrize("news", [1, 4])
def test_window_and_sinks(nfp, chunks_of, window, sinks, news, fp8):
    lens = [news, 20, 99, 116, 117, 400, 777]
    for tokens in (-1, 128):
        chunks_of(tokens)
        _check(nfp, lens, [news] * len(lens), 8, 2, 128, 16, fp8, window, sinks)


@pytest.mark.parametrize("fp8", [False, True], ids=["fp16", "e4m3"])
def test_pages_outside_the_window_are_not_read(nfp, fp8):
    # their entries are gone, and other sequences' pages hold NaN: see _case
    lens, window, sinks = [500, 333], 64, 5
    cache, table, q = _case(lens, [1, 1], 4, 2, 128, 16, fp8)
    ref, a = attention_ref(q, cache, table, lens, [1, 1], 4, 128 ** -0.5, window, sinks)
    for b, n in enumerate(lens):
        gone = table[b, 1:(n - window) // 16].copy()
        cache.k[gone], cache.v[gone] = (0x7f, 0x7f) if fp8 else (np.float16(np.nan), np.float16(np.inf))
        table[b, 1:(n - window) // 16] = [-1, 2 ** 31 - 1, 10 ** 6][b]
    assert_attention_close(_run(nfp, cache, table, q, lens, [1, 1], window=window, sinks=sinks), ref, a)


def test_an_entry_outside_the_cache_gives_nan_where_it_is_seen(nfp):
    lens = [100, 100, 100]
    cache, table, q = _case(lens, [1, 1, 1], 4, 2, 64, 16, False)
    ref, a = attention_ref(q, cache, table, lens, [1, 1, 1], 4, 0.125)
    table[1, 3] = -1
    got = _run(nfp, cache, table, q, lens, [1, 1, 1])
    assert torch.isnan(got[1]).all()
    assert_attention_close(got[[0, 2]], ref[[0, 2]], a[[0, 2]])
    table[1, 3] = cache.shape[0]
    assert torch.isnan(_run(nfp, cache, table, q, lens, [1, 1, 1])[1]).all()


def test_sequences_without_tokens_and_rows_that_see_nothing(nfp):
    lens, news = [0, 5, 2, 40], [3, 3, 3, 3]           # (lengths below the new tokens: the first of these see nothing)
    for with_starts in (False, True):
        got = _check(nfp, lens, news, 4, 1, 64, 16, False, with_starts=with_starts)
        assert not got[:3].any() and not got[6].any() and got[7].any()


def test_ragged_new_tokens(nfp):
    news = [1, 0, 5, 2, 0, 1, 40]
    lens = [300, 17, 5, 64, 0, 1, 90]
    for fp8 in (False, True):
        _check(nfp, lens, news, 8, 2, 128, 16, fp8)


def test_starts_and_lengths_outside_their_arrays_are_cut_off(nfp):
    lens, news = [50, 60], [2, 2]
    cache, table, q = _case(lens, news, 4, 2, 64, 16, False)
    dev = cache.to_device(nfp)
    for starts, ls in (([0, 2, 400], lens), ([-5, 2, 4], lens), ([0, 2, 4], [-3, 1 << 30]), ([3, 1, 2], lens)):
        got = nfp.paged_attention(_dev(q), dev, _dev(table), _dev(np.asarray(ls, dtype=np.int32)), _dev(np.asarray(starts, dtype=np.int32)),
                                  max_new=2, max_len=60)
        torch.cuda.synchronize()
        assert got.shape == (4, 256)


def test_longer_sequences_than_the_launch_was_sized_for(nfp, chunks_of):
    lens = [1000, 30, 600]
    cache, table, q = _case(lens, [1] * 3, 4, 2, 128, 16, False)
    ref, a = attention_ref(q, cache, table, lens, [1] * 3, 4, 128 ** -0.5)
    chunks_of(128)
    for most in (1, 200, 1000):
        got = nfp.paged_attention(_dev(q), cache.to_device(nfp), _dev(table), _dev(np.asarray(lens, dtype=np.int32)), max_len=most)
        assert_attention_close(got, ref, a)


def test_strided_rows(nfp):
    lens, d = [77, 5, 200], 128
    cache, table, q = _case(lens, [1] * 3, 8, 2, d, 32, False)
    ref, a = attention_ref(q, cache, table, lens, [1] * 3, 8, d ** -0.5)
    wide = torch.full((3, 8 * d + 512), float("nan"), dtype=torch.float16, device="cuda:0")
    wide[:, 256:256 + 8 * d] = _dev(q)
    out = torch.zeros((3, 8 * d + 64), dtype=torch.float16, device="cuda:0")
    tab = torch.full((3, table.shape[1] + 5), -7, dtype=torch.int32, device="cuda:0")
    tab[:, :table.shape[1]] = _dev(table)
    nfp.paged_attention(wide[:, 256:256 + 8 * d], cache.to_device(nfp), tab[:, :table.shape[1]], _dev(np.asarray(lens, dtype=np.int32)),
                        out=out[:, 64:])
    assert_attention_close(out[:, 64:], ref, a)
    assert not out[:, :64].any()


@pytest.mark.parametrize("scale", [0.0, 3.0, -0.2])
def test_scales(nfp, scale):
    _check(nfp, [5, 130, 300], [1] * 3, 4, 2, 64, 16, False, scale=scale)


def test_scores_far_from_zero(nfp):
    # one key that outweighs all others, at either end; scores of some thousands
    for place in (0, 299):
        lens = [300]
        cache, table, q = _case(lens, [1], 4, 1, 64, 16, False)
        q *= np.float16(20)
        cache.k[table[0, place // 16], place % 16] *= np.float16(20)
        ref, a = attention_ref(q, cache, table, lens, [1], 4, 1.0)
        # scores up to about 2^13 in 32 bits are 2^-10 off, and so may probabilities be
        got = _run(nfp, cache, table, q, lens, [1], scale=1.0).cpu().numpy().astype(np.float64).reshape(ref.shape)
        assert np.all(np.abs(got - ref) <= 2.0 ** -11 * np.abs(ref) + 2.0 ** -7 * a + 2.0 ** -24)


def test_an_infinite_or_nan_value_that_is_seen_stays_in_its_sequence(nfp):
    lens = [60, 60, 60]
    cache, table, q = _case(lens, [1] * 3, 4, 2, 64, 16, False)
    ref, a = attention_ref(q, cache, table, lens, [1] * 3, 4, 0.125)
    cache.v[table[1, 1], 3, 0, 5] = np.inf
    cache.v[table[1, 2], 3, 1, 6] = np.nan
    got = _run(nfp, cache, table, q, lens, [1] * 3)
    mid = got[1].float().cpu().numpy().reshape(4, 64)
    assert np.all(np.isposinf(mid[:2, 5])) and np.all(np.isnan(mid[2:, 6]))
    assert np.isfinite(np.delete(mid[:2], 5, 1)).all() and np.isfinite(np.delete(mid[2:], 6, 1)).all()
    assert_attention_close(got[[0, 2]], ref[[0, 2]], a[[0, 2]])


def test_the_same_bits_every_time_and_on_another_stream(nfp):
    lens = [4000, 100, 2500]
    cache, table, q = _case(lens, [1] * 3, 8, 2, 128, 16, False)
    first = bits(_run(nfp, cache, table, q, lens, [1] * 3))
    side = torch.cuda.Stream()
    for _ in range(3):
        assert np.array_equal(first, bits(_run(nfp, cache, table, q, lens, [1] * 3)))
        with torch.cuda.stream(side):
            assert np.array_equal(first, bits(_run(nfp, cache, table, q, lens, [1] * 3)))


def test_in_a_graph(nfp):
    lens = [4000, 100, 2500]
    cache, table, q = _case(lens, [1] * 3, 8, 2, 128, 16, False)
    dev, qd, td, ld = cache.to_device(nfp), _dev(q), _dev(table), _dev(np.asarray(lens, dtype=np.int32))
    out = torch.zeros((3, 8 * 128), dtype=torch.float16, device="cuda:0")
    ws = nfp.new_workspace(nfp.paged_attention_workspace_size(3, 8, dev, 3, max_new=1, max_len=4000), "cuda:0")
    call = lambda: nfp.paged_attention(qd, dev, td, ld, max_len=4000, out=out, workspace=ws)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for step in range(4):
        ld.copy_(_dev(np.asarray([n - 7 * step for n in lens], dtype=np.int32)))       # (a graph is replayed as sequences grow)
        graph.replay()
        got = bits(out).copy()
        call()
        assert np.array_equal(got, bits(out)), step


def test_refusals(nfp):
    lens = [1000, 30]
    cache, table, q = _case(lens, [1, 1], 4, 2, 64, 16, False)
    dev, qd, td, ld = cache.to_device(nfp), _dev(q), _dev(table), _dev(np.asarray(lens, dtype=np.int32))
    ws = nfp.new_workspace(16384, "cuda:0")
    with pytest.raises(nfp.NestedFPError) as e:
        nfp.paged_attention(qd, dev, td, ld, workspace=ws)
    assert e.value.status == nfp.ERR_WORKSPACE
    for bad in (dict(window=-1), dict(sinks=-2), dict(scale=float("nan")), dict(max_new=0)):
        with pytest.raises(nfp.NestedFPError) as e:
            nfp.paged_attention(qd, dev, td, ld, **bad)
        assert e.value.status == nfp.ERR_ARG
    with pytest.raises(ValueError):
        nfp.paged_attention(qd.float(), dev, td, ld)
    with pytest.raises(ValueError):
        nfp.paged_attention(qd, dev, td.long(), ld)
    with pytest.raises(ValueError):
        nfp.paged_attention(qd, dev, td, ld.long())
    with pytest.raises(ValueError):
        nfp.KVCache(2, 24, 2, 64, device="cuda:0")
    with pytest.raises(ValueError):
        nfp.KVCache(2, 16, 2, 80, device="cuda:0")


@pytest.mark.parametrize("fp8", [False, True], ids=["fp16", "e4m3"])
@pytest.mark.parametrize("news", [4, 60])
def test_a_value_that_is_not_finite_reaches_no_row_before_it(nfp, news, fp8):
    # the third of the new tokens has overflowed: the first two do not see it, the others do
    lens = [300, 300]
    cache, table, q = _case(lens, [news] * 2, 4, 2, 128, 32, fp8)
    ref, a = attention_ref(q, cache, table, lens, [news] * 2, 4, 128 ** -0.5)
    t = 300 - news + 2
    at = table[1, t // 32], t % 32
    cache.v[at[0], at[1], 0, 7] = 0x7f if fp8 else np.float16(np.inf)
    cache.v[at[0], at[1], 1, 9] = 0xff if fp8 else np.float16(-np.inf)
    got = _run(nfp, cache, table, q, lens, [news] * 2)
    assert_attention_close(got[:news + 2], ref[:news + 2], a[:news + 2])
    later = got[news + 2:].float().cpu().numpy().reshape(-1, 4, 128)
    hit = (lambda x, sign: np.isnan(x)) if fp8 else (lambda x, sign: x == sign * np.inf)
    assert hit(later[:, :2, 7], 1).all() and hit(later[:, 2:, 9], -1).all()
    later[:, :2, 7] = later[:, 2:, 9] = 0
    assert np.isfinite(later).all()
    # ... nor one whose own key is not finite
    cache.k[at[0], at[1], :, 3] = 0x7f if fp8 else np.float16(np.nan)
    got = _run(nfp, cache, table, q, lens, [news] * 2)
    assert_attention_close(got[:news + 2], ref[:news + 2], a[:news + 2])
    assert torch.isnan(got[news + 2:]).all()
