"""GPU: batches of more than 64, 128 and 256 sequences, and one workspace for many calls, whose counters each call leaves cleared."""
import numpy as np
import pytest
import torch

from block_helpers import assert_attention_close, attention_ref
from helpers import bits
from test_paged_attention_gpu import _case, _dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def nfp():
    from paper_2506_02024_amd import binding

    return binding


@pytest.fixture
def knobs(nfp):
    names = ("attn_chunk", "attn_groups", "attn_tiles", "attn_waves")

    def pin(**kw):
        for name in names:
            nfp.tune(name, kw.get(name, -1))
    yield pin
    pin()


class Call:
    """A call with a workspace of its own, for as many passes as are asked for."""

    def __init__(self, nfp, lens, news, heads, kv, d, page, fp8, starts=True, window=0, sinks=0, seed=0):
        self.nfp, self.lens, self.news, self.heads, self.window, self.sinks = nfp, lens, news, heads, window, sinks
        self.cache, self.table, self.q = _case(lens, news, heads, kv, d, page, fp8, seed)
        self.ref, self.a = attention_ref(self.q, self.cache, self.table, lens, news, heads, d ** -0.5, window, sinks)
        self.dev = self.cache.to_device(nfp)
        self.args = [_dev(self.table), _dev(np.asarray(lens, dtype=np.int32)),
                     _dev(np.concatenate([[0], np.cumsum(news)]).astype(np.int32)) if starts else None]
        self.qd = _dev(self.q)

    def workspace(self):
        size = self.nfp.paged_attention_workspace_size(len(self.q), self.heads, self.dev, len(self.lens), max_new=max(self.news), max_len=max(self.lens),
                                                       window=self.window, sinks=self.sinks)
        ws = self.nfp.new_workspace(size, "cuda:0")
        ws[self.nfp.WORKSPACE_COUNTER_BYTES:] = 0xff     # (sums that were not written are NaN)
        return ws

    def check(self, passes=3, workspace=None, what="", split=None):
        ws = self.workspace() if workspace is None else workspace
        if split is not None:
            assert (ws.numel() > self.nfp.WORKSPACE_COUNTER_BYTES) == split
        first = None
        for _ in range(passes):
            out = torch.full(self.qd.shape, float("nan"), dtype=torch.float16, device="cuda:0")
            self.nfp.paged_attention(self.qd, self.dev, *self.args, max_new=max(self.news), max_len=max(self.lens), window=self.window,
                                     sinks=self.sinks, out=out, workspace=ws)
            assert_attention_close(out, self.ref, self.a, what)
            if ws.numel() >= self.nfp.WORKSPACE_COUNTER_BYTES:
                assert not ws[:self.nfp.WORKSPACE_COUNTER_BYTES].any()
            first = bits(out) if first is None else first
            assert np.array_equal(first, bits(out))
        return ws


def _lens(batch, longest, seed):
    """Lengths with zeros, ones and a few long ones among them."""
    rng = np.random.default_rng(seed)
    lens = rng.integers(0, 60, batch)
    lens[rng.permutation(batch)[:5]] = longest - rng.integers(0, 40, 5)
    lens[[0, batch // 2, batch - 1]] = 0, 1, longest
    return [int(n) for n in lens]


@pytest.mark.parametrize("fp8", [False, True], ids=["fp16", "e4m3"])
@pytest.mark.parametrize("batch", [63, 64, 65, 127, 128, 129, 130, 192, 193, 255, 256])
def test_one_token_of_many_sequences(nfp, knobs, batch, fp8):
    call = Call(nfp, _lens(batch, 1500, batch), [1] * batch, 2, 1, 64, 16, fp8, starts=False, seed=batch)
    knobs()
    call.check()
    # parts of 128 tokens, shared out over few workgroups and over many
    for groups in (-1, 7, 300):
        knobs(attn_chunk=128, attn_groups=groups)
        call.check(what="%d workgroups" % groups, split=True)


@pytest.mark.parametrize("fp8", [False, True], ids=["fp16", "e4m3"])
@pytest.mark.parametrize("batch,news", [(70, 3), (200, 2), (257, 1), (300, 1), (300, 2)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (200, 20)])
def test_drafted_tokens_and_batches_without_a_schedule(nfp, knobs, window, sinks, batch, news, fp8):
    # more than 256 sequences: a workgroup for every part of every tile
    call = Call(nfp, _lens(batch, 1000, batch), [news] * batch, 4, 2, 64, 32, fp8, starts=False, window=window, sinks=sinks, seed=batch)
    knobs()
    call.check(passes=2)
    knobs(attn_chunk=128)
    call.check(split=True)


def _ragged(batch, seed):
    """New tokens: mostly one, some none, a few drafts; prompt chunks at the ends and around every 64th sequence."""
    rng = np.random.default_rng(seed)
    news = rng.choice([0, 1, 1, 1, 1, 5], batch)
    for at, n in ((2, 40), (62, 33), (63, 50), (64, 20), (65, 129), (batch // 2, 18), (batch - 2, 70), (batch - 1, 260)):
        if at < batch:
            news[at] = n
    lens = [int(n + c) for n, c in zip(news, rng.integers(0, 80, batch))]
    lens[63] += 700
    lens[-1] += 500
    return lens, [int(n) for n in news]


@pytest.mark.parametrize("fp8", [False, True], ids=["fp16", "e4m3"])
@pytest.mark.parametrize("batch", [66, 130, 256, 300])
def test_prompt_chunks_behind_many_sequences(nfp, knobs, batch, fp8):
    lens, news = _ragged(batch, batch)
    call = Call(nfp, lens, news, 4, 2, 64, 16, fp8, seed=batch)
    for kw in (dict(), dict(attn_waves=8), dict(attn_chunk=256), dict(attn_chunk=256, attn_waves=8), dict(attn_tiles=0), dict(attn_tiles=0, attn_chunk=128)):
        knobs(**kw)
        call.check(passes=2, what=str(kw))


@pytest.mark.parametrize("fp8", [False, True], ids=["fp16", "e4m3"])
def test_one_workspace_for_calls_of_many_shapes(nfp, knobs, fp8):
    calls = [Call(nfp, [700, 3, 1200], [1, 1, 1], 8, 2, 128, 32, fp8, starts=False), Call(nfp, [900, 400, 60], [70, 1, 60], 4, 2, 128, 16, fp8),
             Call(nfp, _lens(100, 800, 1), [1] * 100, 2, 1, 64, 16, fp8, starts=False)]
    knobs(attn_chunk=256)
    workspace = max((call.workspace() for call in calls), key=lambda ws: ws.numel())
    for _ in range(2):
        for call in calls:
            call.check(passes=2, workspace=workspace)
