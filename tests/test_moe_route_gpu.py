"""The router of a mixture of experts against 64 bits: the same experts in the same order, weights rounded once."""
import pytest
import torch

import feed_forward_helpers as ff

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def nfp():
    from paper_2506_02024_amd import binding

    return binding


def compare(got, ref):
    ids, weights = got
    assert torch.equal(ids.cpu(), ref[0])
    # one rounding to float32 (2^-24), and 64-bit sums, exponentials and quotients before it
    w = ref[1]
    assert ((weights.cpu().double() - w).abs() <= w.abs() * (2.0 ** -24 + 1e-10) + 1e-44).all()


@pytest.mark.parametrize("M,E,K,top_k", [(1, 1, 16, 1), (1, 8, 1040, 2), (1, 128, 2048, 8), (2, 5, 48, 5), (16, 64, 512, 6), (17, 60, 272, 4), (33, 160, 7168, 6),
                                         (64, 256, 1024, 8), (100, 512, 256, 32), (1000, 65, 528, 3), (5000, 16, 64, 2)])
@pytest.mark.parametrize("sigmoid,with_bias,renormalize", [(False, False, True), (True, True, True), (False, True, False), (True, False, False)])
def test_route(nfp, M, E, K, top_k, sigmoid, with_bias, renormalize):
    g = ff.generator(M + E)
    x, router = ff.normal(g, M, K), ff.normal(g, E, K, sigma=K ** -0.5)
    bias = 0.2 * torch.randn(E, generator=g, device="cuda:0") if with_bias else None
    got = nfp.moe_route(x, router, top_k, scoring="sigmoid" if sigmoid else "softmax", renormalize=renormalize, bias=bias, factor=2.5)
    compare(got, ff.route_ref(x, router, top_k, sigmoid, renormalize, bias, 2.5))


def test_ties_go_to_the_lowest_index(nfp):
    g = ff.generator(1)
    x = ff.normal(g, 20, 256)
    one = ff.normal(g, 1, 256)
    for E in (7, 64, 130, 300):
        ids, weights = nfp.moe_route(x, one.expand(E, 256).contiguous(), 6)
        assert (ids.cpu() == torch.arange(6, dtype=torch.int32)).all()
        assert (weights == weights[:, :1]).all()
        ids, _ = nfp.moe_route(torch.zeros_like(x), ff.normal(g, E, 256) * torch.sign(torch.arange(E, device="cuda:0") - 2.5)[:, None].half(), 6)    # 0 and -0
        assert (ids.cpu() == torch.arange(6, dtype=torch.int32)).all()


def test_logits_that_differ_by_one_step_of_a_long_sum(nfp):
    """Two experts whose logits differ by 2^-24 of their size, which 32-bit sums do not see, stand in the right order."""
    K = 4096
    x = torch.ones((3, K), dtype=torch.float16, device="cuda:0")
    router = torch.full((6, K), 0.25, dtype=torch.float16, device="cuda:0")
    for e, k in ((4, 17), (2, 4000), (5, 1)):
        router[e, k] += 2.0 ** -12
    router[2, 9] += 2.0 ** -12
    ids, _ = nfp.moe_route(x, router, 6)
    assert ids.cpu().tolist() == [[2, 4, 5, 0, 1, 3]] * 3


def test_nan_and_infinity(nfp):
    g = ff.generator(2)
    x, router = ff.normal(g, 40, 512), ff.normal(g, 70, 512, sigma=0.05)
    clean = nfp.moe_route(x, router, 8)
    x2 = x.clone()
    x2[3, 5], x2[7, 100] = float("nan"), float("inf")
    ids, weights = nfp.moe_route(x2, router, 8)
    keep = torch.ones(40, dtype=torch.bool, device="cuda:0")
    keep[3], keep[7] = False, False
    assert torch.equal(ids[keep], clean[0][keep]) and torch.equal(weights[keep], clean[1][keep])
    for row in (3, 7):                                 # ids that can be used as indexes all the same
        got = ids[row].tolist()
        assert len(set(got)) == 8 and all(0 <= e < 70 for e in got)
    assert weights[3].isnan().all()
    r2 = router.clone()
    r2[11] = float("nan")                              # one expert's row: chosen after all others
    ids, _ = nfp.moe_route(x, r2, 32, scoring="sigmoid")
    assert not (ids == 11).any()
    ids, _ = nfp.moe_route(x[:4], r2[8:16].contiguous(), 8, scoring="sigmoid")
    assert (ids[:, 7] == 3).all()


def test_strides_graph_and_workspace(nfp):
    g = ff.generator(3)
    big, table = ff.normal(g, 50, 1024 + 8), ff.normal(g, 96, 1024 + 16, sigma=0.05)
    x, router = big[:, :1024], table[:, :1024]
    ws = nfp.new_workspace(nfp.moe_route_workspace_size(50, 96, 1024), "cuda:0")
    ids, weights = (torch.empty((50, 4), dtype=t, device="cuda:0") for t in (torch.int32, torch.float32))
    call = lambda: nfp.moe_route(x, router, 4, ids=ids, weights=weights, workspace=ws)
    call()
    compare((ids, weights), ff.route_ref(x, router, 4, False, True, None, 1.0))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(4):
        big.normal_(generator=g)
        graph.replay()
        torch.cuda.synchronize()
        compare((ids, weights), ff.route_ref(x, router, 4, False, True, None, 1.0))
        assert nfp.moe_route(torch.empty((0, 1024), dtype=torch.float16, device="cuda:0"), router, 4, workspace=ws)[0].shape == (0, 4)
    assert (ws[:nfp.WORKSPACE_COUNTER_BYTES] == 0).all()


def test_batches_of_several_launches(nfp):
    """More tokens than one launch takes (4 Mi logits)."""
    g = ff.generator(4)
    x, router = ff.normal(g, 9000, 64), ff.normal(g, 500, 64, sigma=0.2)
    assert nfp.moe_route_workspace_size(9000, 500, 64) <= (32 << 20) + nfp.WORKSPACE_COUNTER_BYTES
    compare(nfp.moe_route(x, router, 3), ff.route_ref(x, router, 3, False, True, None, 1.0))


# Many logits: those that may be among the largest are worked out in 64 bits after all of them in 32.

@pytest.mark.parametrize("M,E,K,top_k", [(8192, 16, 48, 2), (2100, 64, 272, 6), (1100, 160, 4112, 8), (600, 256, 7168, 32), (4100, 33, 16, 5), (300, 512, 1040, 1), (9000, 500, 64, 3)])
@pytest.mark.parametrize("sigmoid,with_bias,renormalize", [(False, False, True), (True, True, True), (True, True, False), (True, False, False)])
def test_many_logits(nfp, M, E, K, top_k, sigmoid, with_bias, renormalize):
    g = ff.generator(M + E)
    x, router = ff.normal(g, M, K), ff.normal(g, E, K, sigma=K ** -0.5)
    bias = 0.2 * torch.randn(E, generator=g, device="cuda:0") if with_bias else None
    got = nfp.moe_route(x, router, top_k, scoring="sigmoid" if sigmoid else "softmax", renormalize=renormalize, bias=bias, factor=2.5)
    compare(got, ff.route_ref(x, router, top_k, sigmoid, renormalize, bias, 2.5))


@pytest.mark.parametrize("places", [(0, 1), (2, 3), (4, 5), (6, 7)])
def test_many_logits_of_a_few_columns(nfp, places):
    """Every column counts for what a 32-bit sum may be off by: large sums that cancel, of some of each eight columns alone."""
    M, E, K, top_k = 1500, 128, 2048, 7
    g = ff.generator(8)
    some = torch.zeros(K, dtype=torch.bool, device="cuda:0")
    for p in places:
        some[p::8] = True
    x = torch.where(some, ((12.0 + ff.normal(g, M, K).float()) * 128).round() / 128, 0.0).half()          # multiples of 2^-7
    base = torch.where(torch.arange(K, device="cuda:0") < K // 2, 0.5, -0.5)
    router = (base + (ff.normal(g, E, K).float().round() * 2.0 ** -11)).half()                             # multiples of 2^-12: sums are exact in 64 bits
    compare(nfp.moe_route(x, router, top_k), ff.route_ref(x, router, top_k, False, True, None, 1.0))


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("kind", ["plain", "outliers", "cancelling"])
def test_many_logits_that_32_bits_cannot_tell_apart(nfp, sigmoid, kind):
    """Experts in groups of copies and near copies.  Tokens are multiples of 2^-8 and experts multiples of 2^-16, so that products are multiples of 2^-24 and their 64-bit sums exact, whatever
    their order (all below 2^29); 32-bit sums of the size 1 ... 2^12 are not."""
    M, E, K, top_k = 1500, 128, 2064, 7
    g = ff.generator(5)
    grid = lambda t, step: ((t.float() / step).round() * step).half()
    x = grid(ff.normal(g, M, K), 2.0 ** -8)
    base = grid(ff.normal(g, E // 4, K, sigma=0.02), 2.0 ** -16)
    router = base.repeat_interleave(4, 0)
    router[1::4, 100] = 2.0 ** -16                     # the first and third of each four are copies; the others differ in one place
    router[3::4, 2000] = -(2.0 ** -16)
    if kind == "outliers":
        x[:, 5], x[:, 1111] = 1024.0, -512.0
    if kind == "cancelling":                           # large sums that cancel
        x[:, :1024], x[:, 1024:2048] = 8.0 + x[:, :1024], 8.0 + x[:, 1024:2048]
        x = grid(x, 2.0 ** -8)
        router[:, :1024] += 0.5
        router[:, 1024:2048] -= 0.5
        router = grid(router, 2.0 ** -16)
    ref = ff.route_ref(x, router, top_k, sigmoid, True, None, 1.0)
    compare(nfp.moe_route(x, router, top_k, scoring="sigmoid" if sigmoid else "softmax"), ref)


def test_many_logits_nan_infinity_zero_and_masks(nfp):
    g = ff.generator(6)
    M, E, K, top_k = 1024, 160, 528, 8
    x, router = ff.normal(g, M, K), ff.normal(g, E, K, sigma=0.05)
    x[17] = 0.0
    x[1000:] = 0.0                                     # padding
    clean = nfp.moe_route(x, router, top_k)
    compare(clean, ff.route_ref(x, router, top_k, False, True, None, 1.0))
    x2 = x.clone()
    x2[3, 5], x2[7, 100], x2[1023, 527] = float("nan"), float("inf"), float("-inf")
    ids, weights = nfp.moe_route(x2, router, top_k)
    keep = torch.ones(M, dtype=torch.bool, device="cuda:0")
    keep[[3, 7, 1023]] = False
    assert torch.equal(ids[keep], clean[0][keep]) and torch.equal(weights[keep], clean[1][keep])
    for row in (3, 7, 1023):
        got = ids[row].tolist()
        assert len(set(got)) == top_k and all(0 <= e < E for e in got)
    assert weights[3].isnan().all()
    r2 = router.clone()
    r2[11] = float("nan")                              # chosen after all others; the others as without it
    ids, weights = nfp.moe_route(x, r2, top_k, scoring="sigmoid")
    others = [e for e in range(E) if e != 11]
    ref = ff.route_ref(x, router[others].contiguous(), top_k, True, True, None, 1.0)
    compare((ids, weights), (torch.tensor(others, dtype=torch.int32)[ref[0].long()], ref[1]))
    bias = 0.2 * torch.randn(E, generator=g, device="cuda:0")
    bias[:100] = float("-inf")
    bias[120] = 1e30
    compare(nfp.moe_route(x, router, top_k, scoring="sigmoid", bias=bias), ff.route_ref(x, router, top_k, True, True, bias, 1.0))
    bias[:] = float("-inf")                            # all but three masked
    bias[[40, 90, 159]] = 0.5
    compare(nfp.moe_route(x, router, top_k, scoring="sigmoid", bias=bias), ff.route_ref(x, router, top_k, True, True, bias, 1.0))


def test_many_logits_graph_and_strides(nfp):
    g = ff.generator(7)
    M, E, K = 777, 256, 1024
    big, table = ff.normal(g, M, K + 8), ff.normal(g, E, K + 16, sigma=0.05)
    x, router = big[:, :K], table[:, :K]
    ws = nfp.new_workspace(nfp.moe_route_workspace_size(M, E, K), "cuda:0")
    ids, weights = (torch.full((M + 1, 4), -7, dtype=t, device="cuda:0") for t in (torch.int32, torch.float32))
    big[5, K:], table[5, K:] = float("nan"), float("nan")              # between the rows
    call = lambda: nfp.moe_route(x, router, 4, ids=ids[:M], weights=weights[:M], workspace=ws)
    call()
    compare((ids[:M], weights[:M]), ff.route_ref(x, router, 4, False, True, None, 1.0))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(4):
        x.copy_(ff.normal(g, M, K))
        graph.replay()
        torch.cuda.synchronize()
        compare((ids[:M], weights[:M]), ff.route_ref(x, router, 4, False, True, None, 1.0))
        nfp.moe_route(x[:20], router, 4, workspace=ws)     # (the workspace of the other kind of call)
    assert (ws[:nfp.WORKSPACE_COUNTER_BYTES] == 0).all() and (ids[M] == -7).all() and (weights[M] == -7).all()
