"""The experts of a few tokens against 64 bits."""
import pytest
import torch

import feed_forward_helpers as ff

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def nfp():
    from paper_2506_02024_amd import binding

    return binding


def make(M, E, H, F, top_k, seed=0, exception=False):
    g = ff.generator(seed)
    gate_up, down = ff.normal(g, E, 2 * F, H, sigma=0.05), ff.normal(g, E, H, F, sigma=0.05)
    if exception:
        down[E // 2, 3, 5] = 3.0
    x, r = ff.normal(g, M, H), ff.normal(g, M, H)
    ids = torch.rand((M, E), generator=g, device="cuda:0").topk(top_k, 1).indices.to(torch.int32)
    weights = torch.rand((M, top_k), generator=g, device="cuda:0")
    return x, gate_up, down, ids.contiguous(), weights, r


@pytest.mark.parametrize("mode,exception", [(0, False), (1, False), (0, True), (1, True)])
@pytest.mark.parametrize("M,E,H,F,top_k", [(1, 1, 16, 16, 1), (1, 8, 1040, 528, 2), (1, 40, 256, 48, 8), (3, 4, 128, 272, 2), (16, 10, 512, 128, 3), (17, 4, 144, 64, 2),
                                           (30, 3, 272, 80, 2), (48, 24, 256, 96, 6), (64, 2, 256, 128, 2), (64, 60, 96, 32, 4), (33, 1, 64, 160, 1)])
def test_shapes(nfp, M, E, H, F, top_k, mode, exception):
    x, gate_up, down, ids, weights, r = make(M, E, H, F, top_k, seed=M + E, exception=exception)
    experts = nfp.Experts(gate_up, down)
    assert experts.is_exception == exception
    for residual in (None, r):
        y = nfp.moe(x, experts, ids, weights, mode, residual=residual)
        ref, tol = ff.moe_ref(x, gate_up, down, ids, weights, mode == 1 and not exception, 2, residual)
        ff.assert_within(y, ref, tol, str(residual is not None))


@pytest.mark.parametrize("M,H", [(5, 4096), (2, 4112), (1, 5120), (20, 2064), (40, 2304), (64, 1600)])
def test_long_rows(nfp, M, H):
    """Rows in one pass and in several, that start on lines and inside them, for every number of token tiles."""
    E = 2 if M != 40 else 12
    for mode, exception in ((0, False), (1, False), (0, True)):
        x, gate_up, down, ids, weights, r = make(M, E, H, 64, 2, seed=H, exception=exception)
        y = nfp.moe(x, nfp.Experts(gate_up, down), ids, weights, mode, residual=r)
        ref, tol = ff.moe_ref(x, gate_up, down, ids, weights, mode == 1, 2, r)
        ff.assert_within(y, ref, tol, str((mode, exception)))


@pytest.mark.parametrize("act", range(4))
def test_activations(nfp, act):
    x, gate_up, down, ids, weights, _ = make(6, 5, 96, 80, 2, seed=act)
    y = nfp.moe(x, nfp.Experts(gate_up, down, act), ids, weights, 0)
    ref, tol = ff.moe_ref(x, gate_up, down, ids, weights, False, act)
    ff.assert_within(y, ref, tol)


@pytest.mark.parametrize("M", [1, 7, 40, 64])
def test_ids_from_anywhere(nfp, M):
    """Ids outside the experts add nothing, one named twice counts with both weights, a token may have none at all, all tokens may choose one
    expert, and what lies in the workspace does not matter."""
    x, gate_up, down, ids, weights, r = make(M, 12, 128, 96, 4, seed=M)
    experts = nfp.Experts(gate_up, down)
    cases = {}
    cases["outside"] = ids.clone()
    cases["outside"][:, 1] = -1
    cases["outside"][::2, 2] = 12
    cases["outside"][0, 3] = 2 ** 31 - 1
    cases["twice"] = ids.clone()
    cases["twice"][:, 2] = cases["twice"][:, 0]
    cases["twice"][0, :] = 5
    cases["none"] = torch.full_like(ids, -7)
    cases["some have none"] = ids.clone()
    cases["some have none"][M // 2:] = -1
    cases["one expert"] = torch.full_like(ids, -1)
    cases["one expert"][:, 1] = 11
    cases["crowded"] = torch.randint(0, 2, ids.shape, generator=ff.generator(1), device="cuda:0", dtype=torch.int32)
    ws = nfp.new_workspace(nfp.moe_workspace_size(M, experts, 4), "cuda:0")
    for what, chosen in cases.items():
        for residual in (None, r):
            ws[nfp.WORKSPACE_COUNTER_BYTES:] = 0xff    # (NaN as float16)
            y = nfp.moe(x, experts, chosen, weights, 0, residual=residual, workspace=ws)
            ref, tol = ff.moe_ref(x, gate_up, down, chosen, weights, False, 2, residual)
            ff.assert_within(y, ref, tol, what)
    y = nfp.moe(x, experts, cases["none"], weights, 0, residual=r)
    assert torch.equal(y, r)


def test_nan_stays_with_its_token(nfp):
    for M in (5, 40):
        x, gate_up, down, ids, weights, r = make(M, 6, 128, 64, 2, seed=M)
        experts = nfp.Experts(gate_up, down)
        clean = nfp.moe(x, experts, ids, weights, 0, residual=r)
        x2, w2 = x.clone(), weights.clone()
        x2[1, 3], w2[2, 0], x2[4] = float("nan"), float("inf"), 60000.0
        y = nfp.moe(x2, experts, ids, w2, 0, residual=r)
        keep = torch.ones(M, dtype=torch.bool, device="cuda:0")
        keep[[1, 2, 4]] = False
        assert torch.equal(y[keep], clean[keep]) and y[1].isnan().all()


def test_strides_and_places(nfp):
    """Padded rows, outputs that start anywhere, results over the residual and over the activations."""
    for M in (4, 50):
        x, gate_up, down, ids, weights, r = make(M, 7, 256, 64, 3, seed=M)
        experts = nfp.Experts(gate_up, down)
        apart = nfp.moe(x, experts, ids, weights, 0, residual=r)
        wide = torch.zeros((M, 256 + 24), dtype=torch.float16, device="cuda:0")
        wide[:, :256] = x
        out, rr = torch.full((M, 261), 3.0, dtype=torch.float16, device="cuda:0"), torch.zeros((M, 259), dtype=torch.float16, device="cuda:0")
        rr[:, 2:258] = r
        nfp.moe(wide[:, :256], experts, ids, weights, 0, residual=rr[:, 2:258], out=out[:, 1:257])
        assert torch.equal(out[:, 1:257], apart) and (out[:, 0] == 3).all() and (out[:, 257:] == 3).all()
        r2, x2 = r.clone(), x.clone()
        assert torch.equal(nfp.moe(x, experts, ids, weights, 0, residual=r2, out=r2), apart)
        assert torch.equal(nfp.moe(x2, experts, ids, weights, 0, residual=r, out=x2), apart)


def test_many_experts(nfp):
    """As many experts as there may be, choices of 32."""
    x, gate_up, down, ids, weights, _ = make(64, 512, 32, 16, 32, seed=1)
    experts = nfp.Experts(gate_up, down)
    for M in (64, 20, 1):
        y = nfp.moe(x[:M], experts, ids[:M], weights[:M], 0)
        ref, tol = ff.moe_ref(x[:M], gate_up, down, ids[:M], weights[:M], False, 2)
        ff.assert_within(y, ref, tol, str(M))


def test_graph_of_router_and_experts(nfp):
    """Router, experts with a shared one as their residual, in a graph that is replayed with new activations; a second workspace for a second graph."""
    g = ff.generator(6)
    H, F, E, k, M = 256, 128, 16, 4, 12
    x, router = ff.normal(g, M, H), ff.normal(g, E, H, sigma=0.1)
    gate_up, down = ff.normal(g, E, 2 * F, H, sigma=0.05), ff.normal(g, E, H, F, sigma=0.05)
    shared_up, shared_down = ff.normal(g, 2 * F, H, sigma=0.05), ff.normal(g, H, F, sigma=0.05)
    experts, up, dn = nfp.Experts(gate_up, down), nfp.Layer(nfp.interleave_gate_up(shared_up)), nfp.Layer(shared_down)

    def layer(mode, ws):
        ids, weights = nfp.moe_route(x, router, k, workspace=ws)
        h = nfp.linear_fused(x, up, mode, activation=nfp.ACT_SILU, gated=True, workspace=ws)
        y = nfp.linear_fused(h, dn, mode, residual=x, workspace=ws)
        return ids, weights, nfp.moe(x, experts, ids, weights, mode, residual=y, out=y, workspace=ws)

    graphs = []
    for mode in (0, 1):
        need = max(nfp.moe_route_workspace_size(M, E, H), nfp.moe_workspace_size(M, experts, k), nfp.linear_fused_workspace_size(M, up, mode),
                   nfp.linear_fused_workspace_size(M, dn, mode))
        ws = nfp.new_workspace(need, "cuda:0")
        layer(mode, ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = layer(mode, ws)
        graphs.append((mode, ws, graph, out))
    for _ in range(3):
        x.normal_(generator=g)
        for mode, ws, graph, out in graphs:
            graph.replay()
            torch.cuda.synchronize()
            got = [t.clone() for t in out]
            for a, b in zip(got, layer(mode, nfp.new_workspace(ws.numel(), "cuda:0"))):
                assert torch.equal(a, b)
            ids, weights = ff.route_ref(x, router, k, False, True, None, 1.0)
            assert torch.equal(got[0].cpu(), ids)
            # the shared expert in two calls, whose products are rounded between them
            h, dh = ff.linear_ref(x, nfp.interleave_gate_up(shared_up), mode == 1, None, 2, True)
            if mode == 0:
                y, dy = ff.linear_ref(h.half(), shared_down, False, None, 0, False, x)
                dy = dy + dh @ shared_down.double().abs().t().contiguous() + (h - h.half().double()).abs() @ shared_down.double().abs().t().contiguous()
                ref, tol = ff.moe_ref(x, gate_up, down, got[0], got[1], False, 2, y.half())
                ff.assert_within(got[2], ref, tol + dy + (y - y.half().double()).abs())


@pytest.mark.parametrize("M,E,H,F,top_k", [(3, 2, 160, 2064, 1), (16, 6, 1040, 4112, 2), (20, 2, 96, 2304, 2), (64, 3, 112, 1120, 2), (64, 2, 48, 528, 2)])
def test_long_products(nfp, M, E, H, F, top_k):
    """Down products whose rows take one pass and several, for every number of token tiles, an odd number of row tiles among them."""
    for mode, exception in ((0, False), (1, False), (0, True)):
        x, gate_up, down, ids, weights, r = make(M, E, H, F, top_k, seed=F, exception=exception)
        y = nfp.moe(x, nfp.Experts(gate_up, down), ids, weights, mode, residual=r)
        ref, tol = ff.moe_ref(x, gate_up, down, ids, weights, mode == 1, 2, r)
        ff.assert_within(y, ref, tol, str((mode, exception)))


@pytest.mark.parametrize("M,E,H,F,top_k", [(8, 48, 1552, 2064, 6), (20, 8, 8208, 2064, 4), (16, 32, 4112, 1024, 4)])
def test_units_of_four_tiles(nfp, M, E, H, F, top_k):
    """Enough units in several passes: down products of many experts and of long outputs, up products of rows of 4112."""
    for mode in (0, 1):
        x, gate_up, down, ids, weights, _ = make(M, E, H, F, top_k, seed=H)
        y = nfp.moe(x, nfp.Experts(gate_up, down), ids, weights, mode)
        for rows in (slice(0, 1), slice(M - 1, M)):
            ref, tol = ff.moe_ref(x[rows], gate_up, down, ids[rows], weights[rows], mode == 1, 2)
            ff.assert_within(y[rows], ref, tol, str(mode))


def test_workspace_for_many_calls(nfp):
    """One workspace for calls of different shapes and for linears, one after the other: every call leaves the counters cleared."""
    calls = []
    for M, E, H, F, k in ((1, 8, 512, 64, 2), (16, 12, 1040, 128, 4), (40, 6, 272, 80, 2), (3, 2, 64, 2064, 1)):
        x, gate_up, down, ids, weights, r = make(M, E, H, F, k, seed=M)
        experts = nfp.Experts(gate_up, down)
        calls.append((x, experts, ids, weights, r, nfp.moe(x, experts, ids, weights, 0, residual=r)))
    layer, router = nfp.Layer(ff.normal(ff.generator(1), 512, 4096, sigma=0.02)), ff.normal(ff.generator(2), 40, 4096, sigma=0.02)
    z = ff.normal(ff.generator(3), 5, 4096)
    need = max([nfp.moe_workspace_size(c[0].shape[0], c[1], c[2].shape[1]) for c in calls] + [nfp.linear_fused_workspace_size(5, layer, 0),
                                                                                              nfp.moe_route_workspace_size(5, 40, 4096)])
    ws = nfp.new_workspace(need, "cuda:0")
    want, chosen = nfp.linear_fused(z, layer, 0, activation=nfp.ACT_GELU), nfp.moe_route(z, router, 3)
    for _ in range(3):
        for x, experts, ids, weights, r, y in calls:
            assert torch.equal(nfp.moe(x, experts, ids, weights, 0, residual=r, workspace=ws), y)
            assert torch.equal(nfp.linear_fused(z, layer, 0, activation=nfp.ACT_GELU, workspace=ws), want)
            assert all(torch.equal(a, b) for a, b in zip(nfp.moe_route(z, router, 3, workspace=ws), chosen))
            torch.cuda.synchronize()
            assert (ws[:nfp.WORKSPACE_COUNTER_BYTES] == 0).all()


def test_two_streams_at_once(nfp):
    """Routers (few and many tokens), experts and linears with an epilogue on two streams, each with a workspace of its own, give what they give alone."""
    g = ff.generator(21)
    experts = nfp.Experts(ff.normal(g, 24, 2 * 272, 1040, sigma=0.03), ff.normal(g, 24, 1040, 272, sigma=0.03))
    router, layer = ff.normal(g, 24, 1040, sigma=0.03), nfp.Layer(ff.normal(g, 2 * 528, 1040, sigma=0.03))
    wide = ff.normal(g, 128, 1040, sigma=0.03)
    few = [ff.normal(g, m, 1040) for m in (33, 48)]
    many = [ff.normal(g, m, 1040) for m in (1300, 2048)]
    need = max(nfp.moe_route_workspace_size(2048, 128, 1040), nfp.moe_workspace_size(48, experts, 4), nfp.linear_fused_workspace_size(2048, layer, nfp.MODE_FP8),
               nfp.linear_fused_workspace_size(2048, layer, nfp.MODE_FP16))

    def everything(i, mode, ws):
        ids, weights = nfp.moe_route(few[i], router, 4, workspace=ws)
        y = nfp.moe(few[i], experts, ids, weights, mode, residual=few[i], workspace=ws)
        more = nfp.moe_route(many[i], wide, 6, scoring="sigmoid", workspace=ws)
        z = nfp.linear_fused(many[i], layer, mode, activation=nfp.ACT_SILU, gated=True, workspace=ws)
        return (ids, weights, y, *more, z, nfp.linear_fused(few[i], layer, mode, activation=nfp.ACT_GELU, gated=True, workspace=ws))

    rooms = [nfp.new_workspace(need, "cuda:0") for _ in range(2)]
    alone = [everything(i, i, rooms[i]) for i in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = [[], []]
    for _ in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(everything(i, i, rooms[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for run in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(run, alone[i]))
        assert (rooms[i][:nfp.WORKSPACE_COUNTER_BYTES] == 0).all()


@pytest.mark.parametrize("M,E,H,F,top_k", [(16, 24, 1600, 800, 4), (7, 40, 2048, 528, 6), (1, 32, 1920, 1920, 32), (1, 3, 2064, 2064, 2), (33, 30, 1552, 1040, 5)])
def test_many_units_and_few(nfp, M, E, H, F, top_k):
    """Both lengths of a wave's slice, on either side of what chooses them."""
    for mode, exception in ((0, False), (1, False), (0, True)):
        x, gate_up, down, ids, weights, r = make(M, E, H, F, top_k, seed=F, exception=exception)
        y = nfp.moe(x, nfp.Experts(gate_up, down), ids, weights, mode, residual=r)
        ref, tol = ff.moe_ref(x, gate_up, down, ids, weights, mode == 1 and not exception, 2, r)
        ff.assert_within(y, ref, tol, str((mode, exception)))


@pytest.mark.parametrize("M,top_k", [(1, 8), (8, 4), (9, 4), (33, 2), (64, 6)])
def test_replays_on_a_workspace_that_holds_anything(nfp, M, top_k):
    """Few choices, which the down products' launch adds up, and more, which a launch of their own does: replayed with new choices, some of them outside the experts and some named twice,
    in place, with NaN in the workspace behind its counters."""
    E, H, F = 10, 208, 144
    x, gate_up, down, ids, weights, r = make(M, E, H, F, top_k, seed=M)
    experts, g = nfp.Experts(gate_up, down), ff.generator(M + 1)
    ws = nfp.new_workspace(nfp.moe_workspace_size(M, experts, top_k), "cuda:0")
    y = r.clone()
    call = lambda: nfp.moe(x, experts, ids, weights, 0, residual=y, out=y, workspace=ws)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for turn in range(5):
        ids.copy_(torch.randint(-2, E + 2, ids.shape, generator=g, device="cuda:0") if turn < 4 else torch.full_like(ids, -1))
        x.normal_(generator=g)
        y.copy_(r)
        ws[nfp.WORKSPACE_COUNTER_BYTES:] = 0xff
        graph.replay()
        torch.cuda.synchronize()
        ref, tol = ff.moe_ref(x, gate_up, down, ids, weights, False, 2, r)
        ff.assert_within(y, ref, tol, str(turn))
        assert (ws[:nfp.WORKSPACE_COUNTER_BYTES] == 0).all()
