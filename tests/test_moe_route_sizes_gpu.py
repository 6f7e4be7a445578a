"""Routers of batches of changing sizes: one workspace for all of them."""
import pytest
import torch

import feed_forward_helpers as ff

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def nfp():
    from paper_2506_02024_amd import binding

    return binding


@pytest.mark.parametrize("E,most", [(256, 33), (128, 65), (64, 129), (40, 700), (300, 1000)])
def test_smaller_batches_on_the_workspace_of_the_largest(nfp, E, most):
    """Batches of any size up to the largest give on its workspace what they give on one of their own."""
    K, top_k = 2048, 6
    g = ff.generator(E)
    x, router = ff.normal(g, most, K), ff.normal(g, E, K, sigma=K ** -0.5)
    ws = nfp.new_workspace(nfp.moe_route_workspace_size(most, E, K), "cuda:0")
    for M in sorted({1, 15, 16, 17, 32, 33, 64, 65, 128, most - 1, most}):
        if M > most:
            continue
        for bias in (None, torch.zeros(E, device="cuda:0")):
            ids, weights = nfp.moe_route(x[:M], router, top_k, bias=bias, workspace=ws)
            ref = ff.route_ref(x[:M], router, top_k, False, True, bias, 1.0)
            assert torch.equal(ids.cpu(), ref[0])
            # one rounding to float32 (2^-24), and 64-bit sums, exponentials and quotients before it
            assert ((weights.cpu().double() - ref[1]).abs() <= ref[1] * (2.0 ** -24 + 1e-10) + 1e-44).all()
    assert (ws[:nfp.WORKSPACE_COUNTER_BYTES] == 0).all()


def test_mixture_of_batches_of_changing_sizes(nfp):
    """A mixture's workspace is asked for its largest batch once."""
    from paper_2506_02024_amd.decoder_layer import Mixture

    g = ff.generator(3)
    E, H, F = 256, 2048, 16
    mixture = Mixture(ff.normal(g, E, H, sigma=H ** -0.5), ff.normal(g, E, 2 * F, H, sigma=0.02), ff.normal(g, E, H, F, sigma=0.02), 1)
    x = ff.normal(g, 33, H)
    ws = nfp.new_workspace(mixture.workspace_size(33), "cuda:0")
    for M in (33, 32, 17, 1):
        assert torch.equal(mixture(x[:M], 0, None, ws), mixture(x[:M], 0, None, nfp.new_workspace(mixture.workspace_size(M), "cuda:0")))


@pytest.mark.parametrize("sigmoid,renormalize", [(False, True), (True, True), (True, False)])
@pytest.mark.parametrize("E,K,top_k", [(16, 48, 2), (64, 1040, 16), (128, 2048, 8), (256, 528, 32), (500, 4112, 7)])
def test_padding_among_many_tokens(nfp, E, K, top_k, sigmoid, renormalize):
    """Rows of zeros of either sign choose the first experts, which all tie; rows that hold no more than one number, or the smallest there are, choose by it."""
    M = (1 << 17) // E + 50
    g = ff.generator(E + K)
    x, router = ff.normal(g, M, K), ff.normal(g, E, K, sigma=K ** -0.5)
    x[1::3] = 0.0
    x[4::9] = -0.0
    x[2::7] = 0.0
    x[2::14, K - 1] = 2.0 ** -24
    x[9::14, 0] = -(2.0 ** -24)
    x[5::11] = torch.randint(-3, 4, x[5::11].shape, generator=g, device="cuda:0").half() * 2.0 ** -24
    zeros = (x == 0).all(1).cpu()
    assert M // 5 < int(zeros.sum()) < M
    ids, weights = nfp.moe_route(x, router, top_k, scoring="sigmoid" if sigmoid else "softmax", renormalize=renormalize)
    ref = ff.route_ref(x, router, top_k, sigmoid, renormalize, None, 1.0)
    assert torch.equal(ids.cpu(), ref[0])
    assert (ids.cpu()[zeros] == torch.arange(top_k, dtype=torch.int32)).all()
    # one rounding to float32 (2^-24), and 64-bit sums, exponentials and quotients before it
    assert ((weights.cpu().double() - ref[1]).abs() <= ref[1] * (2.0 ** -24 + 1e-10) + 1e-44).all()


def test_padding_with_a_row_of_the_router_that_is_not_finite(nfp):
    """0 times infinity is no number: an expert with one is chosen after all others, by rows of zeros too."""
    g = ff.generator(5)
    x, router = ff.normal(g, 2200, 256), ff.normal(g, 64, 256, sigma=0.05)
    x[::2] = 0.0
    router[2, 17], router[5, 3] = float("inf"), float("nan")
    ids, weights = nfp.moe_route(x, router, 8, scoring="sigmoid")
    assert (ids[::2].cpu() == torch.tensor([0, 1, 3, 4, 6, 7, 8, 9], dtype=torch.int32)).all() and (weights[::2] == 0.125).all()
    assert not (ids == 5).any()
