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
