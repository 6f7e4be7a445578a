"""Linears with an epilogue in FP8 mode: activations as codes, from quantize_act and from the norm, and with a scale that is known beforehand."""
import itertools

import pytest
import torch

import feed_forward_helpers as ff

pytestmark = pytest.mark.gpu

# streaming kernel that quantises itself and that is given codes, one token tile and several, tiled kernels unsplit and split
SHAPES = [(1, 512, 1024), (1, 260, 4112), (7, 2050, 528), (16, 514, 1280), (16, 1026, 4096), (50, 260, 528), (200, 258, 2064), (300, 514, 8208)]


@pytest.fixture(scope="module")
def nfp():
    from paper_2506_02024_amd import binding

    return binding


def inputs(M, N, K):
    g = ff.generator(M + N)
    return g, ff.normal(g, M, K), ff.normal(g, N, K, sigma=0.03), ff.normal(g, N, sigma=0.5)


def check(y, values, w, *epilogue):
    """Against 64 bits; values: what the codes and their scales stand for."""
    w = ff.upper_values(w)
    z, size = values @ w.t().contiguous(), values.abs() @ w.abs().t().contiguous()
    # (sums as in linear_ref: a step of the sum of magnitudes for each product, the scales and the last additions)
    ff.assert_within(y, *ff.epilogue_ref(z, (values.shape[1] + 4) * ff.STEP * size, *epilogue))


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_codes_give_what_their_activations_give(nfp, M, N, K, packed):
    g, x, w, b = inputs(M, N, K)
    layer = nfp.Layer(w, packed=packed)
    codes, scales = nfp.quantize_act(x)
    for gated in (False, True):
        r = ff.normal(g, M, N // 2 if gated else N)
        args = dict(bias=b, activation=nfp.ACT_SILU, gated=gated, residual=r)
        y = nfp.linear_fused(codes, layer, nfp.MODE_FP8, scales=scales, **args)
        assert torch.equal(y, nfp.linear_fused(x, layer, nfp.MODE_FP8, **args))
        check(y, ff.e4m3(codes) * scales.double()[:, None], w, b, 2, gated, r)


@pytest.mark.parametrize("M,N,K", SHAPES)
def test_codes_of_the_norm(nfp, M, N, K):
    """What the norm in front of a linear leaves, as a layer passes it on."""
    g, x, w, b = inputs(M, N, K)
    layer, weight = nfp.Layer(w), 1.0 + 0.1 * ff.normal(g, K)
    codes, scales = torch.empty((M, K), dtype=torch.uint8, device="cuda:0"), torch.empty(M, device="cuda:0")
    normed = torch.empty_like(x)
    nfp.add_rms_norm(x, weight, 1e-5, out=normed, Xq=codes, scales=scales)
    values = ff.e4m3(codes) * scales.double()[:, None]
    # (a code is half a step off at most: 2^-4 of the value, 2^-10 scales where it is subnormal; the norm's own roundings are far below)
    assert ((values - normed.double()).abs() <= normed.double().abs() * (2.0 ** -4 + 2.0 ** -10) + scales.double()[:, None] * 2.0 ** -10 * 1.01).all()
    for gated, act in itertools.product((False, True), (nfp.ACT_NONE, nfp.ACT_GELU)):
        y = nfp.linear_fused(codes, layer, nfp.MODE_FP8, bias=b, activation=act, gated=gated, scales=scales)
        check(y, values, w, b, act, gated, None)


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("scale", [2.0 ** -7, 0.003, 0.02])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_scale_that_is_known(nfp, M, N, K, scale, packed):
    """One scale for all tokens: the codes are those of x over the scale, limited to 448 (of 0.003, activations beyond 1.3)."""
    g, x, w, b = inputs(M, N, K)
    layer, given = nfp.Layer(w, packed=packed), torch.tensor([scale], dtype=torch.float32, device="cuda:0")
    codes = (x.float() / given).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
    assert scale != 0.003 or (codes.double().abs() == 448.0).any()
    for gated, act in ((False, nfp.ACT_NONE), (False, nfp.ACT_GELU), (True, nfp.ACT_SILU)):
        r = ff.normal(g, M, N // 2 if gated else N)
        y = nfp.linear_fused(x, layer, nfp.MODE_FP8, bias=b, activation=act, gated=gated, residual=r, act_scale=given)
        check(y, codes.double() * float(given), w, b, act, gated, r)
