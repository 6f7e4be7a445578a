"""The activated products between the experts' two launches: what their two FP16 terms keep, seen apart from the rounding of the outputs."""
import pytest
import torch

import feed_forward_helpers as ff

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def nfp():
    from paper_2506_02024_amd import binding

    return binding


# every number of token tiles, one pass over K and several, units of two and of four tiles, sums in the second launch and in a third
SHAPES = [(1, 8, 1040, 528, 2), (16, 10, 512, 128, 3), (5, 2, 4096, 64, 1), (3, 2, 160, 2064, 1), (30, 3, 272, 80, 2), (20, 2, 96, 2304, 2), (64, 2, 256, 128, 2), (64, 3, 112, 1120, 2),
          (8, 48, 1552, 2064, 6), (20, 8, 8208, 2064, 4)]


def choices(g, M, E, top_k):
    return torch.rand((M, E), generator=g, device="cuda:0").topk(top_k, 1).indices.to(torch.int32).contiguous()


@pytest.mark.parametrize("mode,exception", [(0, False), (1, False), (0, True)], ids=["fp16", "fp8", "exception"])
@pytest.mark.parametrize("M,E,H,F,top_k", SHAPES)
def test_products_of_any_size(nfp, M, E, H, F, top_k, mode, exception):
    """Activations of one column and down rows of one weight, so that every sum has one term and nothing but the activated products is rounded on the way; the residual takes away what the
    output's rounding would hide.

    The two terms are off by 2^-22 of the product, 2^-36 where the first is subnormal; the product, the two terms' sum and the sum over the choices and the residual are roundings to binary32
    of 2^-24 each.  (One term alone is off by 2^-11; two of which the second is subnormal by 2^-25 whatever the product.)"""
    g = ff.generator(M + H)
    value = ff.upper_values if mode == 1 and not exception else (lambda w: w.double())
    for size in (1.0, 2.0 ** -4, 2.0 ** -8, 2.0 ** -13, 2.0 ** -18):
        column = torch.randint(0, H, (M,), generator=g, device="cuda:0")
        x = torch.zeros((M, H), dtype=torch.float16, device="cuda:0")
        x[torch.arange(M, device="cuda:0"), column] = (1.0 + torch.rand((M,), generator=g, device="cuda:0")).half()
        # products of `size` to 16 times it: gate and up weights of the root of it each, divided between them
        gate_up = torch.empty((E, 2 * F, H), dtype=torch.float16, device="cuda:0").uniform_(0.5, 1.0, generator=g)
        gate_up[:, :F] *= size ** 0.5 if size > 2.0 ** -10 else 2.0 ** -5
        gate_up[:, F:] *= size ** 0.5 if size > 2.0 ** -10 else size * 2.0 ** 5
        pick = torch.arange(H, device="cuda:0") % F
        one = torch.empty((E, H), dtype=torch.float16, device="cuda:0").uniform_(0.5, 1.75, generator=g)
        if exception:
            one[E // 2, 3] = 2.5
        down = torch.zeros((E, H, F), dtype=torch.float16, device="cuda:0")
        down.scatter_(2, pick.expand(E, H)[:, :, None], one[:, :, None])
        ids = choices(g, M, E, top_k)
        share = (torch.rand((M, top_k), generator=g, device="cuda:0") + 0.5) / size
        experts = nfp.Experts(gate_up, down, nfp.ACT_NONE)
        assert experts.is_exception == exception
        y0, total, least = (torch.zeros((M, H), dtype=torch.float64, device="cuda:0") for _ in range(3))
        for m in range(M):
            for j in range(top_k):
                e, c = int(ids[m, j]), int(column[m])
                z = value(gate_up[e, :, c]) * float(x[m, c])
                part = float(share[m, j]) * value(one[e]) * (z[:F] * z[F:])[pick]
                y0[m] += part
                total[m] += part.abs()
                least[m] += float(share[m, j]) * value(one[e])
        residual = (-y0).half()
        y = nfp.moe(x, experts, ids, share, mode, residual=residual)
        ref = y0 + residual.double()
        tol = total * (2.0 ** -22 + (3 + top_k) * 2.0 ** -24) + least * 2.0 ** -36
        ff.assert_within(y, ref, tol + (ref.abs() + tol) * ff.HALF_STEP + ff.SUBNORMAL, "products of %g" % size)


@pytest.mark.parametrize("mode", [0, 1])
@pytest.mark.parametrize("size", [1.0, 2.0 ** -5, 2.0 ** -7])
@pytest.mark.parametrize("M,E,H,F,top_k", [(1, 8, 1040, 528, 2), (16, 10, 512, 128, 3), (5, 2, 4096, 64, 1), (48, 24, 1024, 272, 6), (64, 2, 256, 1120, 2)])
def test_errors_are_those_of_the_outputs_rounding(nfp, M, E, H, F, top_k, size, mode):
    """In shapes of use, the outputs' error is that of one rounding to float16 (about 2.1e-4 in the 2-norm).

    Whatever else is off adds up by its squares: 2 % more in all leave 0.2 roundings for it, 4e-5 or 2^-14.5.  Sums of 4096 products in binary32 are off by 2^-18 of their size in this
    norm (the root of as many roundings of 2^-24), the activation by 2^-17.  One FP16 term for the activated products is off by as much as the output's rounding: 41 % more."""
    g = ff.generator(M + F)
    x, gate_up, down = ff.normal(g, M, H, sigma=size), ff.normal(g, E, 2 * F, H, sigma=0.5 * H ** -0.5), ff.normal(g, E, H, F, sigma=0.25)
    ids, share = choices(g, M, E, top_k), (torch.rand((M, top_k), generator=g, device="cuda:0") + 0.5) / size ** 2
    y = nfp.moe(x, nfp.Experts(gate_up, down), ids, share, mode)
    ref, _ = ff.moe_ref(x, gate_up, down, ids, share, mode == 1, 2)
    rounding = (ref.half().double() - ref).norm()
    assert (y.double() - ref).norm() <= 1.02 * rounding
