"""A single row is contiguous whatever its stride: parts of wider tensors, as a program cuts them, are taken for one token."""
import pytest
import torch

import feed_forward_helpers as ff

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def nfp():
    from paper_2506_02024_amd import binding

    return binding


def test_choices_of_one_token(nfp):
    g = ff.generator(1)
    x, experts = ff.normal(g, 3, 128), nfp.Experts(ff.normal(g, 6, 64, 128, sigma=0.05), ff.normal(g, 6, 128, 32, sigma=0.05))
    ids, weights = torch.tensor([[4, 1, 0, 5]] * 3, dtype=torch.int32, device="cuda:0"), torch.rand((3, 4), generator=g, device="cuda:0")
    some, share = ids[:1, :2], weights[:1, :2]
    assert some.is_contiguous() and some.stride(0) == 4
    assert torch.equal(nfp.moe(x[:1], experts, some, share, 0), nfp.moe(x[:1], experts, some.clone(), share.clone(), 0))
    with pytest.raises(ValueError):                        # (of several tokens they have to be dense)
        nfp.moe(x, experts, ids[:, :2], weights[:, :2], 0)


def test_codes_of_one_token(nfp):
    g = ff.generator(2)
    layer = nfp.Layer(ff.normal(g, 64, 128, sigma=0.05))
    x, weight = ff.normal(g, 2, 128), torch.ones(128, dtype=torch.float16, device="cuda:0")
    wide, scales = torch.zeros((2, 256), dtype=torch.uint8, device="cuda:0"), torch.zeros(2, device="cuda:0")
    nfp.add_rms_norm(x[:1], weight, Xq=wide[:1, :128], scales=scales[:1])
    codes, s = torch.zeros((1, 128), dtype=torch.uint8, device="cuda:0"), torch.zeros(1, device="cuda:0")
    nfp.add_rms_norm(x[:1], weight, Xq=codes, scales=s)
    assert torch.equal(wide[:1, :128], codes) and (wide[:, 128:] == 0).all() and torch.equal(scales[:1], s)
    assert torch.equal(nfp.linear_fused(wide[:1, :128], layer, 1, scales=s), nfp.linear_fused(codes, layer, 1, scales=s))
    for call in (lambda: nfp.add_rms_norm(x, weight, Xq=wide[:, :128], scales=scales), lambda: nfp.linear_fused(wide[:, :128], layer, 1, scales=scales)):
        with pytest.raises(ValueError):
            call()


def test_angles_of_one_token(nfp):
    g = ff.generator(3)
    q, k, v = ff.normal(g, 1, 128), ff.normal(g, 1, 64), ff.normal(g, 1, 64)
    at = torch.tensor([3], dtype=torch.int32, device="cuda:0")
    wide = torch.rand((5, 96), generator=g, device="cuda:0")
    got = []
    for cos, sin in ((wide[:1, :32], wide[:1, 32:64]), (wide[:1, :32].clone(), wide[:1, 32:64].clone())):
        cache = nfp.KVCache(2, 16, 1, 64, device="cuda:0")
        cache.k.zero_()
        cache.v.zero_()
        got.append((nfp.rope_append(q, k, v, torch.zeros(1, dtype=torch.int32, device="cuda:0"), at, cache, cos, sin), cache.k.clone(), cache.v.clone()))
    assert all(torch.equal(a, b) for a, b in zip(*got))
    assert not torch.equal(got[0][0], q)
