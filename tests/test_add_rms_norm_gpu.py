"""GPU: residual addition, root-mean-square norm and its E4M3 codes against a plain form in 64 bits."""
import numpy as np
import pytest
import torch

from helpers import bits

pytestmark = pytest.mark.gpu
EPS = 1e-5


@pytest.fixture(scope="module")
def nfp():
    from paper_2506_02024_amd import binding

    return binding


def _inputs(M, K, seed=0):
    rng = np.random.default_rng(seed + M * 7919 + K)
    x = rng.standard_normal((M, K)).astype(np.float16)
    r = (rng.standard_normal((M, K)) * rng.uniform(0.3, 30.0, (M, 1))).astype(np.float16)
    w = (1 + 0.2 * rng.standard_normal(K)).astype(np.float16)
    return x, r, w


def _ref(h, w, eps=EPS):
    h = h.astype(np.float64)
    return h / np.sqrt((h ** 2).mean(axis=1, keepdims=True) + eps) * w.astype(np.float64)


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda:0")


def _close(y, ref):
    # FP16 output: half a unit; and the 32-bit sum of squares, root and products: 2^-18 covers K up to 2^21 (sums in parts)
    got = y.cpu().numpy().astype(np.float64)
    assert np.all(np.abs(got - ref) <= (2.0 ** -11 + 2.0 ** -18) * np.abs(ref) + 2.0 ** -24)


def _codes_close(Xq, scales, ref):
    amax = np.abs(ref).max(axis=1)
    scale = np.where(amax == 0, 1.0, amax / 448.0)
    got = scales.cpu().numpy().astype(np.float64)
    assert np.all(np.abs(got - scale) <= 2.0 ** -18 * scale)
    q = ref / scale[:, None]
    value = Xq.cpu().view(torch.float8_e4m3fn).double().numpy()
    # half a unit of E4M3 (3 bits: 2^-4 of the value; 2^-10 below its normal numbers), and what y and scale are off
    assert np.all(np.abs(value - q) <= (2.0 ** -4 + 2.0 ** -16) * np.abs(q) + 2.0 ** -10 * 1.001)


@pytest.mark.parametrize("M,K", [(1, 16), (1, 1040), (3, 4096), (7, 5120), (2, 8192), (3, 16384), (2, 32768), (2, 32784), (700, 2048), (1025, 528), (3000, 4096)])
def test_all_outputs(nfp, M, K):
    x, r, w = _inputs(M, K)
    h = (x.astype(np.float32) + r.astype(np.float32)).astype(np.float16)
    out, Xq = torch.empty((M, K), dtype=torch.float16, device="cuda:0"), torch.empty((M, K), dtype=torch.uint8, device="cuda:0")
    scales, total = torch.empty(M, dtype=torch.float32, device="cuda:0"), torch.empty_like(out)
    nfp.add_rms_norm(_dev(x), _dev(w), EPS, residual=_dev(r), sum_out=total, out=out, Xq=Xq, scales=scales)
    assert np.array_equal(bits(total), h.view(np.uint16))
    ref = _ref(h, w)
    _close(out, ref)
    _codes_close(Xq, scales, ref)
    # each output by itself, and the ones that nobody asked for: the same bits
    alone = nfp.add_rms_norm(_dev(x), _dev(w), EPS, residual=_dev(r))[0]
    assert np.array_equal(bits(alone), bits(out))
    Xq2, scales2 = torch.empty_like(Xq), torch.empty_like(scales)
    nfp.add_rms_norm(_dev(x), _dev(w), EPS, residual=_dev(r), Xq=Xq2, scales=scales2)
    assert torch.equal(Xq, Xq2) and torch.equal(scales, scales2)
    # the sum in place of the residual, and in place of X
    for target in ("residual", "x"):
        xd, rd = _dev(x), _dev(r)
        nfp.add_rms_norm(xd, _dev(w), EPS, residual=rd, sum_out=rd if target == "residual" else xd, out=out, Xq=Xq2, scales=scales2)
        assert np.array_equal(bits(rd if target == "residual" else xd), h.view(np.uint16))
        assert np.array_equal(bits(alone), bits(out)) and torch.equal(Xq, Xq2)


@pytest.mark.parametrize("M,K", [(5, 1040), (300, 4096), (2, 40000)])
def test_without_residual_and_strided(nfp, M, K):
    x, r, w = _inputs(M, K, 3)
    wide = torch.full((M, K + 48), float("nan"), dtype=torch.float16, device="cuda:0")
    wide[:, 16:16 + K] = _dev(x)
    out = torch.zeros((M, K + 24), dtype=torch.float16, device="cuda:0")
    nfp.add_rms_norm(wide[:, 16:16 + K], _dev(w), EPS, out=out[:, 8:8 + K])
    _close(out[:, 8:8 + K], _ref(x, w))
    assert not out[:, :8].any() and not out[:, 8 + K:].any()


def test_rows_of_zeros_and_extremes(nfp):
    K = 512
    x = np.zeros((5, K), dtype=np.float16)
    x[1] = 6e-8                                         # subnormal: eps decides
    x[2] = 65504
    x[3, 7] = 65504
    x[4, ::2] = -6e-8
    w = np.ones(K, dtype=np.float16)
    Xq, scales = torch.empty((5, K), dtype=torch.uint8, device="cuda:0"), torch.empty(5, dtype=torch.float32, device="cuda:0")
    for eps in (1e-5, 1.0, 1e-30):
        out, _, _, _ = nfp.add_rms_norm(_dev(x), _dev(w), eps, out=torch.empty((5, K), dtype=torch.float16, device="cuda:0"), Xq=Xq, scales=scales)
        ref = _ref(x, w, eps)
        _close(out, ref)
        _codes_close(Xq, scales, ref)
        assert scales[0] == 1.0 and not Xq[0].any()


def test_an_overflow_stays_in_its_row(nfp):
    x, r, w = _inputs(4, 256)
    x[1, 9], r[1, 9] = 60000, 60000
    x[2, 3] = np.nan
    total = torch.empty((4, 256), dtype=torch.float16, device="cuda:0")
    y = nfp.add_rms_norm(_dev(x), _dev(w), EPS, residual=_dev(r), sum_out=total)[0]
    assert torch.isinf(total[1, 9]) and torch.isnan(y[1, 9]) and torch.isnan(y[2]).all()
    h = (x.astype(np.float32) + r.astype(np.float32)).astype(np.float16)
    _close(y[[0, 3]], _ref(h[[0, 3]], w))


def test_codes_feed_the_linear(nfp):
    from paper_2506_02024_amd import workloads

    M, K, N = 33, 1040, 304
    x, r, w = _inputs(M, K, 5)
    W = workloads.weight_host(N, K, seed=2)
    up, _ = nfp.decompose(_dev(W))
    Xq, scales = torch.empty((M, K), dtype=torch.uint8, device="cuda:0"), torch.empty(M, dtype=torch.float32, device="cuda:0")
    nfp.add_rms_norm(_dev(x), _dev(w), EPS, residual=_dev(r), Xq=Xq, scales=scales)
    y = nfp.gemm_fp8_prequantized(Xq, scales, up)
    a = Xq.cpu().view(torch.float8_e4m3fn).double().numpy() * scales.cpu().numpy().astype(np.float64)[:, None]
    b = up.cpu().view(torch.float8_e4m3fn).double().numpy() / 256.0
    ref = a @ b.T
    assert np.linalg.norm(y.cpu().numpy().astype(np.float64) - ref) <= 1e-3 * np.linalg.norm(ref)


def test_refusals(nfp):
    x = torch.zeros((4, 64), dtype=torch.float16, device="cuda:0")
    w = torch.ones(64, dtype=torch.float16, device="cuda:0")
    for eps in (-1.0, float("nan"), float("inf")):
        with pytest.raises(nfp.NestedFPError) as e:
            nfp.add_rms_norm(x, w, eps)
        assert e.value.status == nfp.ERR_ARG
    with pytest.raises(nfp.NestedFPError) as e:
        nfp.add_rms_norm(x[:, :40], torch.ones(40, dtype=torch.float16, device="cuda:0"))
    assert e.value.status == nfp.ERR_SHAPE
    with pytest.raises(nfp.NestedFPError) as e:
        nfp.add_rms_norm(x[:, 4:36], w[:32].clone())     # rows that do not start on 16 bytes
    assert e.value.status == nfp.ERR_SHAPE
    for bad in (dict(residual=x.float()), dict(out=x[:3]), dict(Xq=torch.empty((4, 64), dtype=torch.uint8, device="cuda:0"))):
        with pytest.raises(ValueError):
            nfp.add_rms_norm(x, w, **bad)
    with pytest.raises(ValueError):
        nfp.add_rms_norm(x, w[:32])
    assert nfp.add_rms_norm(x[:0], w)[0].shape == (0, 64)
