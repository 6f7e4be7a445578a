"""CPU: linears with an epilogue, the router and the experts reject bad arguments before they touch a device."""
import ctypes

import pytest
import torch

OK, ARG, SHAPE, RANGE, WORKSPACE = 0, 1, 2, 3, 4
FAKE = 0x10000                                             # aligned, never dereferenced


class Epilogue(ctypes.Structure):
    _fields_ = [("bias", ctypes.c_void_p), ("residual", ctypes.c_void_p), ("ldr", ctypes.c_int64), ("activation", ctypes.c_int32), ("gated", ctypes.c_int32)]


@pytest.fixture(scope="module")
def nfp():
    from paper_2506_02024_amd import binding, build

    if build.is_stale():
        build.build_library()
    binding.lib()
    return binding


def test_linear_fused(nfp):
    def call(pre=False, X=FAKE, M=4, ldx=64, N=32, K=64, exception=0, layout=0, upper=FAKE, lower=FAKE, mode=0, bias=FAKE, res=FAKE, ldr=32, act=2, gated=0,
             epi=True, layer=True, Y=FAKE, ldy=32, ws=FAKE, bytes_=0, scales=FAKE):
        c = nfp._LayerStruct(N, K, exception, layout, upper, lower, FAKE, K, 0)
        e = Epilogue(bias, res, ldr, act, gated)
        layer_ref, epi_ref = ctypes.byref(c) if layer else None, ctypes.byref(e) if epi else None
        if pre:
            return nfp.lib().nestedfp_linear_fused_prequantized(X, scales, M, layer_ref, epi_ref, Y, ldy, ws, bytes_, None)
        return nfp.lib().nestedfp_linear_fused(X, M, ldx, layer_ref, mode, None, epi_ref, Y, ldy, ws, bytes_, None)

    assert call(M=0, X=0, Y=0) == OK and call(pre=True, M=0) == OK and call(N=0) == OK
    for bad in (dict(X=0), dict(Y=0), dict(upper=0), dict(lower=0), dict(epi=False), dict(layer=False), dict(mode=2), dict(act=4), dict(act=-1), dict(gated=2),
                dict(M=-1), dict(layout=3), dict(K=0)):
        assert call(**bad) == ARG, bad
    for bad in (dict(K=72, ldx=72), dict(ldx=56), dict(ldx=68), dict(X=FAKE + 8), dict(ldy=28), dict(ldr=28), dict(ldr=1 << 32), dict(res=FAKE + 1), dict(bias=FAKE + 1),
                dict(N=33, gated=1, ldy=64, ldr=64), dict(gated=1, ldy=12), dict(gated=1, ldr=12), dict(upper=FAKE + 8)):
        assert call(**bad) == SHAPE, bad
    assert call(pre=True, exception=1) == RANGE
    for bad in (dict(X=0), dict(scales=0), dict(upper=0), dict(Y=0), dict(epi=False), dict(layer=False), dict(act=9), dict(layout=2)):
        assert call(pre=True, **bad) == ARG, bad
    for bad in (dict(X=FAKE + 8), dict(scales=FAKE + 2), dict(ldy=31), dict(N=31, gated=1)):
        assert call(pre=True, **bad) == SHAPE, bad
    assert call(mode=1, M=40) == WORKSPACE


def test_moe_route(nfp):
    def call(X=FAKE, M=4, K=64, ldx=64, R=FAKE, E=8, ldr=64, k=2, scoring=0, factor=1.0, bias=None, ids=FAKE, w=FAKE, ws=FAKE, bytes_=1 << 20):
        return nfp.lib().nestedfp_moe_route(X, M, K, ldx, R, E, ldr, k, scoring, 1, factor, bias, ids, w, ws, bytes_, None)

    assert call(M=0, X=0) == OK
    for bad in (dict(X=0), dict(R=0), dict(ids=0), dict(w=0), dict(M=-1), dict(E=0), dict(K=0), dict(k=0), dict(scoring=2), dict(scoring=-1), dict(factor=float("nan")),
                dict(factor=float("inf"))):
        assert call(**bad) == ARG, bad
    for bad in (dict(E=513), dict(k=9), dict(E=64, k=33), dict(K=72, ldx=72, ldr=72), dict(ldx=56), dict(ldr=68), dict(X=FAKE + 8), dict(R=FAKE + 2), dict(ids=FAKE + 2),
                dict(w=FAKE + 2), dict(bias=FAKE + 2), dict(ldx=(1 << 21) + 8), dict(M=1 << 30)):
        assert call(**bad) == SHAPE, bad
    for bad in (dict(ws=0), dict(bytes_=16384), dict(ws=FAKE + 8)):
        assert call(**bad) == WORKSPACE, bad
    size = nfp.lib().nestedfp_moe_route_workspace_size
    assert size(0, 8, 64) == 0 and size(4, 0, 64) == 0 and size(4, 513, 64) == 0 and size(4, 8, 40) == 0
    for M in (1, 100, 16384, 1 << 20):
        for E in (1, 8, 129, 512):
            assert 16384 < size(M, E, 4096) <= 16384 + (32 << 20)


def test_moe(nfp):
    def call(X=FAKE, M=4, ldx=64, E=8, H=64, F=48, exception=0, act=2, up=FAKE, lo=FAKE, down=FAKE, dlo=FAKE, mode=0, ids=FAKE, w=FAKE, k=2, res=FAKE, ldr=64, Y=FAKE,
             ldy=64, ws=FAKE, bytes_=1 << 20, experts=True):
        c = nfp._ExpertsStruct(E, H, F, exception, act, up, lo, down, dlo)
        return nfp.lib().nestedfp_moe(X, M, ldx, ctypes.byref(c) if experts else None, mode, ids, w, k, res, ldr, Y, ldy, ws, bytes_, None)

    assert call(M=0, X=0, Y=0) == OK
    for bad in (dict(X=0), dict(Y=0), dict(ids=0), dict(w=0), dict(up=0), dict(down=0), dict(lo=0), dict(dlo=0), dict(experts=False), dict(E=0), dict(H=0), dict(F=-16), dict(M=-1),
                dict(k=0), dict(mode=2), dict(act=4), dict(act=-1)):
        assert call(**bad) == ARG, bad
    for bad in (dict(M=65), dict(E=513), dict(k=33), dict(H=72, ldx=72, ldr=72, ldy=72), dict(F=40), dict(ldx=56), dict(ldx=68), dict(ldy=60), dict(ldr=60), dict(X=FAKE + 8),
                dict(Y=FAKE + 1), dict(res=FAKE + 1), dict(up=FAKE + 8), dict(dlo=FAKE + 4), dict(ids=FAKE + 2), dict(w=FAKE + 1), dict(H=1 << 16, F=1 << 14, ldx=1 << 16, ldr=1 << 16, ldy=1 << 16)):
        assert call(**bad) == SHAPE, bad
    for bad in (dict(ws=0), dict(bytes_=16384), dict(ws=FAKE + 4)):
        assert call(**bad) == WORKSPACE, bad
    c = nfp._ExpertsStruct(8, 64, 48, 0, 2, FAKE, FAKE, FAKE, FAKE)
    size = lambda M, k: nfp.lib().nestedfp_moe_workspace_size(M, ctypes.byref(c), k)
    assert size(0, 2) == 0 and size(65, 2) == 0 and size(4, 0) == 0 and size(4, 33) == 0 and size(64, 32) > size(1, 1) > 16384
    assert nfp.lib().nestedfp_moe_workspace_size(4, None, 2) == 0


def test_gate_and_up_rows_in_turn(nfp):
    w = torch.arange(12.0).reshape(6, 2)
    assert nfp.interleave_gate_up(w)[:, 0].tolist() == [0.0, 6.0, 2.0, 8.0, 4.0, 10.0]
    assert nfp.interleave_gate_up(torch.arange(4)).tolist() == [0, 2, 1, 3]


def test_descriptions_of_experts(nfp):
    h = lambda *s: torch.zeros(s, dtype=torch.float16)
    for up, down in ((h(4, 8), h(4, 16, 8)), (h(2, 32, 16), h(2, 16, 8)), (h(2, 32, 16).float(), h(2, 16, 16)), (h(3, 32, 16), h(2, 16, 16))):
        with pytest.raises(ValueError):
            nfp.Experts(up, down)


def test_tensors_on_the_host_are_refused(nfp):
    x = torch.zeros((2, 64), dtype=torch.float16)
    m = nfp._marshalled()
    c = nfp._LayerStruct(32, 64, 0, 0, FAKE, FAKE, None, 0, 0)
    e = nfp._ExpertsStruct(8, 64, 48, 0, 2, FAKE, FAKE, FAKE, FAKE)
    with pytest.raises(ValueError):
        m.linear_fused(x, None, ctypes.addressof(c), 0, None, None, 0, False, None, x, x, 0)
    with pytest.raises(ValueError):
        m.moe_route(x, x, 2, 0, True, 1.0, None, x, x, x, 0)
    with pytest.raises(ValueError):
        m.moe(x, ctypes.addressof(e), 0, x, x, None, x, x, 0)
    with pytest.raises(ValueError):
        nfp.moe_route(x, x, 2, scoring="tanh")
