"""CPU: a workspace for the largest batch of a router or of experts takes every smaller one."""
import ctypes

import pytest

FAKE = 0x10000                                             # aligned, never dereferenced


@pytest.fixture(scope="module")
def nfp():
    from paper_2506_02024_amd import binding, build

    if build.is_stale():
        build.build_library()
    binding.lib()
    return binding


@pytest.mark.parametrize("K", [16, 512, 2048, 7168])
@pytest.mark.parametrize("E", [1, 8, 60, 64, 128, 250, 256, 512])
def test_router(nfp, E, K):
    size, most = nfp.lib().nestedfp_moe_route_workspace_size, 0
    for M in list(range(1, 4097)) + [8192, 8193, 16384, 16385, 1 << 20]:
        need = size(M, E, K)
        assert need >= most, (M, need, most)
        assert need <= nfp.WORKSPACE_COUNTER_BYTES + (32 << 20)
        most = need


def test_experts(nfp):
    for E, H, F, top in ((8, 1040, 528, 2), (128, 2048, 768, 8), (512, 32, 16, 32)):
        c = nfp._ExpertsStruct(E, H, F, 0, 2, FAKE, FAKE, FAKE, FAKE)
        sizes = [nfp.lib().nestedfp_moe_workspace_size(M, ctypes.byref(c), top) for M in range(1, nfp.MOE_MOST_TOKENS + 1)]
        assert sizes == sorted(sizes)
