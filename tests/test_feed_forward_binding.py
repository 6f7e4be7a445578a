"""CPU: what the binding refuses of a linear's codes before it looks at their tensors."""
import ctypes

import pytest
import torch

FAKE = 0x10000                                             # aligned, never dereferenced


@pytest.fixture(scope="module")
def nfp():
    from paper_2506_02024_amd import binding, build

    if build.is_stale():
        build.build_library()
    binding.lib()
    return binding


def test_codes_are_multiplied_in_fp8_mode_by_their_own_scales(nfp):
    """Codes with FP16 mode, or with a scale for activations that are still to be quantised: neither can be meant."""
    c = nfp._LayerStruct(32, 64, 0, 0, FAKE, FAKE, None, 0, 0)
    codes, scales, y = torch.zeros((2, 64), dtype=torch.uint8), torch.ones(2), torch.zeros((2, 32), dtype=torch.float16)
    m = nfp._marshalled()
    call = lambda mode, act_scale: m.linear_fused(codes, scales, ctypes.addressof(c), mode, act_scale, None, 0, False, None, y, y, 0)
    with pytest.raises(ValueError, match="mode"):
        call(nfp.MODE_FP16, None)
    with pytest.raises(ValueError, match="act_scale"):
        call(nfp.MODE_FP8, torch.ones(1))
    with pytest.raises(ValueError, match="on the GPU"):    # (the right call gets as far as its tensors)
        call(nfp.MODE_FP8, None)
