"""CPU: launch parameters of the attention that no kernel is built for."""
import pytest


@pytest.fixture(scope="module")
def nfp():
    from paper_2506_02024_amd import binding, build

    if build.is_stale():
        build.build_library()
    binding.lib()
    return binding


@pytest.mark.parametrize("value", [1, 2, 3, 5, 6, 7, 9, 12, 16, 1 << 40])
def test_a_number_of_waves_that_no_kernel_has_is_refused(nfp, value):
    # (a call would have launched no tile kernel, and returned success)
    with pytest.raises(nfp.NestedFPError) as e:
        nfp.tune("attn_waves", value)
    assert e.value.status == nfp.ERR_ARG


def test_the_numbers_that_there_are(nfp):
    try:
        for value in (4, 8, 0, -1, -5):
            nfp.tune("attn_waves", value)
    finally:
        nfp.tune("attn_waves", -1)
