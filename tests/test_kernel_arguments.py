"""Arguments of the built kernels, from the notes of the library's code objects: what only an epilogue needs is not among those of the bare kernels, whose launches
it would make longer.  Needs no GPU."""
import os
import re
import subprocess

import pytest

from test_kernel_registers import READELF, code_objects

EPILOGUE = 40                                              # bytes of its description


@pytest.mark.skipif(not os.path.exists(READELF), reason="no llvm-readelf")
def test_bare_kernels_are_not_given_an_epilogue(tmp_path):
    from paper_2506_02024_amd import build

    if build.is_stale():
        build.build_library()
    sizes = {}                                             # (family, has an epilogue) -> bytes of what the host passes
    for i, image in enumerate(code_objects(build.lib_path())):
        path = tmp_path / ("image%d.o" % i)
        path.write_bytes(image)
        notes = subprocess.run([READELF, "--notes", str(path)], stdout=subprocess.PIPE, text=True, check=True).stdout
        for kernel in notes.split("- .agpr_count")[1:]:
            name = re.search(r"\.name:\s+(\S+)", kernel).group(1)
            family = re.search(r"(small_gemm|large_gemm|nested_bypass|nested_rows|e4m3_bypass|splitk_reduce)_kernelI(.*?)EEEv", name)
            if family is None:
                continue
            given = [int(size) for size, kind in re.findall(r"\.size:\s+(\d+)\s+\.value_kind:\s+(\w+)", kernel) if not kind.startswith("hidden")]
            integers = re.findall(r"L[bi](\d+)", family.group(2))
            epilogue = int(integers[0] if family.group(1) == "splitk_reduce" else integers[-1]) != 0
            sizes.setdefault((family.group(1), epilogue), set()).add(sum(given))
    assert len(sizes) == 12 and all(len(s) == 1 for s in sizes.values()), sizes
    for family, epilogue in sizes:
        if not epilogue:
            bare, fused = (max(sizes[family, e]) for e in (False, True))
            # (an empty structure in the place of the description takes a byte)
            assert bare <= fused - EPILOGUE + 1, (family, bare, fused)
