"""Every kernel is built into the library once: a launch that no call of a source reaches carries another copy of its kernel along.  Needs no GPU."""
import collections
import os
import re
import subprocess

import pytest

from test_kernel_registers import READELF, code_objects


@pytest.mark.skipif(not os.path.exists(READELF), reason="no llvm-readelf")
def test_no_kernel_is_built_twice(tmp_path):
    from paper_2506_02024_amd import build

    if build.is_stale():
        build.build_library()
    built = collections.Counter()
    for i, image in enumerate(code_objects(build.lib_path())):
        path = tmp_path / ("image%d.o" % i)
        path.write_bytes(image)
        notes = subprocess.run([READELF, "--notes", str(path)], stdout=subprocess.PIPE, text=True, check=True).stdout
        built.update(re.search(r"\.name:\s+(\S+)", kernel).group(1) for kernel in notes.split("- .agpr_count")[1:])
    assert len(built) > 100
    twice = {name: n for name, n in built.items() if n > 1}
    assert not twice, twice
