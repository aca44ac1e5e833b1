"""The key/value cache's kernels spill no registers (read from the built library)."""
import os
import re
import shutil

import pytest

from paper_2606_21023_amd import build as hbuild
from test_spills import READELF, spills


def test_no_kernel_of_the_cache_spills(tmp_path):
    if not (os.path.exists(hbuild.LIBRARY) and os.path.exists(READELF) and shutil.which("c++filt")):
        pytest.skip("libheal.so, llvm-readelf or c++filt not available")
    found = {name: n for name, n in spills(tmp_path).items()
             if re.search(r"kv_(append|read|select|attention|prompt|combine)_kernel<", name)}
    assert len(found) >= 70, "kernels not found in the library"
    assert {name: n for name, n in found.items() if n} == {}
