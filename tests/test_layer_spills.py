"""The kernels of the residual norms, the adapters and the pages spill no registers (read from the
built library)."""
import os
import re
import shutil

import pytest

from paper_2606_21023_amd import build as hbuild
from test_spills import READELF, spills


def test_no_kernel_of_a_layer_spills(tmp_path):
    if not (os.path.exists(hbuild.LIBRARY) and os.path.exists(READELF) and shutil.which("c++filt")):
        pytest.skip("libheal.so, llvm-readelf or c++filt not available")
    found = {name: n for name, n in spills(tmp_path).items()
             if re.search(r"norm_(any_)?kernel|lora_(down|up)_kernel|IDF16_|kv_(release|fork|reserve|reserve_many|count|moves|moved|compact|copy)_kernel",
                          name)}
    assert len(found) >= 40, "kernels not found in the library: %s" % sorted(found)
    assert {name: n for name, n in found.items() if n} == {}
