"""Which loads of the adapters' kernels need a check of their bounds.  No GPU."""
import os
import shutil
import subprocess

import pytest

from paper_2606_21023_amd import build as hbuild

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_loads_of_b_stay_within_the_bank(tmp_path):
    """All ranks, every N modulo 32, 16-bit and 32-bit adapters."""
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    exe = str(tmp_path / "lora_index")
    subprocess.run([gxx, "-std=c++17", "-O2", "-D__HIP_PLATFORM_AMD__", "-I", hbuild.INCLUDE, "-I", hbuild.CSRC,
                    "-I", "/opt/rocm/include", os.path.join(ROOT, "tests", "c", "lora_index.cpp"), "-L/opt/rocm/lib",
                    "-lamdhip64", "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.stdout.strip() == "ok", r.stdout + r.stderr
