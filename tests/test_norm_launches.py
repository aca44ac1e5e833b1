"""Norms of more rows than one launch takes: how they are cut.  No GPU."""
import os
import shutil
import subprocess

import pytest

from paper_2606_21023_amd import build as hbuild

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_launches_cover_every_row_once(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    exe = str(tmp_path / "norm_launches")
    subprocess.run([gxx, "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover", "-D__HIP_PLATFORM_AMD__",
                    "-I", hbuild.INCLUDE, "-I", hbuild.CSRC, "-I", "/opt/rocm/include",
                    os.path.join(ROOT, "tests", "c", "norm_launches.cpp"), "-L/opt/rocm/lib", "-lamdhip64", "-o", exe],
                   check=True)
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.stdout.strip() == "ok", r.stdout + r.stderr
