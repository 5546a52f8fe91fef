"""The bookkeeping of csrc/lds_limits.h (kernels' limits of dynamic LDS), compiled for the host and run
by tests/lds_limits_driver.cpp."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_limits_only_rise(tmp_path):
    cxx = shutil.which(os.environ.get("CXX", "g++"))
    if cxx is None:
        pytest.skip("no host compiler")
    exe = str(tmp_path / "lds_limits")
    b = subprocess.run([cxx, "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                        "-I", os.path.join(ROOT, "paper_2401_06118_amd", "csrc"),
                        os.path.join(ROOT, "tests", "lds_limits_driver.cpp"), "-o", exe],
                       capture_output=True, text=True, timeout=300)
    assert b.returncode == 0, b.stdout + b.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "lds limits ok" in r.stdout, r.stdout + r.stderr
