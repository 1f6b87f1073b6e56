"""Launch parameters of the residual norm, checked on the CPU: the C entries' host code compiled with a checker in the
kernels' place (tests/norm_launch_check.cpp)."""
import os
import subprocess

import pytest

from paper_2609_30342_gb300 import build as pkg_build

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def checker(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("norm") / "norm_launch_check")
    subprocess.run([pkg_build.nvcc(), "-x", "c++", "-std=c++17", "-O1", "-cudart", "none", "-I", pkg_build.INCLUDE, "-I",
                    pkg_build.CSRC, os.path.join(HERE, "norm_launch_check.cpp"), os.path.join(HERE, "host_runtime.cpp"), "-o", exe],
                   check=True)
    return exe


@pytest.mark.parametrize("what", ["copies", "shapes"])
def test_launches(checker, what):
    out = subprocess.run([checker, what], capture_output=True, text=True, timeout=300)
    assert out.returncode == 0 and out.stdout.strip().endswith("OK"), out.stdout + out.stderr
