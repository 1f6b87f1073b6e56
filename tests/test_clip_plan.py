"""The clipping plan, checked on the CPU: the C entries' host code compiled with host memory in the CUDA runtime's place
(tests/clip_plan_check.cu)."""
import os
import subprocess

import pytest

from paper_2609_30342_gb300 import build as pkg_build

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def checker(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("clip") / "clip_plan_check")
    # no device code is run: the kernels are not assembled
    subprocess.run([pkg_build.nvcc(), "-gencode", "arch=compute_103a,code=compute_103a", "-std=c++17", "-O1", "-cudart",
                    "none", "-I", pkg_build.INCLUDE, "-I", pkg_build.CSRC, os.path.join(HERE, "clip_plan_check.cu"),
                    os.path.join(HERE, "host_runtime.cpp"), "-o", exe], check=True)
    return exe


@pytest.mark.parametrize("what", ["upload", "shares"])
def test_plans(checker, what):
    out = subprocess.run([checker, what], capture_output=True, text=True, timeout=300)
    assert out.returncode == 0 and out.stdout.strip().endswith("OK"), out.stdout + out.stderr
