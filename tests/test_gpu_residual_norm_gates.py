"""Residual norms whose gates serve few rows each: many gates, most of them within one group of threads."""
import pytest
import torch

from paper_2609_30342_gb300 import build as pkg_build
from paper_2609_30342_gb300.layers import ResidualNorm
from test_gpu_residual_norm import _inputs, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    pkg_build.build()
    yield


@pytest.mark.parametrize("rows,gate_rows", [(4096, 2), (4096, 4), (4098, 3), (6000, 15), (6000, 16), (6000, 40), (9, 3),
                                            (2, 2), (1200, 600), (40000, 5)])
@pytest.mark.parametrize("cols", [24, 136, 260, 777, 1600])
def test_gates_of_few_rows(rows, gate_rows, cols):
    op = ResidualNorm(cols, post="rms", pre="layer")
    run(op, _inputs(rows, cols, "bf16", post="rms", pre="layer", gate="shared", gate_rows=gate_rows), gate_rows)
