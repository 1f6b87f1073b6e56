"""Residual norms of the widest rows, dense and in wider rows: they start anywhere, and a cluster's blocks have no column
left over."""
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


@pytest.mark.parametrize("dtype,residual", [("f32", "same"), ("bf16", "same"), ("f16", "f32")])
@pytest.mark.parametrize("cols,pad", [(32760, 1), (32761, 0), (32762, 0), (32763, 0), (32764, 0), (32766, 0), (32767, 0),
                                      (32768, 1), (32768, 4)])
def test_widest_rows(cols, pad, dtype, residual):
    op = ResidualNorm(cols, post="layer", pre="rms")
    t = _inputs(5, cols, dtype, residual, post="layer", pre="rms", gate="rows")
    for k in ("x", "z", "gate", "du", "dh") if pad else ():
        wide = torch.full((5, cols + pad), float("nan"), dtype=t[k].dtype, device="cuda")
        wide[:, :cols] = t[k]
        t[k] = wide[:, :cols]
    run(op, t)


@pytest.mark.parametrize("cols", [32761, 32767])
def test_shared_gates(cols):
    op = ResidualNorm(cols, post="rms", pre="layer")
    run(op, _inputs(12, cols, "bf16", post="rms", pre="layer", gate="shared", gate_rows=4), 4)
