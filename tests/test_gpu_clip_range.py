"""Clipping whose factor is below float32's normal range, and totals above float32's range."""
import math

import pytest
import torch

from paper_2609_30342_gb300 import build as pkg_build
from paper_2609_30342_gb300.gradients import GradientClipper
from test_gpu_clip import DT, EPS, HALF_ULP, TINY, _check_norms, _check_out, _exact, _grads

pytestmark = pytest.mark.gpu

NUMELS = [20_000, 500, 13]


@pytest.fixture(scope="module", autouse=True)
def built():
    pkg_build.build()
    yield


@pytest.mark.parametrize("std,max_norm", [(1e36, 1e-3), (1e36, 1e-6), (1e34, 1e-9), (3e33, 1.0), (1e30, 1e-6), (1e36, 0.0)])
@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16")])
def test_factors_below_the_normal_range(std, max_norm, dtype, out):
    grads = _grads(NUMELS, dtype, std=std)
    clipper = GradientClipper(NUMELS, dtype, out)
    outs = [torch.empty(n, dtype=DT[out], device="cuda") for n in NUMELS]
    total, norms = clipper.clip(max_norm, grads, out=outs)
    _check_norms(total, norms, grads)
    _check_out(outs, grads, max_norm, out)
    if dtype == out:
        keep = [g.clone() for g in grads]
        clipper.clip(max_norm, grads)
        assert all(torch.equal(g, o) for g, o in zip(grads, outs))
        _check_out(grads, keep, max_norm, out)


@pytest.mark.parametrize("max_norm", [1.0, 1e-4, 1e30])
def test_small_elements_beside_large_ones(max_norm):
    grads = _grads(NUMELS, "f32", std=1.0)
    grads[0][7] = 1e38
    out = [torch.empty_like(g) for g in grads]
    total, norms = GradientClipper(NUMELS, "f32").clip(max_norm, grads, out=out)
    _check_norms(total, norms, grads)
    _check_out(out, grads, max_norm, "f32")


@pytest.mark.parametrize("max_norm", [1.0, 1e-6, 1e37])
def test_totals_above_the_range(max_norm):
    """The total is infinite as a float32, but its factor is formed before it is rounded."""
    grads = [torch.full((n,), 3e38, device="cuda") for n in NUMELS]
    out = [torch.empty_like(g) for g in grads]
    total, norms = GradientClipper(NUMELS, "f32").clip(max_norm, grads, out=out)
    assert math.isinf(float(total)) and all(map(math.isinf, norms.tolist()))
    _check_out(out, grads, max_norm, "f32")
