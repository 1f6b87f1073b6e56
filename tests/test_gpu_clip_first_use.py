"""A clipping plan used as soon as it is made, on streams that do not wait for the legacy one."""
import pytest
import torch

from paper_2609_30342_gb300 import build as pkg_build
from paper_2609_30342_gb300.gradients import GradientClipper
from test_gpu_clip import _check_norms, _check_out, _grads

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    pkg_build.build()
    yield


def test_first_use_on_a_side_stream():
    numels = [300_007, 5, 70_000, 1 << 20] + [131] * 1500
    grads = _grads(numels, "f32")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(4):
        clipper = GradientClipper(numels, "f32")
        with torch.cuda.stream(side):
            out = [torch.empty_like(g) for g in grads]
            total, norms = clipper.clip(0.5, grads, out=out)
        side.synchronize()
        _check_norms(total, norms, grads)
        _check_out(out, grads, 0.5, "f32")
        clipper.close()
