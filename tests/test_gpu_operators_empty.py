"""Empty batches inside autograd.  The gradient of a sum is an expanded scalar, and without elements it stays one: its
strides are 0."""
import pytest
import torch

from paper_2609_30342_gb300 import build as pkg_build
from paper_2609_30342_gb300.layers import ResidualNorm, Rotary

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    pkg_build.build()
    yield


@pytest.mark.parametrize("lead", [(0,), (2, 0), (0, 3)])
def test_residual_norm(lead):
    x, z = (torch.empty(*lead, 64, dtype=torch.bfloat16, device="cuda", requires_grad=True) for _ in range(2))
    w = torch.ones(64, device="cuda", requires_grad=True)
    u, h = ResidualNorm(64, post="rms", pre="layer")(x, z, post_weight=w, pre_weight=w)
    assert u.shape == h.shape == x.shape
    dx, dz, dw = torch.autograd.grad(u.sum() + h.sum(), (x, z, w))
    assert dx.shape == x.shape and dz.shape == z.shape and torch.equal(dw, torch.zeros_like(w))


@pytest.mark.parametrize("shape", [(0, 2, 64), (2, 0, 2, 64), (0, 3, 2, 64), (3, 0, 64)])
def test_rotary(shape):
    q, k = (torch.empty(shape, dtype=torch.bfloat16, device="cuda", requires_grad=True) for _ in range(2))
    a, b = Rotary(64)(q, k)
    dq, dk = torch.autograd.grad(a.sum() + b.sum(), (q, k))
    assert dq.shape == q.shape and dk.shape == k.shape
