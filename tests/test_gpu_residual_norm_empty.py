"""Residual norms of no rows whose gate has rows of its own, as a learned gate has."""
import pytest
import torch

from paper_2609_30342_gb300 import build as pkg_build
from paper_2609_30342_gb300.layers import ResidualNorm

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    pkg_build.build()
    yield


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("gates", [1, 3])
def test_the_gradient_of_a_gate_is_zero(gates, dtype):
    cols = 16384            # large enough for a block of the allocator's own
    op = ResidualNorm(cols, post="rms", pre="rms")
    x, z = (torch.empty(0, cols, dtype=torch.bfloat16, device="cuda", requires_grad=True) for _ in range(2))
    gate = torch.ones(gates, cols, dtype=dtype, device="cuda", requires_grad=True)
    stale = [torch.full_like(gate, float("nan"), requires_grad=False) for _ in range(8)]
    torch.cuda.synchronize()
    del stale                       # the memory that the next allocations of this size get
    u, h = op(x, z, gate)
    got, = torch.autograd.grad(u.sum() + h.sum(), gate)
    assert torch.equal(got, torch.zeros_like(gate))
    _, _, stats = op.forward(x.detach(), z.detach(), gate.detach())
    g = op.backward(x.detach(), z.detach(), x.detach(), z.detach(), gate.detach(), stats=stats)
    assert torch.equal(g.gate, torch.zeros_like(gate))
