"""The residual norm's backward pass without the gradient of u or of h, where the rows do not start on 16 bytes."""
import pytest
import torch

from paper_2609_30342_gb300 import build as pkg_build
from paper_2609_30342_gb300.layers import ResidualNorm
from test_gpu_residual_norm import NAMES, _inputs, check, reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    pkg_build.build()
    yield


def _run(t, gate_rows, **kw):
    op = ResidualNorm(t["x"].shape[1], **kw)
    weights = {k: t[k] for k in NAMES}
    _, _, stats = op.forward(t["x"], t["z"], **weights)
    g = op.backward(t["du"], t["dh"], t["x"], t["z"], stats=stats, **weights)
    ref, tol = reference(op, t, gate_rows)
    for k in ("x", "z") + NAMES:
        if t[k] is not None:
            check("d" + k, getattr(g, k), ref[k], tol[k])


@pytest.mark.parametrize("none", ["du", "dh"])
@pytest.mark.parametrize("dtype,residual", [("f32", "same"), ("bf16", "same"), ("f16", "f32")])
@pytest.mark.parametrize("rows,gate_rows,cols", [(8192, 16, 1001), (1400, 7, 37), (1398, 3, 129), (600, 600, 4099), (1, 1, 9)])
def test_gates_of_few_rows(rows, gate_rows, cols, dtype, residual, none):
    t = _inputs(rows, cols, dtype, residual, post="rms", pre="layer", gate="shared", gate_rows=gate_rows)
    t[none] = None
    _run(t, gate_rows, post="rms", pre="layer")


@pytest.mark.parametrize("none", ["du", "dh"])
@pytest.mark.parametrize("dtype,residual", [("f32", "same"), ("bf16", "same"), ("bf16", "f32")])
@pytest.mark.parametrize("offset", [1, 3, 4])
@pytest.mark.parametrize("cols", [64, 1000, 1001, 8200])
def test_rows_that_start_anywhere(cols, offset, dtype, residual, none):
    t = _inputs(19, cols, dtype, residual, post="layer", pre="rms")
    t["x"] = torch.cat([t["x"].new_zeros(offset), t["x"].flatten()])[offset:].view(19, cols)
    t[none] = None
    _run(t, 1, post="layer", pre="rms")


def test_the_last_norm_of_a_model():
    """Only h reaches the loss: autograd hands no gradient of u to the backward pass."""
    rows, cols, gate_rows = 96, 1001, 4
    op = ResidualNorm(cols, post="rms", pre="rms")
    t = _inputs(rows, cols, "bf16", gate="shared", gate_rows=gate_rows)
    leaves = {k: v.requires_grad_() for k, v in t.items() if v is not None and k not in ("du", "dh")}
    _, h = op(leaves["x"], leaves["z"], *[leaves.get(k) for k in NAMES])
    grads = torch.autograd.grad(h, list(leaves.values()), t["dh"])
    t["du"] = None
    ref, tol = reference(op, {k: None if v is None else v.detach() for k, v in t.items()}, gate_rows)
    for k, g in zip(leaves, grads):
        check("d" + k, g, ref[k], tol[k])
