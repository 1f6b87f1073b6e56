"""The training step's operators inside autograd, and the residual norm's gradients written over its inputs."""
import pytest
import torch

from paper_2609_30342_gb300 import build as pkg_build
from paper_2609_30342_gb300 import layers, rikfad
from paper_2609_30342_gb300.layers import ResidualNorm, Rotary

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    pkg_build.build()
    yield


def _rand(*shape, seed=0, dtype=torch.float32):
    return torch.randn(shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).to(dtype)


def test_second_derivatives_are_refused():
    """The kernels of the gradients have no gradients of their own: asking for one is an error, not a missing term."""
    x, z = _rand(4, 64, seed=1).requires_grad_(), _rand(4, 64, seed=2).requires_grad_()
    u, h = ResidualNorm(64, post="rms", pre="layer")(x, z)
    g, = torch.autograd.grad((u * h).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        g.sum().backward()
    q = _rand(4, 2, 64, seed=3).requires_grad_()
    out, _ = Rotary(64)(q, None)
    g, = torch.autograd.grad((out * out).sum(), q, create_graph=True)
    with pytest.raises(RuntimeError):
        g.sum().backward()


@pytest.mark.parametrize("over", ["dh", "z"])
@pytest.mark.parametrize("gate_rows", [0, 1, 23])
@pytest.mark.parametrize("post,pre", [("rms", "rms"), ("layer", "layer"), (None, "layer"), ("rms", None)])
@pytest.mark.parametrize("rows,cols", [(23, 64), (92, 777), (1610, 768), (46, 4100)])
def test_gradients_over_their_inputs(rows, cols, post, pre, gate_rows, over):
    """dx may be du, and dz dh or z: the same results to the bit."""
    op = ResidualNorm(cols, post=post, pre=pre)
    x, z, du, dh = (_rand(rows, cols, seed=i, dtype=torch.bfloat16) for i in range(4))
    gate = _rand(rows // gate_rows, cols, seed=4, dtype=torch.bfloat16) if gate_rows else None
    weights = dict(gate=gate, post_weight=_rand(cols, seed=5) if post else None,
                   pre_weight=_rand(cols, seed=6) if pre else None)
    _, _, stats = op.forward(x, z, **weights)
    want = op.backward(du, dh, x, z, stats=stats, **weights)
    none = (None, None)
    head, *_ = op._inputs(x, z, gate, (weights["post_weight"], none[0], weights["pre_weight"], none[1]), None)
    dw = [None if weights[k] is None else torch.empty_like(weights[k]) for k in ("post_weight", "pre_weight")]
    dgate = None if gate is None else torch.empty_like(gate)
    dz = dh if over == "dh" else z
    address = lambda t: 0 if t is None else t.data_ptr()
    body = (*head, 0, 0, 0, 0, stats.data_ptr(), du.data_ptr(), cols, dh.data_ptr(), cols, du.data_ptr(), cols,
            dz.data_ptr(), cols, address(dgate), cols, address(dw[0]), 0, address(dw[1]), 0)
    lib = rikfad.lib()
    nbytes = lib.rikfad_residual_norm_workspace(layers._NORM.pack(*body, 0, 0))
    work = torch.empty(max(nbytes, 1), dtype=torch.uint8, device="cuda")
    rikfad._check(lib.rikfad_residual_norm_backward(layers._NORM.pack(*body, work.data_ptr(), nbytes),
                                                    rikfad._raw_stream(0)))
    for got, ref in ((du, want.x), (dz, want.z), (dgate, want.gate), (dw[0], want.post_weight), (dw[1], want.pre_weight)):
        assert (got is None and ref is None) or torch.equal(got, ref)
