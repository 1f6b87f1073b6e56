"""The row operators captured in a graph: the replays work on what the inputs hold by then."""
import pytest
import torch

from paper_2609_30342_gb300 import build as pkg_build
from paper_2609_30342_gb300.layers import ResidualNorm, Rotary

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    pkg_build.build()
    yield


def _rand(*shape, seed=0):
    return torch.randn(shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).bfloat16()


def _check(inputs, call):
    """Captures ``call`` after a warm-up, and compares replays on new inputs with plain calls."""
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for seed in (5, 6):
        for i, t in enumerate(inputs):
            t.copy_(_rand(*t.shape, seed=10 * seed + i))
        want = [t.clone() for t in call()]
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


@pytest.mark.parametrize("rows,cols,gates", [(1, 768, 0), (600, 768, 0), (600, 1001, 4), (40, 5000, 40)])
def test_residual_norm(rows, cols, gates):
    op = ResidualNorm(cols, post="rms", pre="layer")
    x, z, du, dh = inputs = [_rand(rows, cols, seed=i) for i in range(4)]
    gate = _rand(gates, cols, seed=4) if gates else None
    w = _rand(cols, seed=5)

    def call():
        u, h, stats = op.forward(x, z, gate, post_weight=w, pre_weight=w)
        g = op.backward(du, dh, x, z, gate, post_weight=w, pre_weight=w, stats=stats)
        return [t for t in (u, h, *g) if t is not None]

    _check(inputs, call)


@pytest.mark.parametrize("tokens", [1, 700])
def test_rotary(tokens):
    op = Rotary(64)
    q, k = inputs = [_rand(tokens, 12, 64), _rand(tokens, 4, 64, seed=1)]
    positions = torch.arange(tokens, device="cuda")
    _check(inputs, lambda: [*op.rotate(q, k, positions=positions), *op.rotate(q, k, positions=positions, inverse=True)])
