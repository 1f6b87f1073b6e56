"""A call that is refused for its sizes leaves nothing behind: later calls of the same operator are as a new one's."""
import pytest
import torch

from paper_2609_30342_gb300 import build as pkg_build
from paper_2609_30342_gb300 import rikfad
from paper_2609_30342_gb300.embedding import TokenEmbedding
from paper_2609_30342_gb300.layers import RotaryNorm

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    pkg_build.build()
    yield


def _rand(*shape, seed=0):
    return torch.randn(shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))


def test_rotary_norm_after_too_many_heads():
    """More than 65536 heads of a token are refused, in the backward call too, which asks for its workspace first."""
    q, dq, w = _rand(5, 2, 8), _rand(5, 2, 8, seed=1), _rand(8, seed=2)
    want = RotaryNorm(8).backward(dq, None, q, q_weight=w)
    op, many = RotaryNorm(8), torch.zeros(1, (1 << 16) + 1, 8, device="cuda")
    for _ in range(2):
        with pytest.raises(rikfad.RikfadError, match="heads is out of range"):
            op.backward(many, None, many, q_weight=w)
    got = op.backward(dq, None, q, q_weight=w)
    assert torch.equal(got.q, want.q) and torch.equal(got.q_weight, want.q_weight)


def test_embedding_after_a_scale_that_is_refused():
    d, ids = _rand(9, 4), torch.arange(9, device="cuda") % 5
    want = TokenEmbedding(5, 4, scale=2.0).backward(d, ids)
    op = TokenEmbedding(5, 4)
    op.scale = float("inf")
    for _ in range(2):
        with pytest.raises(rikfad.RikfadError, match="scale must be finite"):
            op.backward(d, ids)
    op.scale = 2.0
    assert torch.equal(op.backward(d, ids), want)
