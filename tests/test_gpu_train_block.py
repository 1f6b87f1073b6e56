"""The operators together: a small model's gradients against plain torch operations, and a training run."""
import pytest
import torch

from paper_2609_30342_gb300 import build as pkg_build
from paper_2609_30342_gb300 import train_block
from paper_2609_30342_gb300.layers import rotary_frequencies

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    pkg_build.build()
    yield


def _plain_norm(v, weight):
    return v * torch.rsqrt((v * v).mean(-1, keepdim=True) + 1e-6) * weight


class _PlainResidualNorm:
    def __init__(self, branch_scale=1.0):
        self.b = branch_scale

    def __call__(self, x, z=None, gate=None, post_weight=None, pre_weight=None, dtype=None):
        u = x if z is None else x + self.b * gate * _plain_norm(z, post_weight)
        return u, _plain_norm(u, pre_weight)


class _PlainRotary:
    def __init__(self, head_dim):
        self.f = torch.tensor(rotary_frequencies(head_dim)[0], dtype=torch.float64, device="cuda")

    def __call__(self, q, k, positions):
        angle = positions.double()[:, None, None] * self.f
        c, s = torch.cos(angle).to(q.dtype), torch.sin(angle).to(q.dtype)

        def turn(v):
            a, b = v.chunk(2, -1)
            return torch.cat((a * c - b * s, b * c + a * s), -1)
        return turn(q), turn(k)


def test_gradients_match_plain_operations():
    """float32 through both: the operators are off by some units of 2^-24 (their own tests), a dozen operators and
    products in a row by 1e-5 of a tensor's size at most; float64 is the reference of both."""
    width, layers = 64, 2
    tokens, positions = train_block.batch(3, 97, (40, 1, 23))
    kw = dict(vocab=97, width=width, layers=layers, heads=4)
    torch.manual_seed(1)
    own = train_block.Model(dtype=torch.float32, **kw).cuda()
    plain = train_block.Model(dtype=torch.float64, norm=_PlainResidualNorm((2 * layers) ** -0.5),
                              first=_PlainResidualNorm(), rotary=_PlainRotary(width // 4), **kw).cuda().double()
    plain.load_state_dict(own.state_dict())
    for m in (own, plain):
        train_block.loss_of(m, tokens, positions).backward()
    for (name, a), b in zip(own.named_parameters(), plain.parameters()):
        err = float((a.grad.double() - b.grad).norm()) / float(b.grad.norm())
        assert err <= 1e-4, (name, err)


def test_training_lowers_the_loss():
    losses, norms = train_block.train(steps=60, width=128, lengths=(120, 31, 1, 100))
    assert all(0 < n < float("inf") for n in norms)
    assert sum(losses[-5:]) / 5 < 0.75 * losses[0]
