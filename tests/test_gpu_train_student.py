"""Embedding, heads' norms with rotation and the loss against a teacher together: a small model's gradients against plain
torch operations, and a run of the example."""
import pytest
import torch

from paper_2609_30342_gb300 import build as pkg_build
from paper_2609_30342_gb300 import train_block
from paper_2609_30342_gb300.embedding import TokenEmbedding
from paper_2609_30342_gb300.layers import RotaryNorm, rotary_frequencies
from paper_2609_30342_gb300.losses import DistillationLoss

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


class _PlainRotaryNorm:
    eps = 1e-6

    def __init__(self, head_dim):
        self.f = torch.tensor(rotary_frequencies(head_dim)[0], dtype=torch.float64, device="cuda")

    def __call__(self, q, k, q_weight, k_weight, positions):
        angle = positions.double()[:, None, None] * self.f
        c, s = torch.cos(angle), torch.sin(angle)

        def turn(v):
            a, b = v.chunk(2, -1)
            return torch.cat((a * c - b * s, b * c + a * s), -1)
        return turn(_plain_norm(q, q_weight)), turn(_plain_norm(k, k_weight))


class _PlainLoss:
    def __init__(self, T, a, b):
        self.T, self.a, self.b = T, a, b

    def __call__(self, logits, teacher, index, labels):
        there = index >= 0
        soft = torch.log_softmax((teacher / self.T).masked_fill(~there, -1e300), -1)
        log_q = torch.log_softmax(logits / self.T, -1).gather(1, index.clamp(min=0))
        kl = torch.where(there, soft.exp() * (soft - log_q), torch.zeros_like(soft)).sum(1)
        kl = torch.where(there.any(1), kl, torch.zeros_like(kl))
        nll = -torch.log_softmax(logits, -1).gather(1, labels.clamp(min=0)[:, None])[:, 0]
        return self.a * self.T ** 2 * kl + self.b * torch.where(labels >= 0, nll, torch.zeros_like(nll))


@pytest.mark.parametrize("width", [64, 72])
def test_gradients_match_plain_operations(width):
    """float32 through both: the operators are off by some units of 2^-24 (their own tests), some twenty operators and
    products in a row by 1e-5 of a tensor's size at most; float64 is the reference of both."""
    layers = 2
    tokens, positions = train_block.batch(3, 97, (40, 1, 23))
    kw = dict(vocab=97, width=width, layers=layers, heads=4)
    torch.manual_seed(1)
    own = train_block.Model(dtype=torch.float32, rotary=RotaryNorm(width // 4), table=TokenEmbedding(97, width), **kw).cuda()
    plain = train_block.Model(dtype=torch.float64, norm=_PlainResidualNorm((2 * layers) ** -0.5),
                              first=_PlainResidualNorm(), rotary=_PlainRotaryNorm(width // 4), **kw).cuda().double()
    with torch.no_grad():
        for p in own.parameters():
            if p.dim() < 2:
                p.add_(0.1 * torch.randn_like(p))
    plain.load_state_dict(own.state_dict())
    gen = torch.Generator(device="cuda").manual_seed(2)
    teacher = torch.randn(64, 9, device="cuda", generator=gen)
    index = torch.rand(64, 97, device="cuda", generator=gen).argsort(1)[:, :9].contiguous()
    index[5] = -1
    a = train_block.distillation_loss(own, tokens, positions, DistillationLoss(2.0, 0.6, 0.4), teacher, index)
    b = train_block.distillation_loss(plain, tokens, positions, _PlainLoss(2.0, 0.6, 0.4), teacher.double(), index)
    assert abs(float(a.detach()) - float(b.detach())) <= 1e-5 * abs(float(b.detach()))
    for v in (a, b):
        v.backward()
    for (name, p), r in zip(own.named_parameters(), plain.named_parameters()):
        assert name == r[0]
        err = float((p.grad.double() - r[1].grad).norm()) / float(r[1].grad.norm())
        assert err <= 1e-4, (name, err)


def test_student_runs():
    teacher, *_ = train_block.train_model(steps=3, width=128, lengths=(60, 1, 40))
    model, losses, norms = train_block.distil(teacher, steps=3, layers=1, lengths=(60, 1, 40))
    assert all(0 < n < float("inf") for n in norms) and all(0 < v < float("inf") for v in losses)
    assert all(torch.isfinite(p).all() for p in model.parameters())
