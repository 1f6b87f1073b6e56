"""A tensor that an explicit call writes to (``out``) counts as changed: a backward pass through a graph that holds it is
refused, not computed from what was written over its inputs."""
import pytest
import torch

from paper_2609_30342_gb300 import build as pkg_build
from paper_2609_30342_gb300.embedding import TokenEmbedding
from paper_2609_30342_gb300.layers import RotaryNorm
from paper_2609_30342_gb300.losses import DistillationLoss

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    pkg_build.build()
    yield


def _rand(*shape, seed=0):
    return torch.randn(shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))


def _logits():
    x, labels = _rand(6, 50).requires_grad_(), torch.arange(6, device="cuda")
    return x, x * 2.0, labels


def test_the_gradient_written_over_the_logits():
    op = DistillationLoss(label_weight=1.0)
    x, logits, labels = _logits()
    value = op(logits, labels=labels).mean()
    losses, _ = op.loss_and_gradient(logits.detach(), labels=labels, out=logits.detach())
    assert torch.equal(losses.mean(), value.detach())
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        value.backward()
    x, logits, labels = _logits()
    value = op(logits, labels=labels).mean()
    _, stats = op.forward(logits.detach(), labels=labels)
    op.backward(None, logits.detach(), labels=labels, stats=stats, out=logits.detach())
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        value.backward()


def test_heads_in_place():
    op, w = RotaryNorm(16), _rand(16)
    x, y = _rand(5, 2, 16).requires_grad_(), _rand(5, 1, 16).requires_grad_()
    for written in (0, 1):
        q, k = x * 2.0, y * 2.0
        a, b = op(q, k, w, w)
        to = [torch.empty_like(q), torch.empty_like(k)]
        to[written] = (q, k)[written].detach()
        op.forward(q.detach(), k.detach(), w, w, out=to)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            (a.sum() + b.sum()).backward()


def test_rows_and_tables():
    op, ids = TokenEmbedding(7, 8), torch.arange(5, device="cuda")
    for rows, write in ((5, lambda t: op.forward(_rand(7, 8), ids, out=t)), (7, lambda t: op.backward(_rand(5, 8), ids, out=t)),
                        (7, lambda t: op.backward(_rand(5, 8), ids, out=t, accumulate=True))):
        t = _rand(rows, 8).requires_grad_() * 2.0
        value = (t * t).sum()
        write(t.detach())
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            value.backward()


def test_new_results_and_graphs_without_the_tensor_are_not_refused():
    """A fresh result leaves the inputs as they were; so does a graph that holds other tensors."""
    op = DistillationLoss(label_weight=1.0)
    x, logits, labels = _logits()
    value = op(logits, labels=labels).sum()
    _, g = op.loss_and_gradient(logits.detach(), labels=labels)
    d, = torch.autograd.grad(value, x)
    assert torch.equal(d, 2 * op.backward(None, logits.detach(), labels=labels, stats=op.forward(logits.detach(), labels=labels)[1]))
    other = torch.empty_like(g)
    x, logits, labels = _logits()
    value = op(logits, labels=labels).sum()
    op.loss_and_gradient(logits.detach(), labels=labels, out=other)
    assert torch.equal(torch.autograd.grad(value, x)[0], d) and torch.equal(other, g)
    with torch.inference_mode():
        t = torch.empty(6, 50, device="cuda")
        op.loss_and_gradient(logits.detach(), labels=labels, out=t)
        assert torch.equal(t, g)
