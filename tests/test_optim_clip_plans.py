"""The plans that RIKFADOptimizer.clip_grad_norm keeps, where the set of gradients changes from step to step."""
import pytest
import torch

from paper_2609_30342_gb300 import build as pkg_build
from paper_2609_30342_gb300 import gradients, optim
from paper_2609_30342_gb300.optim import RIKFADOptimizer

HP = dict(lr=0.05, alpha=0.2, mu=1e-3)


class _Plans:
    """GradientClipper's stand-in on the CPU: what was planned and closed."""

    def __init__(self, monkeypatch):
        self.made, self.closed = [], []
        plans = self

        class Clipper:
            def __init__(self, numels, dtypes, **kw):
                self.numels = tuple(numels)
                plans.made.append(self.numels)

            def clip(self, max_norm, grads):
                assert tuple(g.numel() for g in grads) == self.numels and self not in plans.closed
                return (max_norm,)

            def close(self):
                plans.closed.append(self)

        monkeypatch.setattr(gradients, "GradientClipper", Clipper)


def _step(opt, params, chosen):
    for i, p in enumerate(params):
        p.grad = torch.zeros_like(p) if i in chosen else None
    return opt.clip_grad_norm(1.0)


def test_alternating_sets_are_planned_once(monkeypatch):
    plans = _Plans(monkeypatch)
    params = [torch.nn.Parameter(torch.zeros(3 + i)) for i in range(4)]
    opt = RIKFADOptimizer(params, **HP)
    for _ in range(5):
        for chosen in ((0, 1), (0, 2), (), (0, 1, 2, 3)):
            _step(opt, params, chosen)
    assert plans.made == [(3, 4), (3, 5), (), (3, 4, 5, 6)] and plans.closed == []
    opt.close()
    assert len(plans.closed) == 4
    _step(opt, params, (0, 1))
    assert len(plans.made) == 5


def test_the_number_of_plans_is_bounded_and_the_oldest_goes(monkeypatch):
    plans = _Plans(monkeypatch)
    params = [torch.nn.Parameter(torch.zeros(1 + i)) for i in range(optim.CLIP_PLANS + 4)]
    opt = RIKFADOptimizer(params, **HP)
    for i in range(len(params)):
        _step(opt, params, (0,))            # stays in use
        _step(opt, params, (i,))
    assert len(plans.made) == len(params) and len(plans.closed) == 4
    assert [c.numels for c in plans.closed] == [(2,), (3,), (4,), (5,)]


@pytest.mark.gpu
def test_nothing_waits_once_the_lists_are_planned():
    pkg_build.build()
    params = [torch.nn.Parameter(torch.randn(300, 40, device="cuda")) for _ in range(3)]
    opt = RIKFADOptimizer(params, **HP)

    def step(chosen):
        for i, p in enumerate(params):
            p.grad = torch.full_like(p, 2.0) if i in chosen else None
        return opt.clip_grad_norm(1.0)

    sets = [(0, 1), (1, 2), (0, 1, 2), (2,)]
    for chosen in sets:
        step(chosen)
    torch.cuda.synchronize()
    torch.cuda._sleep(1_000_000_000)
    slept = torch.cuda.Event()
    slept.record()
    totals = [step(chosen) for chosen in sets * 2]
    assert not slept.query()
    torch.cuda.synchronize()
    for total, chosen in zip(totals, sets * 2):
        want = 2.0 * (12000 * len(chosen)) ** 0.5
        assert abs(float(total) - want) <= 1e-5 * want
    opt.close()
