"""Clipping plans and calls go to the gradients' device, whichever is current: the library and the runtime's current
device replaced on the CPU."""
import pytest
import torch

from paper_2609_30342_gb300 import gradients, rikfad
from paper_2609_30342_gb300.optim import RIKFADOptimizer


class _Machine:
    """Two devices, the first one current; the calls that went through and the device that each found current."""

    def __init__(self, monkeypatch):
        self.current, self.calls = 0, []
        machine = self

        class device:
            def __init__(self, d):
                self.index = d if isinstance(d, int) else torch.device(d).index

            def __enter__(self):
                self.before, machine.current = machine.current, self.index

            def __exit__(self, *exc):
                machine.current = self.before

        class Library:
            def __getattr__(self, name):
                def call(*args):
                    if name == "rikfad_clip_create":
                        machine.plan = machine.current
                    elif machine.current != machine.plan:
                        return rikfad.ERR_STATE
                    machine.calls.append((name, machine.current))
                    return 0
                return call

        real = torch.empty
        monkeypatch.setattr(torch.cuda, "device", device)
        monkeypatch.setattr(torch.cuda, "current_device", lambda: machine.current)
        monkeypatch.setattr(torch, "empty", lambda *a, **kw: real(*a, **dict(kw, device="cpu")))
        monkeypatch.setattr(rikfad, "lib", lambda: library)
        monkeypatch.setattr(rikfad, "_raw_stream", lambda index: 0)
        library = Library()


class _Pointers:
    def __init__(self, index):
        self.grads = self.out = None
        self.device = torch.device("cuda", index)


@pytest.mark.parametrize("index", [0, 1])
def test_plan_and_call(monkeypatch, index):
    machine = _Machine(monkeypatch)
    clipper = gradients.GradientClipper([3], "f32", device=torch.device("cuda", index))
    clipper.norm(ptrs=_Pointers(index))
    assert machine.calls == [("rikfad_clip_create", index), ("rikfad_clip_run", index)] and machine.current == 0


def test_a_plan_of_another_device_is_refused(monkeypatch):
    _Machine(monkeypatch)
    clipper = gradients.GradientClipper([3], "f32", device=torch.device("cuda", 1))
    monkeypatch.setattr(rikfad, "_check", _raise)
    with pytest.raises(RuntimeError):
        clipper.norm(ptrs=_Pointers(0))


def _raise(code):
    if code:
        raise RuntimeError(code)


def test_the_optimiser_plans_where_the_gradients_are(monkeypatch):
    made = []

    class Clipper:
        def __init__(self, numels, dtypes, device=None):
            made.append((tuple(numels), device))

        def clip(self, max_norm, grads):
            return (max_norm,)

        def close(self):
            pass

    monkeypatch.setattr(gradients, "GradientClipper", Clipper)
    p = torch.nn.Parameter(torch.zeros(5))
    opt = RIKFADOptimizer([p], lr=0.05, alpha=0.2, mu=1e-3)
    opt.clip_grad_norm(1.0)
    p.grad = torch.zeros(5)
    opt.clip_grad_norm(1.0)
    assert made == [((), None), ((5,), p.device)]
