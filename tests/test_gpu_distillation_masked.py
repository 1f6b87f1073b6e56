"""Losses that name a masked element of an ordinary row: those of its finite value, however low, against float64.

Tolerance: that of the loss's other tests; an element this far below the others is in the loss by its value times its
weight, which the bound on a power's argument covers."""
import pytest
import torch

from paper_2609_30342_gb300 import build as pkg_build
from paper_2609_30342_gb300.losses import DistillationLoss
from test_gpu_distillation import DT, _all_ways, _inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    pkg_build.build()
    yield


@pytest.mark.parametrize("low", [None, -1e38, -1e30, -1e20, -1e9, -1e5])
@pytest.mark.parametrize("temperature", [0.5, 1.0, 2.0])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_masked_elements_that_are_named(dtype, temperature, low):
    """By a label, by some of the teacher's entries, by both; None: the type's lowest value.  The weights keep every
    loss within float32's range."""
    low = torch.finfo(DT[dtype]).min if low is None else low
    logits, t, index, labels = _inputs(8, 2048, 9, dtype)
    logits[:, 100:1900] = low
    index, labels = index % 100, labels % 100
    labels[1], index[2, 3], labels[3], index[3, 0] = 500, 600, 700, 700
    index[4], labels[5], index[5, :2] = torch.arange(800, 809, device="cuda"), -100, 1500
    loss, *_ = _all_ways(DistillationLoss(temperature, 0.25, 0.25), logits, t, index, labels)
    assert loss.isfinite().all()


@pytest.mark.parametrize("rows,vocab", [(3, 131072), (2, 33)])
def test_masked_labels_of_long_and_short_rows(rows, vocab):
    logits, _, _, labels = _inputs(rows, vocab, 0)
    logits[:, vocab // 2] = torch.finfo(torch.float32).min
    labels[0] = vocab // 2
    loss, *_ = _all_ways(DistillationLoss(label_weight=0.5), logits, None, None, labels)
    assert loss.isfinite().all()


def test_rows_that_are_not_finite_stay_nan():
    """With a label at the type's lowest value, or at -inf."""
    lowest = torch.finfo(torch.float32).min
    logits, t, index, labels = _inputs(6, 300, 3)
    logits[:, 7] = lowest
    logits[0, 9], logits[1, 9], logits[2], logits[3, 9] = float("nan"), float("inf"), -float("inf"), 1e30
    logits[2, 7] = -float("inf")
    labels[:] = 7
    index[:, 0] = 7
    loss, g = DistillationLoss(2.0, 0.25, 0.25).loss_and_gradient(logits, t, index, labels)
    assert loss[:4].isnan().all() and loss[4:].isfinite().all()
    logits[4, 7] = -float("inf")
    loss, g = DistillationLoss(2.0, 0.25, 0.25).loss_and_gradient(logits, t, index, labels)
    assert loss[4] == float("inf") and g[4].isfinite().all()
