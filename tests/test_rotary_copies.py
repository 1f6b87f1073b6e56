"""Copies of a Rotary turn by their own frequencies: deepcopy (an averaged model) and pickle (a saved one) give an object
that knows nothing of the first one's memory."""
import copy
import pickle

import pytest
import torch

from paper_2609_30342_gb300 import build as pkg_build
from paper_2609_30342_gb300.layers import Rotary


@pytest.fixture(scope="module", autouse=True)
def built():
    pkg_build.build()
    yield


COPIES = {"deepcopy": copy.deepcopy, "pickle": lambda op: pickle.loads(pickle.dumps(op))}


@pytest.mark.parametrize("kind", COPIES)
def test_no_address_is_copied(kind):
    op = Rotary(64, device="cpu")
    other = COPIES[kind](op)
    assert torch.equal(other.turns, op.turns) and other.turns.data_ptr() != op.turns.data_ptr()
    assert op.turns.data_ptr() not in [v for v in vars(other).values() if isinstance(v, int)]


@pytest.mark.gpu
@pytest.mark.parametrize("kind", COPIES)
def test_a_copy_turns_by_its_own_frequencies(kind):
    op = Rotary(64)
    q = torch.randn(9, 2, 64, device="cuda")
    want, _ = op.rotate(q, start=5)
    other = COPIES[kind](op)
    op.turns.zero_()                    # the first object's memory, still its own, gets other contents
    got, _ = other.rotate(q, start=5)
    assert torch.equal(got, want)
    assert torch.equal(op.rotate(q, start=5)[0], q)


@pytest.mark.gpu
def test_frequencies_may_be_replaced():
    op, other = Rotary(64), Rotary(64, base=500.0)
    q = torch.randn(9, 2, 64, device="cuda")
    want, _ = other.rotate(q)
    op.turns = other.turns.clone()
    assert torch.equal(op.rotate(q)[0], want)
    for wrong in (op.turns[:8], op.turns.int(), op.turns.repeat(2)[::2]):
        with pytest.raises(ValueError):
            op.turns = wrong
    assert torch.equal(op.rotate(q)[0], want)
