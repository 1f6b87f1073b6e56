"""The weights' gradients of the heads' norms over many heads and tokens, to the last head.

Heads of +-1 without eps have r = 1, and a rotation by position 0 leaves them alone: dweight is then a sum of dout x, whole
numbers of magnitude 3 or less, of fewer than 2^22 heads, so that every partial sum is a whole number below 2^24, exact in
float32 in any order.  The result has to be equal.  That r is 1, to the bit, is looked at first, in the forward call; a
reciprocal root that is not exact there (its bound is two units in the last place) leaves the sums off by at most
(2 units + the depth of the sums) 2^-24 of the magnitudes: 4 for r and its product, the heads of one group, its block's
groups, 15 rows of a warp of the join and 32 warps."""
import pytest
import torch

from paper_2609_30342_gb300 import build as pkg_build
from paper_2609_30342_gb300.layers import RotaryNorm

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
U = 2.0 ** -24
BLOCKS = 3 * 152        # of the backward call at most


@pytest.fixture(scope="module", autouse=True)
def built():
    pkg_build.build()
    yield


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _signs(*shape, seed, dtype):
    return (torch.randint(0, 2, shape, device="cuda", generator=_gen(seed)) * 2 - 1).to(dtype)


def _whole(*shape, seed, dtype):
    return torch.randint(-3, 4, shape, device="cuda", generator=_gen(seed)).to(dtype)


# blocks of one tile and of several; 8-byte and 16-byte vectors, one and two units a lane, whole heads
@pytest.mark.parametrize("tokens,q_heads,k_heads", [(1, 1, 0), (300, 3, 1), (20000, 9, 3), (16384, 12, 12), (60001, 4, 4)])
@pytest.mark.parametrize("dtype,layout,head_dim,rotary_dim", [
    ("bf16", "half", 64, 64), ("bf16", "interleaved", 128, 20), ("f16", "half", 72, 8), ("f32", "half", 64, 0),
    ("f32", "interleaved", 256, 256), ("bf16", "half", 70, 70), ("f32", "half", 33, 16), ("bf16", "interleaved", 131, 102)])
def test_every_head_counts(tokens, q_heads, k_heads, dtype, layout, head_dim, rotary_dim):
    op, t = RotaryNorm(head_dim, rotary_dim, layout=layout, eps=0.0), DT[dtype]
    q, k = _signs(tokens, q_heads, head_dim, seed=1, dtype=t), _signs(tokens, k_heads, head_dim, seed=2, dtype=t)
    dq, dk = _whole(tokens, q_heads, head_dim, seed=3, dtype=t), _whole(tokens, k_heads, head_dim, seed=4, dtype=t)
    w = torch.linspace(0.5, 2.0, head_dim, device="cuda")
    positions = torch.zeros(tokens, dtype=torch.int64, device="cuda")
    ones = torch.ones(1, 1, head_dim, device="cuda")
    one = bool((op.forward(ones, positions=positions[:1])[0] == 1).all())
    g = op.backward(dq, dk, q, k, w, w, positions=positions)
    for x, d, got in ((q, dq, g.q_weight), (k, dk, g.k_weight)):
        terms = (d.double() * x.double()).flatten(0, 1)
        want, size = terms.sum(0), terms.abs().sum(0)
        depth = tokens * (q_heads + k_heads) // BLOCKS + 128 + 15 + 32      # a group's heads: all of its block's at most
        limit = torch.zeros_like(size) if one else (4 + depth) * U * size
        assert got.dtype == torch.float32
        assert ((got.double() - want).abs() <= limit).all(), float((got.double() - want).abs().max())
        if tokens > 1 and x.shape[1]:           # a sum that lacks a token of 20 is not accepted
            lacking = terms.view(tokens, -1, head_dim)[::20].sum((0, 1))
            assert (lacking.abs() > limit).any()


def test_two_units_a_lane():
    """float32 heads of 512: a lane's two units."""
    test_every_head_counts(9001, 2, 1, "f32", "half", 512, 512)


def test_the_longest():
    """As many heads as the largest training case's: blocks of ten tiles and more."""
    test_every_head_counts(65536, 32, 8, "bf16", "half", 128, 128)
