"""The training step's operators on a stream other than the current one: what a call allocates there must not be memory
that work of the current stream, enqueued earlier, still writes to."""
import pytest
import torch

from paper_2609_30342_gb300 import build as pkg_build
from paper_2609_30342_gb300.gradients import GradientClipper
from paper_2609_30342_gb300.layers import ResidualNorm, Rotary

pytestmark = pytest.mark.gpu

ROWS, COLS = 512, 768


@pytest.fixture(scope="module", autouse=True)
def built():
    pkg_build.build()
    yield


def _busy(sizes):
    """Enqueues late writes to blocks of these sizes, and frees the blocks: the current stream may have them again."""
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    blocks = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes]
    torch.cuda._sleep(100_000_000)
    for b in blocks:
        b.fill_(0x5a)
    del blocks


def _inputs(*shapes):
    g = torch.Generator(device="cuda").manual_seed(3)
    return [torch.randn(s, device="cuda", generator=g).bfloat16() for s in shapes]


@pytest.mark.parametrize("raw", [False, True])
def test_residual_norm(raw):
    x, z, du, dh = _inputs(*[(ROWS, COLS)] * 4)
    w, = _inputs((COLS,))
    op = ResidualNorm(COLS, post="rms", pre="rms")

    def run(s):
        u, h, stats = op.forward(x, z, post_weight=w, pre_weight=w, stream=s)
        return u, h, *[t for t in op.backward(du, dh, x, z, post_weight=w, pre_weight=w, stats=stats, stream=s)
                       if t is not None]

    want = [t.clone() for t in run(None)]
    side = torch.cuda.Stream()
    _busy([2 * ROWS * COLS] * 4 + [16 * ROWS] + [2 * COLS] * 2 + [1 << 23])
    got = run(side.cuda_stream if raw else side)
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("raw", [False, True])
def test_rotary(raw):
    q, k = _inputs((ROWS, 12, 64), (ROWS, 4, 64))
    op = Rotary(64)
    want = [t.clone() for t in op.rotate(q, k)]
    side = torch.cuda.Stream()
    _busy([2 * ROWS * 12 * 64, 2 * ROWS * 4 * 64])
    got = op.rotate(q, k, stream=side.cuda_stream if raw else side)
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("raw", [False, True])
def test_gradient_norms(raw):
    grads = _inputs((ROWS, COLS), (COLS,))
    clipper = GradientClipper([t.numel() for t in grads], "bf16")
    want = [t.clone() for t in clipper.norm(grads)]
    side = torch.cuda.Stream()
    _busy([4, 8])
    got = clipper.norm(grads, stream=side.cuda_stream if raw else side)
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_inputs_are_checked_before_the_stream_is_taken():
    side = torch.cuda.Stream()
    with pytest.raises(ValueError):
        ResidualNorm(COLS).forward(torch.zeros(2, COLS), stream=side)
    with pytest.raises(ValueError):
        Rotary(64).rotate(torch.zeros(2, 1, 64), stream=side)
