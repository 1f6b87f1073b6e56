"""The heads' norms with rotation on the GPU against float64.

Tolerance (U = 2^-24).  A sum of d squares is off by (d + 1) U, its root by half of that; the reciprocal root is off by two
units in the last place (4 U) and takes an addition and a product before it: r is off by R = (d / 2 + 8) U.  A value times
r and a weight takes two more roundings.  Cosines and sines of an angle leave an element of a turned pair off by at most
8 U of magnitude (|a| + |b|) (see the rotary tests).  Backward, the turned gradient dy is off by that; the sum of g x adds
(d + 3) U of its magnitudes; a sum over n heads and tokens n U of its magnitudes at most.  Then the type's rounding."""
import pytest
import torch

from paper_2609_30342_gb300 import build as pkg_build
from paper_2609_30342_gb300 import rikfad
from paper_2609_30342_gb300.layers import Rotary, RotaryNorm

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_ULP = {v: torch.finfo(v).eps / 2 for v in DT.values()}
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -25}
U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def built():
    pkg_build.build()
    yield


def _rand(*shape, seed=0, dtype=torch.float32, scale=1.0):
    return (torch.randn(shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)) * scale).to(dtype)


def _pairs(op, device):
    i = torch.arange(op.rotary_dim // 2, device=device)
    return (i, i + op.rotary_dim // 2) if op.layout == "half" else (2 * i, 2 * i + 1)


def _turn(v, op, positions, inverse=False):
    """(turned values, |a| + |b| of every element's pair times the magnitude): positions of v's leading sizes."""
    f = torch.tensor(op.frequencies, dtype=torch.float64, device=v.device)
    angle = positions.double()[..., None, None] * f * (-1 if inverse else 1)
    c, s = torch.cos(angle) * op.magnitude, torch.sin(angle) * op.magnitude
    i, j = _pairs(op, v.device)
    a, b = v[..., i], v[..., j]
    out, size = v.clone(), v.abs()
    out[..., i], out[..., j] = a * c - b * s, b * c + a * s
    size[..., i] = size[..., j] = abs(op.magnitude) * (a.abs() + b.abs())
    return out, size


def _close(got, want, bound):
    bound = bound + HALF_ULP[got.dtype] * (want.abs() + bound) + TINY[got.dtype]
    assert ((got.double() - want).abs() <= bound).all(), float(((got.double() - want).abs() / bound).max())


def _check(op, x, weight, positions, out=None, dout=None, dx=None, dw=None):
    d, v = op.head_dim, x.double()
    w = torch.ones(d, dtype=torch.float64, device="cuda") if weight is None else weight.double()
    r = torch.rsqrt((v * v).mean(-1, keepdim=True) + op.eps)
    off = (d / 2 + 8) * U
    positions = positions.expand(x.shape[:-2])
    if out is not None:
        want, size = _turn(v * r * w, op, positions)
        _close(out, want, (off + 12 * U) * size)
    if dout is None:
        return
    dy, size = _turn(dout.double(), op, positions, inverse=True)
    e = 8 * U * size
    g, y = dy * w, v * r
    mean = (g * y).mean(-1, keepdim=True)
    spread = ((e * w.abs() * y.abs()).mean(-1, keepdim=True) + (d + 3) * U * (g * y).abs().mean(-1, keepdim=True)
              + (2 * off + 8 * U) * mean.abs())
    want = r * (g - y * mean)
    bound = r * (e * w.abs() + 4 * U * g.abs() + y.abs() * (spread + 4 * U * mean.abs())) \
        + (off + 4 * U) * r * (g.abs() + (y * mean).abs())
    _close(dx, want, bound)
    if weight is not None:
        rows = v.numel() // d
        terms, errors = (dy * y).reshape(-1, d), (e * y.abs() + (off + 4 * U) * (dy * y).abs()).reshape(-1, d)
        _close(dw, terms.sum(0), errors.sum(0) + rows * U * terms.abs().sum(0))


SIZES = [(64, 64), (64, 20), (128, 128), (80, 40), (96, 36), (70, 70), (17, 8), (17, 16), (131, 102), (256, 256),
         (1, 0), (2, 2), (33, 0), (512, 512), (511, 510), (512, 6), (200, 50)]


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("head_dim,rotary_dim", SIZES)
def test_sizes(head_dim, rotary_dim, layout, dtype):
    op = RotaryNorm(head_dim, rotary_dim, layout=layout, magnitude=1.25)
    t = DT[dtype]
    q, k = _rand(37, 6, head_dim, seed=1, dtype=t, scale=3.0), _rand(37, 2, head_dim, seed=2, dtype=t, scale=0.1)
    dq, dk = _rand(37, 6, head_dim, seed=3, dtype=t), _rand(37, 2, head_dim, seed=4, dtype=t)
    qw, kw = _rand(head_dim, seed=5), _rand(head_dim, seed=6)
    positions = torch.randint(0, 1 << 20, (37,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(7))
    a, b = op.forward(q, k, qw, kw, positions)
    g = op.backward(dq, dk, q, k, qw, kw, positions)
    _check(op, q, qw, positions, a, dq, g.q, g.q_weight)
    _check(op, k, kw, positions, b, dk, g.k, g.k_weight)


@pytest.mark.parametrize("tokens,q_heads,k_heads", [(1, 1, 1), (1, 128, 8), (3, 5, 0), (1000, 1, 1), (4097, 12, 12), (20000, 9, 3)])
def test_many_heads_and_tokens(tokens, q_heads, k_heads):
    op = RotaryNorm(64, eps=1e-5)
    q, k = _rand(tokens, q_heads, 64, seed=1, dtype=torch.bfloat16), _rand(tokens, k_heads, 64, seed=2, dtype=torch.bfloat16)
    dq, dk = _rand(tokens, q_heads, 64, seed=3, dtype=torch.bfloat16), _rand(tokens, k_heads, 64, seed=4, dtype=torch.bfloat16)
    qw, kw = _rand(64, seed=5, dtype=torch.bfloat16), _rand(64, seed=6, dtype=torch.bfloat16)
    at = torch.arange(11, tokens + 11, device="cuda")
    a, b = op.forward(q, k, qw, kw, start=11)
    g = op.backward(dq, dk, q, k, qw, kw, start=11)
    _check(op, q, qw, at, a, dq, g.q, g.q_weight)
    _check(op, k, kw, at, b, dk, g.k, g.k_weight)
    again = op.backward(dq, dk, q, k, qw, kw, start=11)
    assert all(torch.equal(x, y) for x, y in zip(g, again))


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("positions_dtype", [torch.int32, torch.int64, None])
@pytest.mark.parametrize("batch,tokens", [(3, 1), (3, 50), (64, 1), (2, 700)])
def test_batches(batch, tokens, positions_dtype, shared):
    op = RotaryNorm(80, 40, layout="interleaved")
    q, dq = _rand(batch, tokens, 4, 80, seed=1), _rand(batch, tokens, 4, 80, seed=2)
    w = _rand(80, seed=3)
    if positions_dtype is None:
        positions, at = None, torch.arange(5, 5 + tokens, device="cuda")
    else:
        shape = (tokens,) if shared else (batch, tokens)
        positions = at = torch.randint(-100, 5000, shape, device="cuda", dtype=positions_dtype)
    a, none = op.forward(q, q_weight=w, positions=positions, start=5)
    g = op.backward(dq, None, q, q_weight=w, positions=positions, start=5)
    assert none is None and g.k is None and g.k_weight is None
    _check(op, q, w, at, a, dq, g.q, g.q_weight)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shift", [0, 1, 4])
def test_strided_heads(shift, dtype):
    """Queries and keys inside a wider projection, transposed heads, tensors that start anywhere, weights absent."""
    t, op = DT[dtype], RotaryNorm(64, 32)
    big = _rand(211 * 10 * 64 + 8, seed=1, dtype=t)[shift:shift + 211 * 640].view(211, 10, 64)
    q, k = big[:, :6], big[:, 6:8]
    dq = _rand(6, 211, 64, seed=2, dtype=t).transpose(0, 1)
    at = torch.arange(211, device="cuda")
    a, b = op.forward(q, k)
    _check(op, q, None, at, a)
    _check(op, k, None, at, b)
    g = op.backward(dq, None, q, k)
    _check(op, q, None, at, None, dq, g.q)
    assert g.k is None and g.q_weight is None


def test_in_place():
    op = RotaryNorm(64)
    q, k, w = _rand(100, 4, 64, dtype=torch.bfloat16), _rand(100, 2, 64, seed=1, dtype=torch.bfloat16), _rand(64, seed=2)
    want = op.forward(q, k, w, w)
    got = op.forward(q, k, w, w, out=(q, k))
    assert got[0] is q and torch.equal(q, want[0]) and torch.equal(k, want[1])


@pytest.mark.parametrize("over", ["x", "dout"])
@pytest.mark.parametrize("head_dim,rotary_dim", [(64, 64), (80, 40), (70, 70), (131, 102)])
def test_gradients_over_their_inputs(head_dim, rotary_dim, over):
    """dx may be x or dout: the same results to the bit."""
    op = RotaryNorm(head_dim, rotary_dim)
    q, dq = _rand(300, 5, head_dim, seed=1, dtype=torch.bfloat16), _rand(300, 5, head_dim, seed=2, dtype=torch.bfloat16)
    w = _rand(head_dim, seed=3)
    want = op.backward(dq, None, q, q_weight=w)
    first = device, dtype, lead, batch, tokens = op._lead(q)
    strides, dw, to = op._dense(tokens, 5), torch.empty_like(w), q if over == "x" else dq
    lists = (q.data_ptr(), dq.data_ptr(), w.data_ptr(), to.data_ptr(), dw.data_ptr(), 5, *strides, *strides, *strides)
    lib = rikfad.lib()
    nbytes = lib.rikfad_rotary_norm_workspace(op._block(first, None, 0, torch.float32, lists))
    work = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    rikfad._check(lib.rikfad_rotary_norm_backward(
        op._block(first, None, 0, torch.float32, lists, (work.data_ptr(), nbytes)), rikfad._raw_stream(0)))
    assert torch.equal(to, want.q) and torch.equal(dw, want.q_weight)


@pytest.mark.parametrize("shape", [(0, 2, 64), (2, 0, 2, 64), (0, 3, 2, 64), (3, 0, 64)])
def test_empty(shape):
    q, k = (torch.empty(shape, dtype=torch.bfloat16, device="cuda", requires_grad=True) for _ in range(2))
    w = torch.ones(64, device="cuda", requires_grad=True)
    a, b = RotaryNorm(64)(q, k, w, w)
    assert a.shape == b.shape == q.shape
    dq, dk, dw = torch.autograd.grad(a.sum() + b.sum(), (q, k, w))
    assert dq.shape == q.shape and dk.shape == k.shape and torch.equal(dw, torch.zeros_like(w))


def test_without_turns_and_weights_is_a_norm():
    op = RotaryNorm(64, 0)
    q = _rand(50, 3, 64, dtype=torch.bfloat16, scale=20.0)
    a, _ = op.forward(q)
    rms = (a.double() ** 2).mean(-1).sqrt()
    assert ((rms - 1).abs() <= 2.0 ** -7).all()
    _check(op, q, None, torch.zeros(50, device="cuda"), a)


def test_zeros_and_non_finite_heads():
    op, w = RotaryNorm(32, eps=1e-6), _rand(32, seed=1)
    q = _rand(6, 2, 32, seed=2)
    want = op.forward(q, q_weight=w)[0]
    q[1, 0], q[2, 1, 5], q[3, 0, 0] = 0.0, float("nan"), float("inf")
    got = op.forward(q, q_weight=w)[0]
    assert (got[1, 0] == 0).all() and got[2, 1].isnan().all() and not got[3, 0].isfinite().all()
    keep = torch.ones(6, 2, dtype=torch.bool, device="cuda")
    keep[1, 0] = keep[2, 1] = keep[3, 0] = False
    assert torch.equal(got[keep], want[keep])


def test_autograd_and_differences():
    op = RotaryNorm(48, 32, layout="interleaved", magnitude=1.1)
    q, k = _rand(9, 3, 48, seed=1).requires_grad_(), _rand(9, 1, 48, seed=2).requires_grad_()
    w = _rand(48, seed=3).requires_grad_()          # one weight for both: its gradients add up
    dq, dk = _rand(9, 3, 48, seed=4), _rand(9, 1, 48, seed=5)
    a, b = op(q, k, w, w)
    got = torch.autograd.grad((a * dq).sum() + (b * dk).sum(), (q, k, w))
    explicit = op.backward(dq, dk, q.detach(), k.detach(), w.detach(), w.detach())
    assert torch.equal(got[0], explicit.q) and torch.equal(got[1], explicit.k)
    assert torch.equal(got[2], explicit.q_weight + explicit.k_weight)
    # Central differences along one direction, with the function in float64: the step's error is of order 1e-8 of the
    # third derivative, the operator's gradients are off by some 1e-6 of their sizes.
    at = torch.arange(9, device="cuda")
    step = [_rand(*t.shape, seed=6 + i).double() for i, t in enumerate((q, k, w))]

    def value(h):
        x, y, v = (t.detach().double() + h * s for t, s in zip((q, k, w), step))
        total = 0
        for t, d in ((x, dq), (y, dk)):
            n = t * torch.rsqrt((t * t).mean(-1, keepdim=True) + op.eps) * v
            total = total + float((_turn(n, op, at)[0] * d.double()).sum())
        return total

    h = 1e-4
    want = (value(h) - value(-h)) / (2 * h)
    have = sum(float((g.double() * s).sum()) for g, s in zip(got, step))
    size = sum(float((g.double() * s).abs().sum()) for g, s in zip(got, step))
    assert abs(have - want) <= 1e-5 * size
    one, = torch.autograd.grad(op(q, k, w, w)[1].sum(), k)       # the queries' output is not used
    assert one.shape == k.shape
    again, = torch.autograd.grad((op(q, None, w)[0] ** 2).sum(), q, create_graph=True)
    with pytest.raises(RuntimeError):
        again.sum().backward()


def test_agrees_with_rotary():
    """A head whose mean square is one, without eps: the norm does nothing, and the rotation is Rotary's."""
    q = _rand(40, 3, 64, seed=1).sign()
    positions = torch.randint(0, 1 << 20, (40,), device="cuda")
    a, _ = RotaryNorm(64, eps=0.0).forward(q, positions=positions)
    b, _ = Rotary(64).rotate(q, positions=positions)
    assert ((a - b).abs() <= 8 * U).all()


def test_far_heads():
    """Tensors beyond 2^31 elements."""
    op = RotaryNorm(128)
    q = torch.empty(140000, 128, 128, dtype=torch.bfloat16, device="cuda")
    q[-1], q[0] = _rand(128, 128, seed=1), 1
    out, _ = op.forward(q, start=3)
    _check(op, q[-1:], None, torch.tensor([140002], device="cuda"), out[-1:])
    g = op.backward(q, None, q, start=3)
    _check(op, q[-1:], None, torch.tensor([140002], device="cuda"), None, q[-1:], g.q[-1:])


def test_refusals():
    op = RotaryNorm(64)
    q, k, w = _rand(5, 2, 64), _rand(5, 1, 64), _rand(64)
    for call in (lambda: op.forward(q.cpu()), lambda: op.forward(q, k.bfloat16()), lambda: op.forward(q, k[:4]),
                 lambda: op.forward(q, None, w, w), lambda: op.forward(q, k, w, w.bfloat16()), lambda: op.forward(q, k, w[:63]),
                 lambda: op.forward(q, k, w.double()), lambda: op.forward(q, k, w.cpu()), lambda: op.forward(q[..., :32]),
                 lambda: op.forward(q.double()), lambda: op.forward(q, positions=torch.arange(5)),
                 lambda: op.forward(q, positions=torch.arange(4, device="cuda")), lambda: op.forward(q, out=(k, None)),
                 lambda: op.forward(q.transpose(1, 2).contiguous().transpose(1, 2)), lambda: op.forward(3),
                 lambda: op.backward(q, k, q), lambda: op.backward(k, None, q), lambda: op.backward(q.bfloat16(), None, q),
                 lambda: op.backward(q.cpu(), None, q)):
        with pytest.raises(ValueError):
            call()
    for kw in (dict(head_dim=513), dict(head_dim=0), dict(head_dim=64, eps=-1.0), dict(head_dim=64, eps=float("nan")),
               dict(head_dim=64, rotary_dim=66), dict(head_dim=64, rotary_dim=3), dict(head_dim=64, layout="none")):
        with pytest.raises(ValueError):
            RotaryNorm(**kw)
