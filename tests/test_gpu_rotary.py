"""Rotary positions on the GPU against float64.

Tolerance.  The angle is kept in units of 2^-32 of a turn, converted to float32 (half turns, a relative error of 2^-24):
at most pi 2^-24 + 2 pi 2^-32 off, and sine and cosine are a few units of 2^-24 off themselves.  An element of a turned
pair is thus off by at most 8 units of 2^-24 of magnitude (|a| + |b|), plus the output type's rounding."""
import math

import pytest
import torch

from paper_2609_30342_gb300 import build as pkg_build
from paper_2609_30342_gb300 import rikfad
from paper_2609_30342_gb300.layers import Rotary, rotary_frequencies

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_ULP = {v: torch.finfo(v).eps / 2 for v in DT.values()}


@pytest.fixture(scope="module", autouse=True)
def built():
    pkg_build.build()
    yield


def _reference(t, op, positions, inverse=False):
    """(turned values, bound on the error): t [batch, tokens, heads, head_dim], positions [batch, tokens]."""
    rot, v = op.rotary_dim, t.double().clone()
    f = torch.tensor(op.frequencies, dtype=torch.float64, device=t.device)
    angle = positions.double()[..., None, None] * f * (-1 if inverse else 1)
    c, s = torch.cos(angle) * op.magnitude, torch.sin(angle) * op.magnitude
    i = torch.arange(rot // 2, device=t.device)
    i, j = (i, i + rot // 2) if op.layout == "half" else (2 * i, 2 * i + 1)
    a, b = v[..., i], v[..., j]
    bound = torch.zeros_like(v)
    bound[..., i] = bound[..., j] = 8 * 2.0 ** -24 * abs(op.magnitude) * (a.abs() + b.abs())
    v[..., i], v[..., j] = a * c - b * s, b * c + a * s
    return v, bound + HALF_ULP[t.dtype] * (v.abs() + bound) + (2.0 ** -25 if t.dtype is torch.float16 else 2.0 ** -149)


def _check(got, src, op, positions, inverse=False):
    if src.dim() == 3:
        got, src, positions = got[None], src[None], positions[None]
    want, bound = _reference(src, op, positions.expand(src.shape[:2]), inverse)
    assert bool(((got.double() - want).abs() <= bound).all())
    rot = op.rotary_dim
    assert torch.equal(got[..., rot:], src[..., rot:])


def _heads(shape, dtype, seed=0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return torch.randn(*shape, generator=gen, device="cuda").to(DT[dtype])


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("head_dim,rotary_dim", [(64, 64), (64, 32), (80, 20), (128, 126), (2, 2), (7, 6), (5, 0), (96, 24),
                                                 (256, 256), (1, 0)])
@pytest.mark.parametrize("tokens,q_heads,k_heads", [(1, 12, 12), (37, 8, 2), (300, 1, 1)])
def test_rotation_and_inverse(layout, dtype, head_dim, rotary_dim, tokens, q_heads, k_heads):
    op = Rotary(head_dim, rotary_dim, layout=layout)
    q, k = _heads((tokens, q_heads, head_dim), dtype), _heads((tokens, k_heads, head_dim), dtype, 1)
    positions = torch.arange(tokens, device="cuda") + 5
    for inverse in (False, True):
        for kw in (dict(positions=positions), dict(positions=positions.int()), dict(start=5)):
            q2, k2 = op.rotate(q, k, inverse=inverse, **kw)
            _check(q2, q, op, positions, inverse)
            _check(k2, k, op, positions, inverse)


@pytest.mark.parametrize("positions", [[0, 1, 2], [1 << 20, (1 << 20) + 1, 3], [(1 << 31) - 1, 1 << 31, (1 << 40) + 12345],
                                       [-1, -1000, 0]])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_far_and_negative_positions(positions, layout):
    op = Rotary(64, layout=layout)
    q = _heads((3, 4, 64), "f32")
    pos = torch.tensor(positions, device="cuda")
    got, _ = op.rotate(q, positions=pos)
    # float64 angles are off by |position| 2^-52 themselves
    slack = 2.0 ** -51 * float(pos.abs().max()) * float(q.abs().max()) * 2
    want, bound = _reference(q[None], op, pos[None])
    assert bool(((got[None].double() - want).abs() <= bound + slack).all())


@pytest.mark.parametrize("scaling", [dict(kind="linear", factor=4.0), dict(kind="base", factor=8.0),
                                     dict(kind="ramp", factor=8.0, original_context=1024),
                                     dict(kind="ramp", factor=2.0, original_context=64, fast=4.0, slow=0.5)])
def test_scaled_frequencies(scaling):
    op = Rotary(64, 48, base=500000.0, layout="half", scaling=scaling)
    f, m = rotary_frequencies(48, 500000.0, scaling)
    assert f == op.frequencies and m == op.magnitude
    q = _heads((50, 3, 64), "f32")
    pos = torch.arange(50, device="cuda") * 977
    _check(op.rotate(q, positions=pos)[0], q, op, pos)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strided_heads_batches_and_offsets(layout, dtype):
    op = Rotary(64, 40, layout=layout)
    qkv = _heads((3, 17, 10 * 64 + 1), dtype)
    for offset in (0, 1):                   # 16-byte aligned heads and heads that start anywhere
        rows = qkv[:, :, offset:offset + 640]
        q, k = rows[..., :384].unflatten(2, (6, 64)), rows[..., 384:512].unflatten(2, (2, 64))
        pos = torch.arange(17, device="cuda").repeat(3, 1) + torch.tensor([[0], [100], [7]], device="cuda")
        q2, k2 = op.rotate(q, k, positions=pos)
        _check(q2, q, op, pos)
        _check(k2, k, op, pos)
        q3, _ = op.rotate(q, positions=pos[1].contiguous())
        _check(q3, q, op, pos[1:2])
        # heads before tokens: [batch, heads, tokens, d] seen as [batch, tokens, heads, d]
        t = q.transpose(1, 2).contiguous().transpose(1, 2)
        out = torch.zeros_like(t)
        op.rotate(t, positions=pos, out=(out, None))
        _check(out, q, op, pos)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_in_place_leaves_the_rest_alone(layout):
    op = Rotary(64, 32, layout=layout)
    qkv = _heads((21, 6 * 64), "bf16")
    keep = qkv.clone()
    q, k = qkv[:, :192].unflatten(1, (3, 64)), qkv[:, 192:320].unflatten(1, (2, 64))
    op.rotate(q, k, out=(q, k))
    pos = torch.arange(21, device="cuda")
    _check(q, keep[:, :192].unflatten(1, (3, 64)), op, pos)
    _check(k, keep[:, 192:320].unflatten(1, (2, 64)), op, pos)
    assert torch.equal(qkv[:, 320:], keep[:, 320:])


def test_offsets_beyond_32_bits():
    op = Rotary(64)
    big = torch.empty((1 << 31) + (1 << 20), dtype=torch.bfloat16, device="cuda")
    q = torch.as_strided(big, (3, 2, 64), (1 << 30, 1 << 19, 1))
    q.copy_(_heads((3, 2, 64), "bf16"))
    pos = torch.arange(3, device="cuda")
    _check(op.rotate(q, positions=pos)[0], q, op, pos)


def test_empty():
    op = Rotary(64)
    for shape in ((0, 4, 64), (5, 0, 64), (2, 0, 4, 64)):
        q = torch.empty(shape, device="cuda")
        assert op.rotate(q)[0].shape == q.shape


def test_special_values_stay_in_their_pair():
    op = Rotary(8, layout="half")
    q = torch.ones(2, 3, 8, device="cuda")
    q[1, 2, 1] = float("nan")
    q[0, 0, 3] = float("inf")
    got, _ = op.rotate(q)
    bad = ~got.isfinite()
    want = torch.zeros_like(bad)
    want[1, 2, [1, 5]] = True
    want[0, 0, [3, 7]] = True           # position 0: inf cos 0 = inf, inf sin 0 = nan
    assert torch.equal(bad, want)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_autograd_against_the_formula_and_differences(layout):
    op = Rotary(16, 12, layout=layout, magnitude=1.25)
    q = _heads((9, 2, 16), "f32").requires_grad_()
    k = _heads((9, 1, 16), "f32", 1).requires_grad_()
    pos = torch.arange(9, device="cuda") * 3
    wq, wk = _heads((9, 2, 16), "f32", 2), _heads((9, 1, 16), "f32", 3)

    def loss(a, b):
        x, y = op(a, b, positions=pos)
        return (x.double() * wq).sum() + (y.double() * wk).sum()

    dq, dk = torch.autograd.grad(loss(q, k), (q, k))
    _check(dq, wq, op, pos, inverse=True)
    _check(dk, wk, op, pos, inverse=True)
    direction = _heads((9, 2, 16), "f32", 4)
    with torch.no_grad():                   # linear: a central difference is exact up to rounding
        diff = float(loss(q + direction, k) - loss(q - direction, k)) / 2
    assert abs(diff - float((dq.double() * direction).sum())) <= 1e-4 * float((wq.abs() * direction.abs()).sum())


def test_streams():
    op = Rotary(64)
    q = _heads((4000, 4, 64), "bf16")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out = torch.zeros_like(q)
    op.rotate(q, out=(out, None), stream=s)
    s.synchronize()
    _check(out, q, op, torch.arange(4000, device="cuda"))


def test_refusals():
    op = Rotary(64)
    q = torch.zeros(4, 2, 64, device="cuda")
    for bad in (torch.zeros(4, 2, 64), torch.zeros(4, 2, 32, device="cuda"), torch.zeros(4, 64, device="cuda"),
                torch.zeros(4, 2, 64, dtype=torch.float64, device="cuda"),
                torch.zeros(4, 2, 128, device="cuda")[..., ::2]):
        with pytest.raises(ValueError):
            op.rotate(bad)
    for k in (q.bfloat16(), q[:3], torch.zeros(4, 2, 64)):
        with pytest.raises(ValueError):
            op.rotate(q, k)
    for positions in (torch.zeros(3, dtype=torch.int64, device="cuda"), torch.zeros(4, device="cuda"),
                      torch.zeros(4, dtype=torch.int64)):
        with pytest.raises(ValueError):
            op.rotate(q, positions=positions)
    with pytest.raises(rikfad.RikfadError) as e:         # in place with other strides
        t = torch.zeros(4, 4, 64, device="cuda")
        op.rotate(t, out=(t.transpose(0, 1), None))
    assert e.value.code == rikfad.ERR_ARG
