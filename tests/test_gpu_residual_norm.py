"""The residual sum with its norms on the GPU, forward and backward, against float64.

Tolerances.  With e = 2^-24, every float32 operation is off by e of its result, and a sum over a row or over rows by
(chain + 16) e of the sum of its terms' sizes, where chain is the number of terms that one thread adds, at most
count / 8 + 8.  Subtracting a mean magnifies the error of v by r |v| (r: 1 / deviation).  The bounds below follow
the formulas with these sizes taken as maxima over a row (K e = 64 e for its handful of operations and sums), and end in
the output type's own rounding."""
import itertools

import pytest
import torch

from paper_2609_30342_gb300 import build as pkg_build
from paper_2609_30342_gb300 import rikfad
from paper_2609_30342_gb300.layers import ResidualNorm

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_ULP = {v: torch.finfo(v).eps / 2 for v in DT.values()}
NAMES = ("gate", "post_weight", "post_bias", "pre_weight", "pre_bias")


@pytest.fixture(scope="module", autouse=True)
def built():
    pkg_build.build()
    yield


def _inputs(rows, cols, dtype="bf16", residual="same", params="f32", post="rms", pre="rms", gate="none", gate_rows=1,
            z=True, seed=0, bias=None, weights=True):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt = DT[dtype]
    rt = torch.float32 if residual == "f32" else dt
    pt = torch.float32 if params == "f32" else dt

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    t = dict(x=(1.5 * normal(rows, cols) + 0.3).to(rt), z=(0.7 * normal(rows, cols) - 0.2).to(dt) if z else None)
    t["gate"] = None if gate == "none" else normal(rows // gate_rows, cols).to(pt if gate == "shared" else dt)
    for side, kind in (("post", post), ("pre", pre)):
        t[side + "_weight"] = (1 + 0.2 * normal(cols)).to(pt) if kind and weights else None
        t[side + "_bias"] = (0.3 * normal(cols)).to(pt) if (kind == "layer" if bias is None else bias and kind) else None
    t["du"], t["dh"] = (0.3 * normal(rows, cols)).to(rt), (0.3 * normal(rows, cols)).to(dt)
    return t


def _norm64(v, kind, w, b, eps):
    """(normed and scaled, y, r, scale of the values whose error the norm magnifies)."""
    if kind is None:
        return v, None, None
    c = v - v.mean(1, keepdim=True) if kind == "layer" else v
    r = torch.rsqrt((c * c).mean(1, keepdim=True) + eps)
    y = c * r
    n = y if w is None else y * w
    return n if b is None else n + b, y, r


def _mx(v):
    return v.abs().amax(1, keepdim=True) if v.shape[0] else v.new_zeros(0, 1)


def reference(op, t, gate_rows=1):
    """Float64 results and bounds of the float32 computation, before the outputs' rounding."""
    d = {k: None if v is None else v.double() for k, v in t.items()}
    x, z, a, b = d["x"], d["z"], op.residual_scale, op.branch_scale
    rows, cols = x.shape
    K = (64 + cols / 8) * E                 # a handful of operations and one sum over a row
    one = x.new_ones(rows, 1)
    w2 = x.new_ones(cols) if d["post_weight"] is None else d["post_weight"]
    w1 = x.new_ones(cols) if d["pre_weight"] is None else d["pre_weight"]
    ref, tol = {}, {}
    gate = None if d["gate"] is None else d["gate"].repeat_interleave(gate_rows, 0)
    g = x.new_ones(1) if gate is None else gate
    y2 = r2 = None
    if z is None:
        n = en = torch.zeros_like(x)
    else:
        n, y2, r2 = _norm64(z, op.post, d["post_weight"], d["post_bias"], op.post_eps)
        if op.post is None:
            en, ey2 = torch.zeros_like(n), 0 * one
        else:
            ey2 = K * (_mx(y2) + r2 * _mx(z))
            en = w2.abs() * ey2 + 4 * E * (n.abs() + (w2 * y2).abs())
    u = a * x + b * g * n
    eu = abs(b) * g.abs() * en + 4 * E * (abs(a) * x.abs() + abs(b) * (g * n).abs())
    h, y1, r1 = _norm64(u, op.pre, d["pre_weight"], d["pre_bias"], op.pre_eps)
    if op.pre is None:
        eh = eu
    else:
        ey1 = 2 * r1 * _mx(eu) * (1 + _mx(y1) ** 2) + K * (_mx(y1) + r1 * _mx(u))
        eh = w1.abs() * ey1 + 4 * E * (h.abs() + (w1 * y1).abs())
    ref.update(u=u, h=h)
    tol.update(u=eu, h=eh)
    du = torch.zeros_like(x) if d["du"] is None else d["du"]
    dh = torch.zeros_like(x) if d["dh"] is None else d["dh"]

    def back(gv, egv, y, ey, r, kind):
        """Gradient of a norm's input and its bound; gv the weighted gradient of its output."""
        m = (gv * y).mean(1, keepdim=True)
        m0 = gv.mean(1, keepdim=True) if kind == "layer" else 0 * one
        v = r * (gv - m0 - y * m)
        top, ytop = _mx(gv), _mx(y)
        ev = r * (_mx(egv) * (2 + ytop ** 2) + 3 * ey * top * (1 + ytop) + 2 * K * top * (1 + ytop ** 2))
        return v, ev + 2 * K * _mx(v) + _mx(v) * (ey * (1 + ytop))

    if op.pre is None:
        e, ee = du + dh, 4 * E * (du.abs() + dh.abs())
    else:
        v, ev = back(dh * w1, E * (dh * w1).abs(), y1, ey1, r1, op.pre)
        e, ee = du + v, ev + 4 * E * (du.abs() + v.abs())
    ref["x"], tol["x"] = a * e, abs(a) * ee + 2 * E * (a * e).abs()
    chain = (rows / 8 + 64) * E
    sums = {}
    if op.pre is not None:
        sums["pre_weight"] = (dh * y1, dh.abs() * ey1)
        sums["pre_bias"] = (dh, 0 * dh)
    if z is not None:
        q, eq = b * g * e, abs(b) * g.abs() * ee + 2 * E * (b * g * e).abs()
        if op.post is None:
            ref["z"], tol["z"] = q, eq
        else:
            sums["post_weight"] = (q * y2, eq * y2.abs() + q.abs() * ey2)
            sums["post_bias"] = (q, eq)
            ref["z"], tol["z"] = back(q * w2, eq * w2.abs() + 2 * E * (q * w2).abs(), y2, ey2, r2, op.post)
        if gate is not None:
            dg, edg = b * e * n, abs(b) * (ee * n.abs() + e.abs() * en) + 4 * E * (b * e * n).abs()
            split = (rows // gate_rows, gate_rows, cols)
            ref["gate"] = dg.view(split).sum(1)
            tol["gate"] = edg.view(split).sum(1) + (gate_rows / 8 + 64) * E * dg.abs().view(split).sum(1)
    for k, (v, ev) in sums.items():
        if d[k] is not None:
            ref[k], tol[k] = v.sum(0), ev.sum(0) + chain * v.abs().sum(0)
    return ref, tol


def check(name, got, ref, tol):
    err = (got.double() - ref).abs()
    tiny = 2.0 ** -25 if got.dtype is torch.float16 else 2.0 ** -149
    bound = tol + HALF_ULP[got.dtype] * (ref.abs() + tol) + tiny
    assert got.shape == ref.shape, name
    bad = ~(err <= bound)
    assert not bool(bad.any()), "%s: %d beyond, worst %g of its bound" % (name, int(bad.sum()), float((err / bound).max()))


def run(op, t, gate_rows=1):
    weights = {k: t[k] for k in NAMES}
    u, h, stats = op.forward(t["x"], t["z"], **weights)
    g = op.backward(t["du"], t["dh"], t["x"], t["z"], stats=stats, **weights)
    ref, tol = reference(op, t, gate_rows)
    check("u", u, ref["u"], tol["u"])
    check("h", h, ref["h"], tol["h"])
    for k in ("x", "z") + NAMES:
        if t[k] is None:
            assert getattr(g, k) is None
        else:
            check("d" + k, getattr(g, k), ref[k], tol[k])
    return u, h, g


KINDS = [None, "rms", "layer"]


@pytest.mark.parametrize("post,pre", list(itertools.product(KINDS, KINDS)))
@pytest.mark.parametrize("gate,gate_rows", [("none", 1), ("rows", 1), ("shared", 6), ("shared", 1), ("shared", 24)])
@pytest.mark.parametrize("cols", [64, 129])
def test_kinds_and_gates(post, pre, gate, gate_rows, cols):
    op = ResidualNorm(cols, post=post, pre=pre, residual_scale=1.2, branch_scale=-0.7, post_eps=1e-5)
    run(op, _inputs(24, cols, "f32", post=post, pre=pre, gate=gate, gate_rows=gate_rows), gate_rows)


@pytest.mark.parametrize("dtype,residual,params", [("f32", "same", "f32"), ("bf16", "same", "f32"), ("bf16", "f32", "same"),
                                                   ("f16", "same", "same"), ("f16", "f32", "f32"), ("bf16", "f32", "f32")])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 768), (3, 7), (5, 8), (2, 31), (17, 33), (300, 48), (700, 256), (33, 257),
                                       (40, 1001), (9, 1600), (6, 4095), (5, 4104), (3, 8200), (2, 16391), (2, 32768)])
def test_types_and_sizes(dtype, residual, params, rows, cols):
    op = ResidualNorm(cols, post="layer", pre="rms")
    run(op, _inputs(rows, cols, dtype, residual, params, post="layer", pre="rms", gate="rows"))


@pytest.mark.parametrize("rows,gate_rows", [(5000, 1), (5000, 5000), (5000, 1000), (5001, 3), (4998, 17), (40000, 10000)])
@pytest.mark.parametrize("gate", ["rows", "shared"])
def test_many_rows(rows, gate_rows, gate):
    if gate == "rows":
        gate_rows = 1
    op = ResidualNorm(96, post="rms", pre="layer")
    run(op, _inputs(rows, 96, "bf16", post="rms", pre="layer", gate=gate, gate_rows=gate_rows), gate_rows)


@pytest.mark.parametrize("rows,gate_rows", [(1400, 1400), (1400, 700), (1400, 28), (1400, 7), (1398, 3), (1398, 1), (40, 20)])
@pytest.mark.parametrize("cols", [37, 129, 1001, 1002, 1004, 2500])
@pytest.mark.parametrize("gate", ["rows", "shared"])
def test_odd_widths_and_gates(rows, gate_rows, cols, gate):
    """Rows that start anywhere, with sums over the rows of gates that last short and long."""
    if gate == "rows":
        gate_rows = 1
    op = ResidualNorm(cols, post="rms", pre="layer")
    run(op, _inputs(rows, cols, "f16", "f32", post="rms", pre="layer", gate=gate, gate_rows=gate_rows), gate_rows)


@pytest.mark.parametrize("cols", [129, 1001, 4104, 9001, 20003])
def test_odd_widths_in_wider_rows(cols):
    """Row strides that drift by the same number of elements, and by different ones."""
    op = ResidualNorm(cols, post="layer", pre="rms")
    for pads in ((3, 3, 3, 3, 3), (0, 8, 16, 0, 8), (0, 1, 2, 3, 4)):
        t = _inputs(21, cols, "bf16", post="layer", pre="rms", gate="rows", bias=True)
        for k, pad in zip(("x", "z", "gate", "du", "dh"), pads):
            wide = torch.full((21, cols + pad), float("nan"), dtype=t[k].dtype, device="cuda")
            wide[:, :cols] = t[k]
            t[k] = wide[:, :cols]
        run(op, t)


@pytest.mark.parametrize("cols", [72, 1001])
def test_a_shared_gate_without_its_gradient(cols):
    """Through the C entry: dgate and other outputs may be left out."""
    from paper_2609_30342_gb300 import layers
    op = ResidualNorm(cols, post="rms", pre="rms")
    t = _inputs(60, cols, "bf16", gate="shared", gate_rows=20)
    weights = {k: t[k] for k in NAMES}
    _, _, stats = op.forward(t["x"], t["z"], **weights)
    full = op.backward(t["du"], t["dh"], t["x"], t["z"], stats=stats, **weights)
    head = op._inputs(t["x"], t["z"], t["gate"], tuple(t[k] for k in NAMES[1:]), None)[0]
    dz = torch.zeros_like(t["z"])
    block = layers._NORM.pack(*head, 0, 0, 0, 0, stats.data_ptr(), t["du"].data_ptr(), cols, t["dh"].data_ptr(), cols,
                              0, 0, dz.data_ptr(), cols, 0, 0, 0, 0, 0, 0, 0, 0)
    assert rikfad.lib().rikfad_residual_norm_workspace(block) == 0
    assert rikfad.lib().rikfad_residual_norm_backward(block, torch.cuda.current_stream().cuda_stream) == rikfad.OK
    torch.cuda.synchronize()
    assert torch.equal(dz, full.z)


@pytest.mark.parametrize("pre", KINDS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_without_a_branch(pre, dtype):
    op = ResidualNorm(200, pre=pre, residual_scale=0.5)
    run(op, _inputs(11, 200, dtype, post=None, pre=pre, z=False))


@pytest.mark.parametrize("bias,weights", [(True, False), (False, False), (True, True)])
def test_weights_and_biases_are_optional(bias, weights):
    op = ResidualNorm(72, post="rms", pre="layer")
    run(op, _inputs(10, 72, "f32", post="rms", pre="layer", bias=bias, weights=weights))


@pytest.mark.parametrize("none", ["du", "dh"])
@pytest.mark.parametrize("cols", [128, 1001])
def test_one_gradient_may_be_absent(none, cols):
    op = ResidualNorm(cols, post="layer", pre="layer")
    t = _inputs(13, cols, "f32", post="layer", pre="layer", gate="rows")
    weights = {k: t[k] for k in NAMES}
    _, _, stats = op.forward(t["x"], t["z"], **weights)
    t[none] = None
    g = op.backward(t["du"], t["dh"], t["x"], t["z"], stats=stats, **weights)
    ref, tol = reference(op, t)
    for k in ("x", "z") + NAMES:
        check("d" + k, getattr(g, k), ref[k], tol[k])


def test_no_rows():
    op = ResidualNorm(64, post="layer", pre="rms")
    t = _inputs(0, 64, "bf16", post="layer", pre="rms")
    weights = {k: t[k] for k in NAMES}
    u, h, stats = op.forward(t["x"], t["z"], **weights)
    assert u.shape == h.shape == (0, 64)
    g = op.backward(t["du"], t["dh"], t["x"], t["z"], stats=stats, **weights)
    for k in ("post_weight", "post_bias", "pre_weight"):
        assert torch.equal(getattr(g, k), torch.zeros(64, device="cuda"))


@pytest.mark.parametrize("cols,pad", [(64, 8), (64, 3), (100, 1), (1000, 24), (777, 0)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_row_strides_and_offsets(cols, pad, dtype):
    """Rows inside wider rows, starting anywhere."""
    op = ResidualNorm(cols, post="rms", pre="rms")
    t = _inputs(19, cols, dtype, gate="rows")
    for k in ("x", "z", "gate", "du", "dh"):
        wide = torch.zeros(19, cols + pad + 1, dtype=t[k].dtype, device="cuda")
        wide[:, 1:1 + cols] = t[k]
        t[k] = wide[:, 1:1 + cols]
    u, h, _ = run(op, t)
    wide = torch.full((2, 19, cols + pad + 1), 5.0, dtype=u.dtype, device="cuda")
    out = (wide[0][:, 1:1 + cols], wide[1][:, 1:1 + cols])
    op.forward(t["x"], t["z"], out=out, **{k: t[k] for k in NAMES})
    assert torch.equal(out[0], u) and torch.equal(out[1], h)
    wide[:, :, 1:1 + cols] = 5.0
    assert bool((wide == 5.0).all())


@pytest.mark.parametrize("cols", [64, 100, 777, 4100])
@pytest.mark.parametrize("post,pre", [("rms", "rms"), (None, None), (None, "layer")])
def test_in_place_forward(cols, post, pre):
    op = ResidualNorm(cols, post=post, pre=pre)
    t = _inputs(41, cols, "bf16", post=post, pre=pre)
    weights = {k: t[k] for k in NAMES}
    u, h, _ = op.forward(t["x"], t["z"], **weights)
    x, z = t["x"].clone(), t["z"].clone()
    op.forward(x, z, out=(x, z), need_stats=False, **weights)
    assert torch.equal(x, u) and torch.equal(z, h)


def test_outputs_may_be_left_out():
    op = ResidualNorm(96, post="rms", pre="rms")
    t = _inputs(7, 96, "bf16")
    weights = {k: t[k] for k in NAMES}
    u, h, _ = op.forward(t["x"], t["z"], **weights)
    only = torch.zeros_like(h)
    assert op.forward(t["x"], t["z"], out=(None, only), **weights)[0] is None
    assert torch.equal(only, h)
    op.forward(t["x"], t["z"], out=(only, None), **weights)
    assert torch.equal(only, u)


def test_large_means_and_outliers():
    """A mean 1e4 deviations away, and one element 1e4 times the others."""
    op = ResidualNorm(1024, post=None, pre="layer")
    t = _inputs(8, 1024, "f32", post=None, pre="layer", z=False)
    t["x"] = torch.randn(8, 1024, device="cuda") + 1e4
    run(op, t)
    t["x"] = torch.randn(8, 1024, device="cuda")
    t["x"][:, 0] = 1e4
    run(op, t)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_special_values_stay_in_their_row(bad):
    op = ResidualNorm(300, post="layer", pre="rms")
    t = _inputs(9, 300, "bf16", post="layer", pre="rms", gate="rows")
    weights = {k: t[k] for k in NAMES}
    u0, h0, stats0 = op.forward(t["x"], t["z"], **weights)
    g0 = op.backward(t["du"], t["dh"], t["x"], t["z"], stats=stats0, **weights)
    t["z"][4, 11] = bad
    u, h, stats = op.forward(t["x"], t["z"], **weights)
    g = op.backward(t["du"], t["dh"], t["x"], t["z"], stats=stats, **weights)
    others = torch.arange(9, device="cuda") != 4
    for a, b in ((u, u0), (h, h0), (g.x, g0.x), (g.z, g0.z), (g.gate, g0.gate)):
        assert torch.equal(a[others], b[others])
        assert not bool(a[4].isfinite().all())
    assert not bool(g.pre_weight.isfinite().any())


def test_zero_rows_of_values():
    op = ResidualNorm(256, post="layer", pre="rms")
    t = _inputs(4, 256, "f32", post="layer", pre="rms")
    t["x"].zero_()
    t["z"].zero_()
    t["post_bias"].zero_()
    run(op, t)


def test_gradients_against_differences():
    """Directional derivatives of sum(u du + h dh) by central differences of the float32 kernels: the second order
    is gone, the third times step^2 = 1e-4 and rounding of 1e-7 / step remain."""
    op = ResidualNorm(40, post="layer", pre="rms", residual_scale=0.8, branch_scale=1.3)
    t = _inputs(12, 40, "f32", post="layer", pre="rms", gate="shared", gate_rows=4, bias=True)
    names = ("x", "z") + NAMES

    def loss(v):
        u, h, _ = op.forward(v["x"], v["z"], **{k: v[k] for k in NAMES})
        return float((u.double() * t["du"]).sum() + (h.double() * t["dh"]).sum())

    _, _, stats = op.forward(t["x"], t["z"], **{k: t[k] for k in NAMES})
    g = op.backward(t["du"], t["dh"], t["x"], t["z"], stats=stats, **{k: t[k] for k in NAMES})
    step = 1e-2
    for k in names:
        gen = torch.Generator(device="cuda")
        gen.manual_seed(5)
        direction = torch.randn(t[k].shape, generator=gen, device="cuda")
        diff = (loss(dict(t, **{k: t[k] + step * direction})) - loss(dict(t, **{k: t[k] - step * direction}))) / (2 * step)
        got = float((getattr(g, k).double() * direction).sum())
        size = float((getattr(g, k).double() * direction).abs().sum())
        assert abs(diff - got) <= 2e-3 * size, k


def test_autograd():
    op = ResidualNorm(48, post="rms", pre="layer")
    t = _inputs(10, 48, "f32", post="rms", pre="layer", gate="shared", gate_rows=5)
    leaves = {k: None if v is None else v.requires_grad_() for k, v in t.items() if k not in ("du", "dh")}
    u, h = op(leaves["x"].view(2, 5, 48), leaves["z"].view(2, 5, 48), *[leaves[k] for k in NAMES])
    assert u.shape == h.shape == (2, 5, 48)
    have = [k for k in leaves if leaves[k] is not None]
    grads = torch.autograd.grad((u.view(10, 48), h.view(10, 48)), [leaves[k] for k in have], (t["du"], t["dh"]))
    ref, tol = reference(op, {k: None if v is None else v.detach() for k, v in t.items()}, 5)
    for k, g in zip(have, grads):
        check("d" + k, g, ref[k], tol[k])
    only, = torch.autograd.grad(op(leaves["x"], leaves["z"], *[leaves[k] for k in NAMES])[1].sum(), [leaves["x"]])
    assert bool(only.isfinite().all())


def test_repeats_are_bitwise_equal_and_streams_are_honoured():
    op = ResidualNorm(768, post="rms", pre="rms")
    t = _inputs(3000, 768, "bf16", gate="rows")
    weights = {k: t[k] for k in NAMES}
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    runs = []
    for _ in range(2):
        u, h, stats = op.forward(t["x"], t["z"], stream=s, **weights)
        runs.append((u, h, stats, *op.backward(t["du"], t["dh"], t["x"], t["z"], stats=stats, stream=s, **weights)))
    s.synchronize()
    for a, b in zip(*runs):
        assert a is b or torch.equal(a, b)


def test_offsets_beyond_32_bits():
    op = ResidualNorm(64, post=None, pre="rms")
    t = _inputs(3, 64, "bf16", post=None, pre="rms")
    big = torch.empty((1 << 31) + 4096, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(big, (3, 64), (1 << 30, 1))
    x.copy_(t["x"])
    t["x"] = x
    run(op, t)


def test_refusals():
    op = ResidualNorm(64, post="rms", pre="rms")
    t = _inputs(8, 64, "bf16")
    x, z, w = t["x"], t["z"], t["pre_weight"]
    for kw in (dict(x=x.cpu(), z=z), dict(x=x[:4], z=z), dict(x=x, z=z[:, :32]), dict(x=x.half(), z=z),
               dict(x=x, z=z.double()), dict(x=x, z=None), dict(x=x, z=z, gate=x[:3]), dict(x=x, z=z, gate=x.half()),
               dict(x=x, z=z, pre_weight=w[:32]), dict(x=x, z=z, pre_weight=w.half()), dict(x=x.t().contiguous().t(), z=z),
               dict(x=x, z=z, pre_weight=w, post_weight=w.bfloat16()), dict(x=x[:1].expand(8, 64), z=z)):
        with pytest.raises(ValueError):
            op.forward(**kw)
    _, _, stats = op.forward(x, z)
    for kw in (dict(stats=None), dict(stats=stats[:4]), dict(stats=stats.double())):
        with pytest.raises(ValueError):
            op.backward(x, z, x, z, **kw)
    with pytest.raises(ValueError):
        op.backward(x.half(), z, x, z, stats=stats)
    for args in ((0,), (32769,)):
        with pytest.raises(ValueError):
            ResidualNorm(*args)
    with pytest.raises(ValueError):
        ResidualNorm(64, pre="batch")
    with pytest.raises(ValueError):
        ResidualNorm(64, pre_eps=-1.0)
