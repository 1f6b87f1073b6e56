"""Gradient norms and clipping on the GPU against float64.

Tolerances.  A norm is the root of a sum of squares, every term positive: a chain of L float32 additions leaves a
relative error of at most (L + 2) 2^-24 in the sum, half of it in the root, and the result is rounded once more.
A thread adds at most numel / 1024 + 8 terms to one of its sums.  A clipped element is c g with c off by the norm's error
and one rounding, the product's rounding and the output type's."""
import math

import pytest
import torch

from paper_2609_30342_gb300 import build as pkg_build
from paper_2609_30342_gb300 import rikfad
from paper_2609_30342_gb300.gradients import GradientClipper

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_ULP = {k: torch.finfo(v).eps / 2 for k, v in DT.items()}
TINY = {"f32": 2.0 ** -149, "bf16": 2.0 ** -134, "f16": 2.0 ** -25}     # half a step (or a step) of the subnormals


@pytest.fixture(scope="module", autouse=True)
def built():
    pkg_build.build()
    yield


def _grads(numels, dtype, std=1e-2, seed=0, offset=0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    out = []
    for n in numels:
        flat = torch.randn(n + offset, generator=gen, device="cuda").mul_(std).to(DT[dtype])
        out.append(flat[offset:])
    return out


def _exact(grads):
    sq = [float((g.double() ** 2).sum()) for g in grads]
    return math.sqrt(math.fsum(sq)), [math.sqrt(v) for v in sq]


def _norm_tol(numels):
    return ((max(numels) / 1024 + 10) / 2 + 2) * EPS


def _check_norms(total, norms, grads):
    want, each = _exact(grads)
    tol = _norm_tol([g.numel() for g in grads] + [1])
    assert abs(float(total) - want) <= tol * want
    for got, w in zip(norms.tolist(), each):
        assert abs(got - w) <= tol * w


def _check_out(out, grads, max_norm, dtype):
    want, _ = _exact(grads)
    c = max_norm / want if want > max_norm else 1.0
    tol = _norm_tol([g.numel() for g in grads] + [1]) + 3 * EPS + HALF_ULP[dtype]
    for o, g in zip(out, grads):
        ref = g.double() * c
        assert bool(((o.double() - ref).abs() <= tol * ref.abs() + TINY[dtype]).all())


LISTS = [[1], [0, 1, 0], [7, 64, 65, 8191], [256 * 512, 512], [1 << 20, 3, 1 << 17, 100_003], [5] * 40, [130] * 300,
         [1_000_003]]


@pytest.mark.parametrize("numels", LISTS, ids=lambda v: "x".join(map(str, v[:4])))
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_norms_and_clipping(numels, dtype):
    grads = _grads(numels, dtype)
    keep = [g.clone() for g in grads]
    clipper = GradientClipper(numels, dtype)
    _check_norms(*clipper.norm(grads), grads)
    want, _ = _exact(grads)
    for max_norm in (0.3 * want, 2.0 * want):
        out = [torch.full_like(g, 7.0) for g in grads]
        total, norms = clipper.clip(max_norm, grads, out=out)
        _check_norms(total, norms, grads)
        _check_out(out, grads, max_norm, dtype)
        if max_norm > want:
            assert all(torch.equal(o, g) for o, g in zip(out, grads))
    assert all(torch.equal(g, k) for g, k in zip(grads, keep))
    total, _ = clipper.clip(0.3 * want, grads)           # in place
    _check_out(grads, keep, 0.3 * want, dtype)
    clipper.close()


@pytest.mark.parametrize("dtype,out", [("f32", "bf16"), ("f32", "f16"), ("bf16", "f32"), ("f16", "bf16")])
@pytest.mark.parametrize("offset", [0, 1])
def test_other_output_type_and_alignment(dtype, out, offset):
    numels = [40_003, 8, 1, 77_777]
    grads = _grads(numels, dtype, offset=offset, seed=3)
    clipper = GradientClipper(numels, dtype, out)
    outs = [torch.zeros(n + 3, dtype=DT[out], device="cuda")[3 * offset:3 * offset + n] for n in numels]
    ptrs = clipper.pack(grads, outs)
    total, norms = clipper.clip(0.5, ptrs=ptrs)
    _check_norms(total, norms, grads)
    _check_out(outs, grads, 0.5, out)


def test_mixed_types_and_many_tensors():
    numels = [(i * 37) % 301 for i in range(2500)]           # more tensors than one launch takes
    types = [("f32", "bf16", "f16")[i % 3] for i in range(2500)]
    grads = [g for n, t, i in zip(numels, types, range(2500)) for g in _grads([n], t, seed=i)]
    clipper = GradientClipper(numels, types)
    out = [torch.zeros_like(g) for g in grads]
    total, norms = clipper.clip(0.1, grads, out=out)
    _check_norms(total, norms, grads)
    want, _ = _exact(grads)
    for o, g, t in zip(out, grads, types):
        _check_out_one(o, g, 0.1 / want, t)


def _check_out_one(o, g, c, dtype):
    ref = g.double() * c
    tol = _norm_tol([1024]) + 3 * EPS + HALF_ULP[dtype]
    assert bool(((o.double() - ref).abs() <= tol * ref.abs() + TINY[dtype]).all())


@pytest.mark.parametrize("std", [1e-30, 1e-22, 1e-12, 1e15, 1e25, 1e33])
def test_squares_outside_the_range_of_float32(std):
    grads = _grads([20_000, 500], "f32", std=std)
    clipper = GradientClipper([20_000, 500], "f32")
    want, _ = _exact(grads)
    out = [torch.empty_like(g) for g in grads]
    total, norms = clipper.clip(0.25 * want, grads, out=out)
    _check_norms(total, norms, grads)
    _check_out(out, grads, 0.25 * want, "f32")


def test_zero_gradients_and_zero_max_norm():
    clipper = GradientClipper([1000, 10], "f32")
    grads = [torch.zeros(1000, device="cuda"), torch.zeros(10, device="cuda")]
    total, norms = clipper.clip(1.0, grads)
    assert float(total) == 0.0 and norms.tolist() == [0.0, 0.0]
    assert not any(g.any() for g in grads)
    grads = _grads([1000, 10], "f32")
    total, _ = clipper.clip(0.0, grads)
    assert float(total) > 0 and not any(g.any() for g in grads)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_a_norm_that_is_not_finite_scales_nothing(bad, dtype):
    grads = _grads([3000, 50, 9000], dtype)
    grads[1][17] = bad
    keep = [g.clone() for g in grads]
    clipper = GradientClipper([3000, 50, 9000], dtype)
    total, norms = clipper.clip(1e-3, grads)
    norms = norms.tolist()
    assert not math.isfinite(float(total)) and not math.isfinite(norms[1])
    assert math.isfinite(norms[0]) and math.isfinite(norms[2])
    assert all(torch.equal(g.nan_to_num(123.0), k.nan_to_num(123.0)) for g, k in zip(grads, keep))


def test_no_tensors():
    clipper = GradientClipper([], "f32")
    total, norms = clipper.clip(1.0, [])
    assert float(total) == 0.0 and norms.numel() == 0


def test_repeats_are_bitwise_equal_and_streams_are_honoured():
    numels = [300_000, 17, 50_000]
    grads = _grads(numels, "bf16")
    clipper = GradientClipper(numels, "bf16")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    outs, totals = [], []
    for _ in range(3):
        out = [torch.empty_like(g) for g in grads]
        totals.append(clipper.clip(0.5, grads, out=out, stream=s)[0])
        outs.append(out)
    s.synchronize()
    for out, total in zip(outs[1:], totals[1:]):
        assert torch.equal(total, totals[0]) and all(torch.equal(a, b) for a, b in zip(out, outs[0]))
    _check_out(outs[0], grads, 0.5, "bf16")


def test_capture_in_a_graph():
    numels = [70_000, 9]
    grads = _grads(numels, "f32")
    clipper = GradientClipper(numels, "f32")
    out = [torch.empty_like(g) for g in grads]
    ptrs = clipper.pack(grads, out)
    clipper.clip(0.5, ptrs=ptrs)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        total, norms = clipper.clip(0.5, ptrs=ptrs)
    for seed in (5, 6):
        for g, new in zip(grads, _grads(numels, "f32", seed=seed)):
            g.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        _check_norms(total, norms, grads)
        _check_out(out, grads, 0.5, "f32")


def test_page_locked_gradients():
    g = torch.randn(5000).mul_(0.01).pin_memory()
    clipper = GradientClipper([5000], "f32")
    out = [torch.empty(5000, device="cuda")]
    total, norms = clipper.clip(0.1, [g], out=out)
    _check_norms(total, norms, [g.cuda()])
    _check_out(out, [g.cuda()], 0.1, "f32")


def test_more_than_2_to_the_31_elements():
    n = (1 << 31) + 9
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g[0], g[n // 2], g[n - 1] = 3.0, 4.0, 12.0
    clipper = GradientClipper([n], "bf16")
    total, _ = clipper.clip(6.5, [g])
    assert float(total) == 13.0
    assert [float(g[i]) for i in (0, n // 2, n - 1)] == [1.5, 2.0, 6.0]


def test_refusals():
    clipper = GradientClipper([100, 10], ["f32", "bf16"], ["bf16", "bf16"])
    grads = [torch.zeros(100, device="cuda"), torch.zeros(10, dtype=torch.bfloat16, device="cuda")]
    for wrong in ([grads[0]], [grads[0], grads[1].float()], [grads[0][:50], grads[1]],
                  [torch.zeros(200, device="cuda")[::2], grads[1]], [torch.zeros(100), grads[1]]):
        with pytest.raises(ValueError):
            clipper.norm(wrong)
    with pytest.raises(ValueError):
        clipper.clip(1.0, grads)                        # in place, but the first tensor changes type
    out = [torch.zeros(100, dtype=torch.bfloat16, device="cuda"), torch.zeros_like(grads[1])]
    for max_norm in (-1.0, float("nan")):
        with pytest.raises(rikfad.RikfadError) as e:
            clipper.clip(max_norm, grads, out=out)
        assert e.value.code == rikfad.ERR_ARG
    with pytest.raises(ValueError):
        clipper.clip(1.0, ptrs=clipper.pack(grads))
    clipper.close()
    with pytest.raises(RuntimeError):
        clipper.norm(grads)


def test_allocations_are_released_and_failures_reported():
    before = rikfad.debug_live_allocations()
    rikfad.debug_fail_allocation(1)
    try:
        with pytest.raises(rikfad.RikfadError) as e:
            GradientClipper([1000, 20], "f32")
        assert e.value.code == rikfad.ERR_OOM
    finally:
        rikfad.debug_fail_allocation(0)
    assert rikfad.debug_live_allocations() == before
    clipper = GradientClipper([1000, 20], "f32")
    assert clipper.workspace_bytes() > 0 and rikfad.debug_live_allocations() > before
    clipper.close()
    assert rikfad.debug_live_allocations() == before


def test_optimizer_clips_every_group():
    from paper_2609_30342_gb300.optim import RIKFADOptimizer
    torch.manual_seed(1)
    a, b = torch.nn.Linear(40, 30).cuda(), torch.nn.LayerNorm(30).cuda()
    opt = RIKFADOptimizer([{"params": list(a.parameters())}, {"params": list(b.parameters())}], lr=0.05, alpha=0.2,
                          mu=1e-3)
    (b(a(torch.randn(16, 40, device="cuda"))) ** 3).sum().backward()
    b.bias.grad = None
    grads = [p.grad for p in [*a.parameters(), b.weight]]
    keep = [g.clone() for g in grads]
    want, _ = _exact(keep)
    total = opt.clip_grad_norm(0.1 * want)
    assert abs(float(total) - want) <= _norm_tol([1200]) * want
    _check_out(grads, keep, 0.1 * want, "f32")
    opt.step()
    torch.cuda.synchronize()
    assert all(bool(p.isfinite().all()) for p in a.parameters())
    opt.close()
