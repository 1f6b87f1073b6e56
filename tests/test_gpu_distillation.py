"""The loss against a teacher's top logits and labels on the GPU against float64.

Tolerance (U = 2^-24).  A power of two of an argument is off by 4 U (the approximate instruction's bound) and by the
argument's own error, at most 2 U of its size: its scale log2(e) / T is rounded once, the fused product once; the
reference's rounding is the same everywhere.  A sum of n such terms adds n U at most, and as much again for the factors
by which parts of it move to a larger maximum; here threads add V / 256 terms or fewer, then trees: n = V / 128 + 64.
Logarithms are good to 2 U of their value and U.  Shares are off by the errors of their power and their sum, losses by
those of their logarithms, weighted by the shares.  Then the type's rounding."""
import pytest
import torch

from paper_2609_30342_gb300 import build as pkg_build
from paper_2609_30342_gb300.losses import DistillationLoss

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_ULP = {v: torch.finfo(v).eps / 2 for v in DT.values()}
# what is too small for a type's range: float32 powers below 2^-126 are zero
TINY = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -25}
U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def built():
    pkg_build.build()
    yield


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _rand(*shape, seed=0, dtype=torch.float32, scale=1.0):
    return (torch.randn(shape, device="cuda", generator=_gen(seed)) * scale).to(dtype)


def _inputs(rows, vocab, k, dtype="f32", teacher="f32", index_dtype=torch.int64, label_dtype=torch.int64, absent=0.0, seed=0,
            scale=3.0):
    """logits, teacher, index, labels: entries of every kind, some of them twice."""
    logits = _rand(rows, vocab, seed=seed, dtype=DT[dtype], scale=scale)
    t = index = None
    if k:
        t = _rand(rows, k, seed=seed + 1, dtype=DT[teacher], scale=scale)
        index = torch.randint(0, vocab, (rows, k), device="cuda", generator=_gen(seed + 2))
        if absent:
            u = torch.rand(rows, k, device="cuda", generator=_gen(seed + 3))
            index = torch.where(u < absent, torch.where(u < absent / 2, -1, vocab), index)
            index[0] = -5
        index = index.to(index_dtype)
    labels = torch.randint(0, vocab, (rows,), device="cuda", generator=_gen(seed + 4))
    if absent:
        labels[::3] = -100
    return logits, t, index, labels.to(label_dtype)


def _soft(x, scale):
    """(log2 shares, sizes of their errors in units of U) of softmax(x scale) with x of [rows, n]; -inf is absent."""
    n = x.shape[1]
    arg = (x - x.max(1, keepdim=True).values) * (scale / 0.6931471805599453)
    share = torch.exp2(arg)
    total = share.sum(1, keepdim=True)
    finite = torch.where(share > 0, arg, torch.zeros_like(arg)).abs()
    mean = (share * finite).sum(1, keepdim=True) / total
    log_total = torch.log2(total)
    off = 2 * finite + 2 * mean + 2 * log_total.abs() + n / 128 + 64 + 16
    return arg - log_total, off


def _check(op, logits, teacher, index, labels, loss=None, dlogits=None, scale=None):
    rows, vocab = logits.shape
    x, T = logits.double(), op.temperature
    want, bound = torch.zeros(rows, dtype=torch.float64, device="cuda"), torch.zeros(rows, dtype=torch.float64, device="cuda")
    grad, error = torch.zeros_like(x), torch.zeros_like(x)
    if teacher is not None and op.teacher_weight and teacher.shape[1]:
        a, i = op.teacher_weight, index.long()
        there = (i >= 0) & (i < vocab) & (teacher != -float("inf"))
        some = there.any(1, keepdim=True)
        i = torch.where(there, i, torch.zeros_like(i))
        t = torch.where(there, teacher.double(), torch.full_like(teacher.double(), -float("inf")))
        lp, lp_off = _soft(torch.where(some, t, torch.zeros_like(t)), 1 / T)
        lq, lq_off = _soft(x, 1 / T)
        p = torch.where(there, torch.exp2(lp), torch.zeros_like(lp))
        gap = torch.where(p > 0, lp - lq.gather(1, i), torch.zeros_like(lp))
        f = a * T * T * 0.6931471805599453
        want += f * (p * gap).sum(1)
        off = lp_off + lq_off.gather(1, i) + (lp_off + teacher.shape[1] + 8) * gap.abs()
        bound += abs(f) * U * torch.where(p > 0, p * off, torch.zeros_like(p)).sum(1)
        grad += torch.where(some, a * T * torch.exp2(lq), torch.zeros_like(lq))
        error += torch.where(some, abs(a * T) * torch.exp2(lq) * (lq_off + 8) * U, torch.zeros_like(lq))
        grad.scatter_add_(1, i, -a * T * p)
        error.scatter_add_(1, i, abs(a * T) * p * (lp_off + teacher.shape[1] + 8) * U)
    if labels is not None and op.label_weight:
        b, i = op.label_weight, labels.long()[:, None]
        there = (i >= 0) & (i < vocab)
        i = torch.where(there, i, torch.zeros_like(i))
        lq, lq_off = _soft(x, 1.0)
        at = torch.where(there, lq.gather(1, i), torch.zeros_like(there, dtype=torch.float64))[:, 0]
        want -= b * 0.6931471805599453 * at
        bound += abs(b) * U * (lq_off.gather(1, i)[:, 0] + 8 * at.abs()) * there[:, 0]
        grad += torch.where(there, b * torch.exp2(lq), torch.zeros_like(lq))
        error += torch.where(there, abs(b) * torch.exp2(lq) * (lq_off + 8) * U, torch.zeros_like(lq))
        grad.scatter_add_(1, i, -b * there.double())
        error.scatter_add_(1, i, abs(b) * there.double() * 4 * U)
    if loss is not None:
        assert loss.dtype == torch.float32 and loss.shape == (rows,)
        limit = bound + 4 * U * want.abs() + 2.0 ** -126
        assert ((loss.double() - want).abs() <= limit).all(), float(((loss.double() - want).abs() / limit).max())
    if dlogits is not None:
        s = torch.ones(rows, 1, dtype=torch.float64, device="cuda") if scale is None else scale
        g, e = grad * s, (error + 4 * U * grad.abs()) * s.abs()
        limit = e + HALF_ULP[dlogits.dtype] * (g.abs() + e) + TINY[dlogits.dtype]
        assert dlogits.dtype == logits.dtype
        assert ((dlogits.double() - g).abs() <= limit).all(), float(((dlogits.double() - g).abs() / limit).max())


def _all_ways(op, logits, teacher, index, labels):
    """Forward, the two directions apart and in one pass, with a factor for every row."""
    rows = logits.shape[0]
    dloss = _rand(rows, seed=99)
    loss, stats = op.forward(logits, teacher, index, labels)
    apart = op.backward(dloss, logits, teacher, index, labels, stats, grad_scale=0.5)
    both, fused = op.loss_and_gradient(logits, teacher, index, labels, grad_scale=0.5, dloss=dloss)
    scale = 0.5 * dloss.double()[:, None]
    _check(op, logits, teacher, index, labels, loss, apart, scale)
    _check(op, logits, teacher, index, labels, both, fused, scale)
    return loss, apart, both, fused


@pytest.mark.parametrize("weights", [(1.0, 0.0), (0.9, 0.5), (0.0, 1.0)])
@pytest.mark.parametrize("rows,vocab,k", [(1, 1, 1), (3, 2, 2), (5, 15, 3), (4, 100, 100), (33, 257, 5), (8, 50257, 16),
                                          (3, 32003, 300), (2, 131072, 128), (2, 262144, 64), (700, 1000, 33), (2, 2000, 1024)])
def test_sizes(rows, vocab, k, weights):
    op = DistillationLoss(2.0, *weights)
    _all_ways(op, *_inputs(rows, vocab, k))


@pytest.mark.parametrize("vocab", [64, 1003, 40003])
@pytest.mark.parametrize("index_dtype,label_dtype", [(torch.int32, torch.int64), (torch.int64, torch.int32)])
@pytest.mark.parametrize("teacher", list(DT))
@pytest.mark.parametrize("dtype", list(DT))
def test_types(dtype, teacher, index_dtype, label_dtype, vocab):
    op = DistillationLoss(1.5, 0.7, 0.3)
    _all_ways(op, *_inputs(9, vocab, 20, dtype, teacher, index_dtype, label_dtype, absent=0.4))


@pytest.mark.parametrize("rows", [1, 150, 400, 2000])
@pytest.mark.parametrize("temperature", [0.001, 0.7, 1.0, 3.21, 1000.0])
def test_temperatures(temperature, rows):
    op = DistillationLoss(temperature, 1.0, 0.5)
    _all_ways(op, *_inputs(rows, 3001, 12, "bf16", absent=0.2))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_largest_vocabulary(dtype):
    op = DistillationLoss(2.0, 1.0, 0.5)
    logits, t, index, labels = _inputs(2, 1 << 24, 64, dtype)
    index[:, 0], labels[1] = (1 << 24) - 1, (1 << 24) - 1
    loss, g = op.loss_and_gradient(logits, t, index, labels)
    _check(op, logits, t, index, labels, loss, g)
    apart, stats = op.forward(logits, t, index, labels)
    _check(op, logits, t, index, labels, apart, op.backward(None, logits, t, index, labels, stats))


def test_terms_apart():
    logits, t, index, labels = _inputs(50, 777, 10, absent=0.3)
    for op, args in ((DistillationLoss(2.0), (logits, t, index, None)), (DistillationLoss(2.0, 0.0, 1.0), (logits, None, None, labels)),
                     (DistillationLoss(2.0, 1.0, 0.0), (logits, t, index, labels)),
                     (DistillationLoss(2.0, 1.0, 1.0), (logits, t[:, :0], index[:, :0], labels))):
        _all_ways(op, *args)


def test_cross_entropy():
    logits, _, _, labels = _inputs(64, 5003, 0, absent=0.2)
    op = DistillationLoss(label_weight=1.0)
    loss, _ = op.forward(logits, labels=labels)
    want = torch.nn.functional.cross_entropy(logits.double(), labels, reduction="none", ignore_index=-100)
    assert torch.allclose(loss.double(), want, rtol=1e-5, atol=1e-5)
    assert (loss[labels < 0] == 0).all()


def test_rows_without_a_term():
    """Losses and gradients of exactly 0, whatever the logits hold."""
    logits, t, index, labels = _inputs(12, 999, 7, "bf16")
    index[2:6], labels[2:6] = -1, -100
    t[6:9], labels[6:9] = -float("inf"), 999
    logits[2], logits[3, 5], logits[4], logits[7, 1] = float("nan"), float("inf"), -float("inf"), float("nan")
    op = DistillationLoss(2.0, 1.0, 0.5)
    loss, stats = op.forward(logits, t, index, labels)
    grads = [op.backward(None, logits, t, index, labels, stats), op.loss_and_gradient(logits, t, index, labels)[1]]
    assert (loss[2:9] == 0).all()
    for g in grads:
        assert (g[2:9] == 0).all()
    keep = torch.tensor([0, 1, 9, 10, 11], device="cuda")
    for g in grads:
        _check(op, logits[keep], t[keep], index[keep], labels[keep], loss[keep], g[keep])


def test_masked_logits():
    """Logits of -inf, and of the type's lowest value, have no share; a teacher's -inf entries are absent."""
    for low in (-float("inf"), torch.finfo(torch.float32).min):
        logits, t, index, labels = _inputs(6, 2048, 9)
        logits[:, 100:1900] = low
        index, labels = index % 100, labels % 100
        t[1, :8], t[2, 0] = -float("inf"), -float("inf")
        _all_ways(DistillationLoss(2.0, 1.0, 0.5), logits, t, index, labels)
        # a masked element that is asked for: an infinite loss (a huge one), the gradient stays finite
        loss, g = DistillationLoss(2.0, 1.0, 0.5).loss_and_gradient(logits, t, index, torch.full_like(labels, 500))
        assert (loss > 1e37).all() and g.isfinite().all() and (g[:, 500] == -0.5).all()


@pytest.mark.parametrize("temperature", [0.5, 1.0, 2.0])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_rows_of_the_lowest_value(dtype, temperature):
    """A row masked all over with the type's lowest value has equal shares; with -inf beside it, the rest has."""
    logits, t, index, labels = _inputs(4, 1000, 5, dtype)
    low = torch.finfo(DT[dtype]).min
    logits[0], logits[1], logits[1, ::2] = low, low, -float("inf")
    index[1], labels[1] = 2 * (index[1] // 2) + 1, 2 * (labels[1] // 2) + 1
    t[2], t[3, 1:] = torch.finfo(torch.float32).min, torch.finfo(torch.float32).min
    op = DistillationLoss(temperature, 1.0, 0.5)
    _, apart, _, fused = _all_ways(op, logits, t, index, labels)
    rest = torch.ones(1000, dtype=torch.bool, device="cuda")
    rest[index[0]] = rest[labels[0]] = False
    assert (fused[0][rest] == fused[0][rest][0]).all() and fused[0][rest][0] != 0 and (fused[1, ::2] == 0).all()


def test_non_finite_rows():
    logits, t, index, labels = _inputs(8, 513, 4)
    logits[0], logits[1, 7], logits[2, 9], logits[3] = -float("inf"), float("nan"), float("inf"), float("inf")
    op = DistillationLoss(2.0, 1.0, 0.5)
    loss, g = op.loss_and_gradient(logits, t, index, labels)
    assert loss[:4].isnan().all() and g[0].isnan().all() and g[1].isnan().all() and g[3].isnan().all() and g[2].isnan().any()
    _check(op, logits[4:], t[4:], index[4:], labels[4:], loss[4:], g[4:])
    t[4, 0], t[5, 1] = float("nan"), float("inf")
    loss, g = op.loss_and_gradient(logits, t, index, labels)
    assert loss[4:6].isnan().all()
    _check(op, logits[6:], t[6:], index[6:], labels[6:], loss[6:], g[6:])


@pytest.mark.parametrize("offset", [0.0, 1000.0, -30000.0])
def test_far_from_zero(offset):
    """Losses do not depend on where the logits are; float32 ones there are multiples of 2^-9 or so, exactly moved."""
    logits, t, index, labels = _inputs(16, 4001, 8)
    logits, t = (torch.round(v * 256) / 256 + offset for v in (logits, t))
    _all_ways(DistillationLoss(2.0, 1.0, 0.5), logits, t, index, labels)


def test_entries_that_name_one_element():
    logits, t, index, labels = _inputs(40, 300, 60)
    index[:, 10:40] = index[:, :1]
    index[5], labels[5] = 7, 7
    labels[6] = index[6, 0]
    op = DistillationLoss(1.3, 1.0, 0.5)
    *_, g = _all_ways(op, logits, t, index, labels)
    for _ in range(3):
        assert torch.equal(_all_ways(op, logits, t, index, labels)[3], g)


@pytest.mark.parametrize("k,gap", [(1024, 128), (64, 2048), (3, 40000), (2, 1)])
def test_evenly_spaced_entries(k, gap):
    logits, t, _, labels = _inputs(3, 131072, k)
    index = (torch.arange(k, device="cuda") * gap + torch.tensor([[0], [5], [131071]], device="cuda")) % 131072
    _all_ways(DistillationLoss(2.0, 1.0, 0.5), logits, t, index, index[:, -1].contiguous())


@pytest.mark.parametrize("vocab,pad", [(1000, 8), (1000, 3), (1001, 7), (1001, 0), (50257, 15)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strided_rows_at_any_offset(dtype, vocab, pad):
    """Logits, gradients and entries in wider tensors; what is between the rows stays."""
    logits, t, index, labels = _inputs(10, vocab, 9, dtype)
    op = DistillationLoss(2.0, 1.0, 0.5)
    want_loss, want = op.loss_and_gradient(logits, t, index, labels)
    for shift in (0, 1, 5):
        def place(v, value):
            big = torch.full((10 * (v.shape[1] + pad) + shift,), value, dtype=v.dtype, device="cuda")
            view = big[shift:].view(10, v.shape[1] + pad)[:, :v.shape[1]]
            view.copy_(v)
            return big, view
        _, x = place(logits, 7)
        _, tt = place(t, 7)
        _, ii = place(index, 7)
        for shift in (0, 1, 5):
            big, out = place(want, 7)
            loss, g = op.loss_and_gradient(x, tt, ii, labels, out=out)
            assert g is out
            _check(op, logits, t, index, labels, loss, out)
            _, stats = op.forward(x, tt, ii, labels)
            op.backward(None, x, tt, ii, labels, stats, out=out)
            _check(op, logits, t, index, labels, None, out)
            out.fill_(7)
            assert (big == 7).all()


@pytest.mark.parametrize("rows,vocab", [(3, 1000), (2, 60001), (500, 20011)])
def test_in_place(rows, vocab):
    logits, t, index, labels = _inputs(rows, vocab, 30, "bf16")
    op = DistillationLoss(2.0, 1.0, 0.5)
    want_loss, want = op.loss_and_gradient(logits, t, index, labels)
    _, stats = op.forward(logits, t, index, labels)
    apart = op.backward(None, logits, t, index, labels, stats)
    x = logits.clone()
    loss, g = op.loss_and_gradient(x, t, index, labels, out=x)
    assert g is x and torch.equal(x, want) and torch.equal(loss, want_loss)
    x = logits.clone()
    assert torch.equal(op.backward(None, x, t, index, labels, stats, out=x), apart)


def test_shapes_and_empty():
    op = DistillationLoss(2.0, 1.0, 0.5)
    logits, t, index, labels = _inputs(6, 50, 4)
    flat, dflat = op.loss_and_gradient(logits, t, index, labels)
    loss, d = op.loss_and_gradient(logits.view(2, 3, 50), t.view(2, 3, 4), index.view(2, 3, 4), labels.view(2, 3))
    assert torch.equal(loss, flat.view(2, 3)) and torch.equal(d, dflat.view(2, 3, 50))
    loss, d = op.loss_and_gradient(logits[0], t[0], index[0], labels[0])
    assert loss.shape == () and torch.equal(loss, flat[0]) and torch.equal(d, dflat[0])
    x = torch.empty(0, 50, device="cuda", requires_grad=True)
    loss = op(x, t[:0], index[:0], labels[:0])
    g, = torch.autograd.grad(loss.sum(), x)
    assert loss.shape == (0,) and g.shape == (0, 50)


def test_autograd_and_differences():
    op = DistillationLoss(1.7, 0.8, 0.4)
    logits, t, index, labels = _inputs(12, 333, 9, absent=0.2)
    x, dloss = logits.clone().requires_grad_(), _rand(12, seed=5)
    loss = op(x, t, index, labels)
    g, = torch.autograd.grad(loss, x, dloss)
    _check(op, logits, t, index, labels, loss.detach(), g, dloss.double()[:, None])
    # Central differences of the operator's own losses along a direction: they are off by 1e-5 / (2 h) at most, and by
    # h^2 / 6 of the third derivative, which is of the order of the step's cube.
    step, h = _rand(12, 333, seed=6), 0.05
    up, _ = op.forward(logits + h * step, t, index, labels)
    down, _ = op.forward(logits - h * step, t, index, labels)
    want = (up.double() - down.double()) / (2 * h) * dloss
    have = (g.double() * step).sum(1)
    assert ((want - have).abs() <= (1e-5 / (2 * h) + 4 * h * h) * (1 + dloss.abs())).all()
    g, = torch.autograd.grad(op(x, t, index, labels).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        (g * g).sum().backward()


def test_far_rows():
    """Logits beyond 2^31 elements."""
    logits = torch.zeros(17000, 131072, dtype=torch.bfloat16, device="cuda")
    logits[-2:] = _rand(2, 131072, dtype=torch.bfloat16)
    labels = torch.full((17000,), -100, device="cuda")
    labels[-2:] = 131071
    op = DistillationLoss(label_weight=1.0)
    loss, g = op.loss_and_gradient(logits, labels=labels, out=logits.clone())
    _check(op, logits[-2:], None, None, labels[-2:], loss[-2:], g[-2:])
    assert int(torch.count_nonzero(g[:-2])) == 0


def test_refusals():
    op = DistillationLoss(2.0, 1.0, 0.5)
    x, t, i, y = _inputs(4, 30, 3)
    stats = torch.empty(4, 4, device="cuda")
    big = torch.zeros(4, 1025, device="cuda")
    for call in (lambda: op.forward(x), lambda: op.forward(x, t), lambda: op.forward(x, None, i), lambda: op.forward(x.cpu(), t, i),
                 lambda: op.forward(x.double(), t, i), lambda: op.forward(x, t.double(), i), lambda: op.forward(x, t, i.float()),
                 lambda: op.forward(x, t.cpu(), i), lambda: op.forward(x, t[:3], i[:3]), lambda: op.forward(x, t, i[:, :2]),
                 lambda: op.forward(x, big, big.long()), lambda: op.forward(x, labels=y[:3]), lambda: op.forward(x, labels=y.float()),
                 lambda: op.forward(x, labels=y.cpu()), lambda: op.forward(x.t().contiguous().t(), t, i),
                 lambda: op.forward(x[:1].expand(4, 30), t, i), lambda: op.forward(x[:, :0], t, i),
                 lambda: op.loss_and_gradient(x, t, i, out=x[:3]), lambda: op.loss_and_gradient(x, t, i, out=x.bfloat16()),
                 lambda: op.loss_and_gradient(x, t, i, out=torch.empty(4, 30)),
                 lambda: op.loss_and_gradient(x, t, i, dloss=y.float()[:3]), lambda: op.loss_and_gradient(x, t, i, dloss=y),
                 lambda: op.backward(None, x, t, i), lambda: op.backward(None, x, t, i, stats=stats[:3]),
                 lambda: op.forward(x, labels=torch.zeros(8, dtype=torch.int64, device="cuda")[::2])):
        with pytest.raises(ValueError):
            call()
    for args in ((0.0,), (float("nan"),), (1e4,), (1.0, float("inf")), (1.0, 1.0, float("nan"))):
        with pytest.raises(ValueError):
            DistillationLoss(*args)
