"""The token embedding on the GPU against float64.

Tolerance.  A row is one float32 product with the scale, itself rounded to float32 (2^-24 each), rounded to its type.  A
gradient of n tokens is a float32 sum in some fixed order, off by at most (n - 1) 2^-24 of the sum of magnitudes, times
the scale (2^-24 twice), plus the addition to what was there (2^-24), rounded to its type."""
import pytest
import torch

from paper_2609_30342_gb300 import build as pkg_build
from paper_2609_30342_gb300.embedding import TokenEmbedding

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_ULP = {v: torch.finfo(v).eps / 2 for v in DT.values()}
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -25}
U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def built():
    pkg_build.build()
    yield


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _rand(*shape, seed=0, dtype=torch.float32):
    return torch.randn(shape, device="cuda", generator=_gen(seed)).to(dtype)


def _ids(tokens, vocab, kind, seed=0, dtype=torch.int64):
    u = torch.rand(tokens, device="cuda", generator=_gen(seed), dtype=torch.float64)
    if kind == "uniform":
        ids = (u * vocab).long()
    elif kind == "skewed":                  # some ids very often, most of the table never
        ids = (vocab * u ** 8).long()
    elif kind == "one":
        ids = torch.full((tokens,), vocab // 2, device="cuda")
    elif kind == "ends":                    # the first and the last row, and ids outside on both sides
        ids = torch.tensor([0, vocab - 1, -1, vocab, -(1 << 31), (1 << 31) - 1], device="cuda")[(u * 6).long()]
    else:
        ids = torch.full((tokens,), -100, device="cuda")
    return ids.to(dtype)


def _check_forward(got, weight, ids, scale):
    ids = ids.long()
    inside = (ids >= 0) & (ids < weight.shape[0])
    want = weight[torch.where(inside, ids, torch.zeros_like(ids))].double() * scale
    want = torch.where(inside[..., None], want, torch.zeros_like(want))
    bound = want.abs() * (2 * U + HALF_ULP[got.dtype] * (1 + 2 * U)) + TINY[got.dtype]
    assert ((got.double() - want).abs() <= bound).all()
    assert (got[~inside] == 0).all()


def _check_backward(got, dout, ids, scale, before=None):
    vocab, width = got.shape
    ids, d = ids.reshape(-1).long(), dout.reshape(-1, width).double()
    at = torch.nonzero((ids >= 0) & (ids < vocab))[:, 0]
    total = torch.zeros(vocab, width, dtype=torch.float64, device="cuda").index_add_(0, ids[at], d[at])
    size = torch.zeros(vocab, width, dtype=torch.float64, device="cuda").index_add_(0, ids[at], d[at].abs())
    n = torch.bincount(ids[at], minlength=vocab)[:, None].double()
    want, bound = total * scale, size * abs(scale) * (n + 2) * U
    if before is not None:
        want = want + before.double()
        bound = bound + U * (want.abs() + bound)
    bound = bound + HALF_ULP[got.dtype] * (want.abs() + bound) + TINY[got.dtype]
    assert ((got.double() - want).abs() <= bound).all()
    empty = n[:, 0] == 0
    assert torch.equal(got[empty], torch.zeros_like(got[empty]) if before is None else before[empty])


@pytest.mark.parametrize("kind", ["uniform", "skewed", "one", "ends", "none"])
@pytest.mark.parametrize("tokens,vocab,width", [(1, 1, 1), (8, 50257, 768), (33, 7, 64), (513, 300, 1001), (4096, 17, 96),
                                                (5000, 2048, 130), (40000, 70000, 36)])
def test_sizes(tokens, vocab, width, kind):
    op = TokenEmbedding(vocab, width, scale=1.7)
    w, d = _rand(vocab, width, seed=1), _rand(tokens, width, seed=2)
    ids = _ids(tokens, vocab, kind)
    _check_forward(op.forward(w, ids), w, ids, op.scale)
    _check_backward(op.backward(d, ids), d, ids, op.scale)


@pytest.mark.parametrize("id_dtype", [torch.int32, torch.int64])
@pytest.mark.parametrize("rows", list(DT))
@pytest.mark.parametrize("weight", list(DT))
@pytest.mark.parametrize("width", [64, 52, 46, 7])
def test_types(width, weight, rows, id_dtype):
    op = TokenEmbedding(301, width, scale=0.25)
    w, d = _rand(301, width, seed=1, dtype=DT[weight]), _rand(2, 350, width, seed=2, dtype=DT[rows])
    ids = _ids(700, 301, "skewed", dtype=id_dtype).view(2, 350)
    out = op.forward(w, ids, dtype=DT[rows])
    assert out.shape == (2, 350, width) and out.dtype == DT[rows]
    _check_forward(out, w, ids, op.scale)
    got = op.backward(d, ids, dtype=DT[weight])
    assert got.dtype == DT[weight]
    _check_backward(got, d, ids, op.scale)
    before = _rand(301, width, seed=3, dtype=DT[weight])
    got = op.backward(d, ids, out=before.clone(), accumulate=True)
    _check_backward(got, d, ids, op.scale, before)


@pytest.mark.parametrize("tokens", [31, 32, 33, 63, 64, 65, 1055, 1056, 1057, 1089, 8192, 8193, 32768 + 40])
def test_runs_that_end_at_chunks(tokens):
    """Runs of equal ids that start and end around multiples of 32 sorted tokens, of every length up to all of them."""
    for split in (0, 1, 31, 32, 33, 64, tokens - 33, tokens - 1):
        if not 0 <= split <= tokens:
            continue
        ids = torch.cat((torch.full((split,), 3), torch.full((tokens - split,), 5))).cuda()
        ids = ids[torch.randperm(tokens, generator=torch.Generator().manual_seed(split))]
        d = _rand(tokens, 40, seed=tokens)
        _check_backward(TokenEmbedding(9, 40).backward(d, ids), d, ids, 1.0)


@pytest.mark.parametrize("vocab", [1, 2, 255, 511, 512, 513, (1 << 18) - 1, 1 << 18, (1 << 20) + 3])
def test_sort_passes(vocab):
    """One to three passes of the sort, with a last tile that is not full."""
    ids, d = _ids(30011, vocab, "uniform", seed=vocab, dtype=torch.int32), _rand(30011, 4, seed=1)
    _check_backward(TokenEmbedding(vocab, 4).backward(d, ids), d, ids, 1.0)


@pytest.mark.parametrize("shift", [0, 1, 2, 4])
@pytest.mark.parametrize("pad", [0, 1, 2, 8])
def test_strided_rows_at_any_offset(pad, shift):
    """Rows with gaps, and tensors that start anywhere; what is between the rows stays."""
    def place(t):
        big = torch.full((t.shape[0] * (t.shape[1] + pad) + shift + 8,), 7.0, dtype=t.dtype, device="cuda")
        view = big[shift:shift + t.shape[0] * (t.shape[1] + pad)].view(t.shape[0], t.shape[1] + pad)[:, :t.shape[1]]
        view.copy_(t)
        return big, view

    op, ids = TokenEmbedding(97, 48), _ids(300, 97, "ends")
    w, d = _rand(97, 48, seed=1, dtype=torch.bfloat16), _rand(300, 48, seed=2, dtype=torch.bfloat16)
    _, ws = place(w)
    _, ds = place(d)
    big, out = place(torch.zeros_like(d))
    op.forward(ws, ids, out=out)
    assert torch.equal(out, op.forward(w, ids))
    out.fill_(7.0)
    assert (big == 7.0).all()
    big, dw = place(torch.zeros_like(w))
    op.backward(ds, ids, out=dw)
    assert torch.equal(dw, op.backward(d, ids))
    dw.fill_(7.0)
    assert (big == 7.0).all()


def test_equal_inputs_give_equal_results():
    op, ids = TokenEmbedding(5000, 200), _ids(20000, 5000, "skewed")
    d = _rand(20000, 200, seed=1, dtype=torch.bfloat16)
    first = op.backward(d, ids)
    for _ in range(5):
        assert torch.equal(op.backward(d, ids), first)


@pytest.mark.parametrize("tokens,vocab", [(0, 5), (0, 0), (5, 0)])
def test_empty(tokens, vocab):
    op = TokenEmbedding(vocab, 64)
    w, ids = _rand(vocab, 64), torch.zeros(tokens, dtype=torch.int64, device="cuda")
    out = op.forward(w, ids)
    assert out.shape == (tokens, 64) and (out == 0).all()
    dw = op.backward(_rand(tokens, 64), ids)
    assert dw.shape == (vocab, 64) and (dw == 0).all()


def test_non_finite_values_stay_in_their_rows():
    op, ids = TokenEmbedding(50, 32), _ids(400, 50, "uniform")
    d = _rand(400, 32, seed=1)
    d[7, 3], d[9, 4] = float("nan"), float("inf")
    want = op.backward(torch.nan_to_num(d, nan=0.0, posinf=0.0), ids)
    got = op.backward(d, ids)
    where = torch.zeros_like(got, dtype=torch.bool)
    where[ids[7], 3] = where[ids[9], 4] = True
    assert torch.equal(got[~where], want[~where]) and not got[where].isfinite().any()


def test_autograd_and_differences():
    op = TokenEmbedding(40, 24, scale=3.0)
    w = _rand(40, 24, seed=1).requires_grad_()
    ids = _ids(2 * 35, 40, "ends").view(2, 35)
    d = _rand(2, 35, 24, seed=2)
    out = op(w, ids)
    dw, = torch.autograd.grad(out, w, d)
    assert torch.equal(dw, op.backward(d, ids))
    step = _rand(40, 24, seed=3)
    # the operator is linear: a difference over any step is the derivative, to rounding
    change = (op.forward((w + step).detach(), ids).double() - out.detach().double()) * d
    scale = (out.detach().abs() * d.abs()).sum() + (dw.abs() * step.abs()).sum()
    assert abs(float(change.sum() - (dw.double() * step).sum())) <= 64 * U * float(scale)
    out = op(w, ids)
    g, = torch.autograd.grad((out * out).sum(), w, create_graph=True)
    with pytest.raises(RuntimeError):
        g.sum().backward()


@pytest.mark.parametrize("tokens,vocab,width", [(3, 5, 1 << 20), (2, 3, (1 << 20) - 1), (200003, 1 << 24, 1), (7000, 1 << 22, 3)])
def test_widest_rows_and_largest_tables(tokens, vocab, width):
    op = TokenEmbedding(vocab, width)
    w, d = _rand(vocab, width, seed=1, dtype=torch.bfloat16), _rand(tokens, width, seed=2, dtype=torch.bfloat16)
    ids = _ids(tokens, vocab, "skewed")
    _check_forward(op.forward(w, ids), w, ids, 1.0)
    _check_backward(op.backward(d, ids), d, ids, 1.0)


def test_far_rows():
    """A table and rows beyond 2^31 elements."""
    vocab, width = 70000, 32768
    w = torch.empty(vocab, width, dtype=torch.bfloat16, device="cuda")
    w[-1] = _rand(width, seed=1)
    w[0] = 1
    ids = torch.tensor([vocab - 1, 0, vocab - 1], device="cuda")
    op = TokenEmbedding(vocab, width)
    out = op.forward(w, ids)
    assert torch.equal(out[0], w[-1]) and torch.equal(out[2], w[-1]) and (out[1] == 1).all()
    dw = op.backward(out, ids)
    assert torch.equal(dw[-1], (2 * w[-1].float()).bfloat16()) and torch.equal(dw[0], w[0])
    assert int(torch.count_nonzero(dw)) == int(torch.count_nonzero(w[-1])) + width


def test_refusals():
    op = TokenEmbedding(10, 16)
    w, ids, d = _rand(10, 16), torch.zeros(4, dtype=torch.int64, device="cuda"), _rand(4, 16)
    for call in (lambda: op.forward(w.cpu(), ids), lambda: op.forward(w, ids.cpu()), lambda: op.forward(w, ids.float()),
                 lambda: op.forward(w.double(), ids), lambda: op.forward(w[:9], ids), lambda: op.forward(w[:, :15], ids),
                 lambda: op.forward(w, ids, dtype=torch.float64), lambda: op.forward(w, ids, out=d[:3]),
                 lambda: op.forward(w, ids, out=d.double()), lambda: op.forward(w, ids, dtype=torch.float16, out=d),
                 lambda: op.forward(w, torch.zeros(8, dtype=torch.int64, device="cuda")[::2]),
                 lambda: op.forward(w.t().contiguous().t(), ids), lambda: op.backward(d[:3], ids),
                 lambda: op.backward(d, ids, accumulate=True), lambda: op.backward(d, ids, out=w[:9]),
                 lambda: op.backward(d.expand(1, 4, 16), ids), lambda: op.backward(d[:1].expand(4, 16), ids),
                 lambda: op.forward(w, ids, out=torch.empty(4, 16)), lambda: op.backward(d, ids, out=torch.empty(10, 16))):
        with pytest.raises(ValueError):
            call()
    for args in ((-1, 4), (1 << 31, 4), (4, 0), (4, (1 << 20) + 1), (4, 4, float("nan")), (4, 4, 1e39)):
        with pytest.raises(ValueError):
            TokenEmbedding(*args)
