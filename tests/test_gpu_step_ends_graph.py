"""The token embedding, the heads' norms with rotation and the loss against a teacher captured in graphs, on other streams
than the current one, and two graphs at a time."""
import pytest
import torch

from paper_2609_30342_gb300 import build as pkg_build
from paper_2609_30342_gb300.embedding import TokenEmbedding
from paper_2609_30342_gb300.layers import RotaryNorm
from paper_2609_30342_gb300.losses import DistillationLoss

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    pkg_build.build()
    yield


def _rand(*shape, seed=0, dtype=torch.bfloat16):
    return torch.randn(shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).to(dtype)


def _ids(high, *shape, seed=0):
    return torch.randint(-1, high, shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))


def _embedding(tokens, width):
    op = TokenEmbedding(700, width)
    weight, d, ids = _rand(700, width), _rand(tokens, width, seed=1), _ids(700, tokens)

    def fill(seed):
        weight.copy_(_rand(700, width, seed=seed))
        d.copy_(_rand(tokens, width, seed=seed + 1))
        ids.copy_(_ids(700, tokens, seed=seed))
    return fill, lambda stream=None: [op.forward(weight, ids, stream=stream), op.backward(d, ids, stream=stream)]


def _heads(tokens, head_dim):
    op = RotaryNorm(head_dim)
    q, k, dq, dk = (_rand(tokens, h, head_dim, seed=i) for i, h in enumerate((6, 2, 6, 2)))
    w, positions = _rand(head_dim, seed=5), torch.arange(tokens, device="cuda")

    def fill(seed):
        for i, t in enumerate((q, k, dq, dk)):
            t.copy_(_rand(*t.shape, seed=seed + i))
        positions.copy_(torch.randperm(tokens, device="cuda"))
    return fill, lambda stream=None: [*op.forward(q, k, w, w, positions, stream=stream),
                                      *op.backward(dq, dk, q, k, w, w, positions, stream=stream)]


def _loss(rows, vocab):
    op = DistillationLoss(2.0, 1.0, 0.5)
    logits, teacher, index, labels = _rand(rows, vocab), _rand(rows, 9, seed=1), _ids(vocab, rows, 9), _ids(vocab, rows, seed=2)

    def fill(seed):
        logits.copy_(_rand(rows, vocab, seed=seed))
        teacher.copy_(_rand(rows, 9, seed=seed + 1))
        index.copy_(_ids(vocab, rows, 9, seed=seed))
        labels.copy_(_ids(vocab, rows, seed=seed + 2))

    def call(stream=None):
        loss, stats = op.forward(logits, teacher, index, labels, stream=stream)
        return [loss, op.backward(None, logits, teacher, index, labels, stats, stream=stream),
                *op.loss_and_gradient(logits, teacher, index, labels, stream=stream)]
    return fill, call


CASES = [(_embedding, 1, 64), (_embedding, 3000, 64), (_embedding, 9000, 41), (_heads, 1, 64), (_heads, 700, 64),
         (_heads, 333, 70), (_loss, 1, 5001), (_loss, 40, 5001), (_loss, 3, 150000)]


def _capture(call):
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    return graph, out


@pytest.mark.parametrize("make,n,size", CASES)
def test_replays_work_on_what_the_inputs_hold(make, n, size):
    fill, call = make(n, size)
    graph, out = _capture(call)
    for seed in (50, 60):
        fill(seed)
        want = [t.clone() for t in call()]
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


@pytest.mark.parametrize("make,n,size", CASES)
def test_two_graphs_at_a_time(make, n, size):
    """Each has workspaces of its own: replays side by side on two streams do not disturb each other."""
    pairs = []
    for seed in (70, 80):
        fill, call = make(n, size)
        fill(seed)
        want = [t.clone() for t in call()]
        pairs.append((*_capture(call), want, call))
    streams = [torch.cuda.Stream() for _ in pairs]
    torch.cuda.synchronize()
    for _ in range(5):
        for (graph, *_), s in zip(pairs, streams):
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    for _, out, want, _ in pairs:
        assert all(torch.equal(a, b) for a, b in zip(out, want))


@pytest.mark.parametrize("make,n,size", CASES)
def test_other_streams(make, n, size):
    fill, call = make(n, size)
    fill(90)
    want = call()
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    for s in (stream, stream.cuda_stream):
        got = call(s)
        stream.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_later_call_on_the_stream_sees_the_results():
    """Two calls, the second on the first one's results, without a wait of the host's between them."""
    table, loss = TokenEmbedding(300, 512), DistillationLoss(label_weight=1.0)
    weight, ids, labels = _rand(300, 512), _ids(300, 4000), _ids(512, 4000, seed=3)
    for _ in range(5):
        rows = table.forward(weight, ids)
        _, d = loss.loss_and_gradient(rows, labels=labels)
        got = table.backward(d, ids)
    torch.cuda.synchronize()
    rows = table.forward(weight, ids)
    torch.cuda.synchronize()
    _, d = loss.loss_and_gradient(rows, labels=labels)
    torch.cuda.synchronize()
    assert torch.equal(got, table.backward(d, ids))
