"""The table's gradient where runs of equal ids meet the chunks that warps sum, for every size of chunk.

A warp sums a chunk of 8 to 256 sorted tokens, 32 at a time; a run of equal ids over several chunks is joined by one warp
where it goes on in up to 32 chunks after its first, by a block where in more.  The runs here start and end at a chunk's
ends and within it and go on in 0, 1, 2, 31, 32, 33, 34 and 67 chunks, whatever the chunk's size, which is taken from the
size of the workspace.  Gradients of rows are whole numbers of magnitude 2 or less, of fewer than 2^22 tokens: every sum is
exact in float32 in any order, and so is the scale, a power of two.  Results have to be equal."""
import pytest
import torch

from paper_2609_30342_gb300 import build as pkg_build
from paper_2609_30342_gb300 import embedding, rikfad
from paper_2609_30342_gb300.embedding import TokenEmbedding

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module", autouse=True)
def built():
    pkg_build.build()
    yield


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _chunk(tokens, vocab, width, dtype):
    """From the bytes of the workspace: two lists of entries, one of chunks, two partial rows a chunk."""
    block = embedding._EMBEDDING.pack(tokens, vocab, width, 0, dtype, 8, 0, 1.0, 256, 256, width, 256, width, 0, 0)
    nbytes = rikfad.lib().rikfad_embedding_workspace(block)
    fits = []
    for chunk in (8, 16, 32, 64, 128, 256):
        chunks = -(-tokens // chunk)
        if 2 * (-(-8 * tokens // 16) * 16) + (chunks + 2 + 3) // 4 * 16 + 8 * chunks * (-(-width // 4) * 4) == nbytes:
            fits.append(chunk)
    assert len(fits) == 1
    return fits[0]


def _runs(tokens, chunk):
    """Lengths of runs: each of the long ones starts `lead` places into a chunk and ends `end` into its last."""
    lengths = []
    for on, lead, end in ((31, 5, 1), (32, 0, chunk), (33, chunk - 1, 7), (34, 1, chunk), (32, 3, chunk // 2), (1, 0, 1),
                          (2, 7, chunk - 1), (0, 0, chunk), (67, chunk // 2, 3)):
        at = sum(lengths) % chunk
        gap = (lead - at) % chunk
        lengths += [1] * (gap % 3) + ([gap - gap % 3] if gap >= 3 else [])
        lengths.append(chunk - lead + (on - 1) * chunk + end if on else end)
    left = tokens - sum(lengths)
    assert left > 0
    n = 1
    while left > 0:                             # the rest: short runs of every length
        lengths.append(min(n % 71 + 1, left))
        left -= lengths[-1]
        n += 1
    return lengths


# tokens: about as many as the chunk's size is chosen for at that width
CASES = [(8, 3001, 64, "f32"), (8, 3001, 67, "f32"), (16, 6003, 1032, "bf16"), (16, 6003, 1031, "bf16"), (32, 12005, 2052, "f32"),
         (32, 12005, 2047, "f16"), (64, 19999, 4096, "f32"), (64, 19999, 4097, "f32"), (64, 39998, 4096, "bf16"),
         (128, 40005, 4096, "f32"), (128, 40005, 4095, "f32"), (128, 80010, 4095, "bf16"), (256, 80003, 4096, "f32"),
         (256, 80003, 4097, "f32"), (256, 160003, 4096, "bf16")]


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("chunk,tokens,width,dtype", CASES)
def test_runs_over_chunks(chunk, tokens, width, dtype, accumulate):
    lengths = _runs(tokens, chunk)
    vocab = 2 * len(lengths) + 2                # every second row has no token
    assert _chunk(tokens, vocab, width, {"f32": 0, "bf16": 1, "f16": 2}[dtype]) == chunk
    ids = torch.repeat_interleave(2 * torch.arange(len(lengths)) + 1, torch.tensor(lengths)).cuda()
    ids = ids[torch.randperm(tokens, device="cuda", generator=_gen(tokens))]
    d = torch.randint(-2, 3, (tokens, width), device="cuda", generator=_gen(1), dtype=torch.int8).to(DT[dtype])
    op = TokenEmbedding(vocab, width, scale=0.5)
    want = torch.zeros(vocab, width, device="cuda").index_add_(0, ids, d.float()).mul_(0.5)
    out = torch.zeros_like(want)
    if accumulate:
        out.copy_(torch.randint(-9, 9, out.shape, device="cuda", generator=_gen(2)))
        want += out
    got = op.backward(d, ids, out=out, accumulate=accumulate) if accumulate else op.backward(d, ids, dtype=torch.float32)
    assert torch.equal(got, want)


@pytest.mark.parametrize("tokens,width,dtype", [(20001, 4096, "f32"), (80002, 4095, "bf16")])
def test_one_id_and_padding(tokens, width, dtype):
    """One run over all chunks; one that ends where the tokens outside the table begin."""
    d = torch.randint(-2, 3, (tokens, width), device="cuda", generator=_gen(3), dtype=torch.int8).to(DT[dtype])
    op = TokenEmbedding(3, width)
    for kept in (tokens, tokens - 1, tokens // 2, 1, 0):
        ids = torch.where(torch.arange(tokens, device="cuda") < kept, 1, -1)
        got = op.backward(d, ids, dtype=torch.float32)
        assert torch.equal(got[1], d[:kept].sum(0, dtype=torch.float32)) and int(torch.count_nonzero(got[::2])) == 0
