"""The C ABI's argument checks, without a GPU, of the token embedding, the heads' norms with rotation and the loss against a
teacher."""
import math
import subprocess

import pytest

from paper_2609_30342_gb300 import build as pkg_build
from paper_2609_30342_gb300 import embedding, layers, losses, rikfad


@pytest.fixture(scope="module", autouse=True)
def built():
    pkg_build.build()
    yield


def _embedding(**kw):
    f = dict(tokens=4, vocab=9, width=64, table=0, dtype=1, id_bytes=8, scale=1.0)
    f.update(kw)
    return embedding._EMBEDDING.pack(f["tokens"], f["vocab"], f["width"], f["table"], f["dtype"], f["id_bytes"], 0, f["scale"],
                                     256, 256, 64, 256, 64, 0, 0)


@pytest.mark.parametrize("kw", [dict(tokens=-1), dict(tokens=(1 << 30) + 1), dict(vocab=-1), dict(vocab=1 << 31),
                                dict(width=0), dict(width=(1 << 20) + 1), dict(table=3), dict(dtype=-1), dict(id_bytes=2),
                                dict(scale=math.nan), dict(scale=1e39)])
def test_embedding_arguments_are_refused(kw):
    L = rikfad.lib()
    block = _embedding(**kw)
    assert L.rikfad_embedding_forward(block, None) == rikfad.ERR_ARG
    assert L.rikfad_embedding_backward(block, None) == rikfad.ERR_ARG
    assert L.rikfad_embedding_workspace(block) == 0 and L.rikfad_last_error()
    assert L.rikfad_embedding_forward(None, None) == rikfad.ERR_ARG


@pytest.mark.parametrize("tokens,vocab,width,dtype", [(1, 1, 1, 0), (8, 50257, 768, 1), (4099, 8191, 1001, 2),
                                                      (65536, 131072, 4096, 1), (131072, 5, 1525, 1), (1 << 30, 9, 8, 0)])
def test_embedding_workspace(tokens, vocab, width, dtype):
    """Two lists of entries, and two partial rows of a chunk of 8 to 256 tokens."""
    n = rikfad.lib().rikfad_embedding_workspace(_embedding(tokens=tokens, vocab=vocab, width=width, dtype=dtype))
    assert 16 * tokens <= n <= 16 * tokens + 64 + 4 * (tokens // 8 + 4) + 8 * (tokens // 8 + 1) * (width + 3)
    assert rikfad.lib().rikfad_embedding_workspace(_embedding(tokens=0)) == 0


def _rotary_norm(strides=(0,) * 9, lists=1, **kw):
    f = dict(batch=1, tokens=2, head_dim=64, rotary_dim=64, layout=0, dtype=1, positions=0, width=8, param=0, nlists=lists,
             magnitude=1.0, eps=1e-6, heads=2)
    f.update(kw)
    return layers._ROTARY_NORM.pack(f["batch"], f["tokens"], f["head_dim"], f["rotary_dim"], f["layout"], f["dtype"], 256,
                                    f["positions"], 0, 0, f["width"], f["param"], f["nlists"], 0, f["magnitude"], f["eps"],
                                    256, 0, 0, 512, 0, f["heads"], *strides, *([0] * 15), 0, 0)


_DENSE = (256, 128, 64) * 3


@pytest.mark.parametrize("kw", [dict(batch=-1), dict(tokens=-1), dict(head_dim=0), dict(head_dim=513), dict(rotary_dim=3),
                                dict(rotary_dim=66), dict(rotary_dim=-2), dict(layout=2), dict(dtype=9), dict(nlists=3),
                                dict(nlists=-1), dict(magnitude=math.nan), dict(eps=-1.0), dict(eps=math.inf), dict(param=2),
                                dict(positions=256, width=2), dict(heads=-1), dict(heads=1 << 17),
                                dict(batch=1 << 39, tokens=1 << 39)])
def test_rotary_norm_arguments_are_refused(kw):
    L = rikfad.lib()
    block = _rotary_norm(_DENSE, **kw)
    assert L.rikfad_rotary_norm_forward(block, None) == rikfad.ERR_ARG
    assert L.rikfad_rotary_norm_backward(block, None) == rikfad.ERR_ARG
    assert L.rikfad_rotary_norm_workspace(block) == 0 and L.rikfad_last_error()
    assert L.rikfad_rotary_norm_forward(None, None) == rikfad.ERR_ARG


@pytest.mark.parametrize("batch,tokens,heads,zero", [(1, 1, 2, 5), (1, 2, 1, 4), (2, 1, 1, 3)])
def test_rotary_norm_outputs_that_overlap_themselves_are_refused(batch, tokens, heads, zero):
    strides = list(_DENSE)
    strides[zero] = 0
    block = _rotary_norm(strides, batch=batch, tokens=tokens, heads=heads)
    assert rikfad.lib().rikfad_rotary_norm_forward(block, None) == rikfad.ERR_ARG
    assert b"stride of 0" in rikfad.lib().rikfad_last_error()


def _distillation(**kw):
    f = dict(rows=4, vocab=100, k=3, dtype=1, teacher=0, index=8, label=8, T=2.0, a=1.0, b=0.5, g=1.0, labels=256)
    f.update(kw)
    return losses._DISTILLATION.pack(f["rows"], f["vocab"], f["k"], f["dtype"], f["teacher"], f["index"], f["label"], 0, f["T"],
                                     f["a"], f["b"], f["g"], 256, 100, 256, 3, 256, 3, f["labels"], 256, 256, 0, 0, 0)


@pytest.mark.parametrize("kw", [dict(rows=-1), dict(rows=1 << 29), dict(vocab=0), dict(vocab=(1 << 24) + 1), dict(k=-1),
                                dict(k=1025), dict(dtype=3), dict(teacher=-1), dict(index=2), dict(label=1), dict(T=0.0),
                                dict(T=math.nan), dict(T=1e4), dict(a=math.inf), dict(b=math.nan), dict(g=1e39),
                                dict(a=1e38, T=1e3)])
def test_distillation_arguments_are_refused(kw):
    L = rikfad.lib()
    block = _distillation(**kw)
    assert L.rikfad_distillation_forward(block, None) == rikfad.ERR_ARG
    assert L.rikfad_distillation_backward(block, None) == rikfad.ERR_ARG
    assert L.rikfad_distillation_forward(None, None) == rikfad.ERR_ARG and L.rikfad_last_error()


def test_parameter_blocks_have_the_size_of_the_structs(tmp_path):
    src = tmp_path / "sizes.c"
    src.write_text('#include <stdio.h>\n#include "rikfad.h"\nint main(void) { printf("%zu %zu %zu", sizeof(rikfad_embedding), '
                   'sizeof(rikfad_rotary_norm), sizeof(rikfad_distillation)); return 0; }\n')
    exe = tmp_path / "sizes"
    subprocess.run(["gcc", "-I", pkg_build.INCLUDE, str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout
    assert out.split() == [str(s.size) for s in (embedding._EMBEDDING, layers._ROTARY_NORM, losses._DISTILLATION)]
