"""The C ABI's argument checks of the training step's operators that need no GPU, and the fixed-point frequencies."""
import ctypes
import math
import struct

import pytest

from paper_2609_30342_gb300 import build as pkg_build
from paper_2609_30342_gb300 import layers, rikfad


@pytest.fixture(scope="module", autouse=True)
def built():
    pkg_build.build()
    yield


def _clip_create(numel, dtypes, out=None):
    h = ctypes.c_void_p()
    n = len(numel)
    return rikfad.lib().rikfad_clip_create((ctypes.c_int64 * max(n, 1))(*numel), (ctypes.c_int * max(n, 1))(*dtypes),
                                           None if out is None else (ctypes.c_int * n)(*out), n, ctypes.byref(h))


@pytest.mark.parametrize("args", [([-1], [0]), ([5], [3]), ([5], [-1]), ([5], [0], [7]), ([1 << 60], [0])])
def test_clip_plans_are_refused(args):
    assert _clip_create(*args) == rikfad.ERR_ARG
    assert rikfad.lib().rikfad_last_error()


def test_clip_null_arguments():
    L = rikfad.lib()
    assert L.rikfad_clip_create(None, None, None, 2, ctypes.byref(ctypes.c_void_p())) == rikfad.ERR_ARG
    assert L.rikfad_clip_create(None, None, None, -1, ctypes.byref(ctypes.c_void_p())) == rikfad.ERR_ARG
    assert L.rikfad_clip_create(None, None, None, 0, None) == rikfad.ERR_ARG
    assert L.rikfad_clip_run(None, None, None, 1.0, None, None, None) == rikfad.ERR_ARG
    L.rikfad_clip_destroy(None)
    assert L.rikfad_clip_workspace_bytes(None) == 0


def _norm(**kw):
    """A parameter block of 4 rows of 64 bfloat16 with some fields changed (no address is looked at)."""
    f = dict(rows=4, cols=64, gate_rows=1, dtype=1, residual=0, param=0, gate_dtype=0, post=0, pre=1, post_eps=1e-6,
             pre_eps=1e-6, a=1.0, b=1.0, x=0, z=0, gate=0, post_weight=0, pre_weight=0)
    f.update(kw)
    return layers._NORM.pack(f["rows"], f["cols"], f["gate_rows"], f["dtype"], f["residual"], f["param"], f["gate_dtype"],
                             f["post"], f["pre"], f["post_eps"], f["pre_eps"], f["a"], f["b"], f["x"], 64, f["z"], 64,
                             f["gate"], 64, f["post_weight"], 0, f["pre_weight"], 0, *([0] * 21))


@pytest.mark.parametrize("kw", [dict(rows=-1), dict(cols=0), dict(cols=32769), dict(dtype=3), dict(residual=2),
                                dict(param=2), dict(gate_dtype=5), dict(post=3), dict(pre=-1), dict(post_eps=-1.0),
                                dict(pre_eps=math.nan), dict(a=math.inf), dict(b=math.nan), dict(gate=256, gate_rows=3),
                                dict(gate=256, z=256, gate_rows=0), dict(post=1), dict(gate=256),
                                dict(z=256, post_weight=256), dict(pre=0, pre_weight=256)])
def test_norm_arguments_are_refused(kw):
    L = rikfad.lib()
    block = _norm(**kw)
    assert L.rikfad_residual_norm_forward(block, None) == rikfad.ERR_ARG
    assert L.rikfad_residual_norm_backward(block, None) == rikfad.ERR_ARG
    assert L.rikfad_residual_norm_workspace(block) == 0 and rikfad.lib().rikfad_last_error()
    assert L.rikfad_residual_norm_forward(None, None) == rikfad.ERR_ARG


def _rotary(**kw):
    f = dict(batch=1, tokens=2, head_dim=64, rotary_dim=64, layout=0, dtype=1, positions=0, width=8, nlists=1,
             magnitude=1.0, heads=2)
    f.update(kw)
    return layers._ROTARY.pack(f["batch"], f["tokens"], f["head_dim"], f["rotary_dim"], f["layout"], f["dtype"], 256,
                               f["positions"], 0, 0, f["width"], 0, f["nlists"], 0, f["magnitude"],
                               256, 256, f["heads"], *([64] * 6), *([0] * 9))


@pytest.mark.parametrize("kw", [dict(batch=-1), dict(tokens=-1), dict(head_dim=0), dict(head_dim=4097), dict(rotary_dim=3),
                                dict(rotary_dim=66), dict(rotary_dim=-2), dict(layout=2), dict(dtype=9), dict(nlists=3),
                                dict(nlists=-1), dict(magnitude=math.nan), dict(positions=256, width=2), dict(heads=-1),
                                dict(batch=1 << 39, tokens=1 << 39)])
def test_rotary_arguments_are_refused(kw):
    assert rikfad.lib().rikfad_rotary_apply(_rotary(**kw), None) == rikfad.ERR_ARG
    assert rikfad.lib().rikfad_rotary_apply(None, None) == rikfad.ERR_ARG


@pytest.mark.parametrize("batch,tokens,heads,zero", [(1, 1, 2, 5), (1, 2, 1, 4), (2, 1, 1, 3)])
def test_rotary_outputs_that_overlap_themselves_are_refused(batch, tokens, heads, zero):
    strides = [64] * 6
    strides[zero] = 0
    block = layers._ROTARY.pack(batch, tokens, 64, 64, 0, 1, 256, 0, 0, 0, 8, 0, 1, 0, 1.0, 256, 512, heads, *strides,
                                *([0] * 9))
    assert rikfad.lib().rikfad_rotary_apply(block, None) == rikfad.ERR_ARG
    assert b"stride of 0" in rikfad.lib().rikfad_last_error()


def test_turns():
    L = rikfad.lib()
    values = [0.0, math.pi, 2 * math.pi, -math.pi / 2, 1.0, 1e-4, 7.0, 1e300]
    out = (ctypes.c_uint64 * len(values))()
    assert L.rikfad_rotary_turns((ctypes.c_double * len(values))(*values), len(values), out) == rikfad.OK
    for v, t in zip(values[:-1], out):
        turn = v / (2 * math.pi)
        err = (t / 2.0 ** 64 - turn) % 1.0
        assert min(err, 1.0 - err) <= 2.0 ** -52
    assert L.rikfad_rotary_turns((ctypes.c_double * 1)(math.inf), 1, out) == rikfad.ERR_ARG
    assert L.rikfad_rotary_turns(None, 1, out) == rikfad.ERR_ARG
    assert L.rikfad_rotary_turns(None, 0, None) == rikfad.OK


def test_frequencies():
    f, m = layers.rotary_frequencies(8, 10000.0)
    assert f == [10000.0 ** (-i / 4) for i in range(4)] and m == 1.0
    assert layers.rotary_frequencies(8, 10000.0, dict(kind="linear", factor=2.0))[0] == [v / 2 for v in f]
    b, _ = layers.rotary_frequencies(8, 10000.0, dict(kind="base", factor=4.0))
    assert b[0] == f[0] and abs(b[-1] * 4 / f[-1] - 1) < 1e-12
    r, m = layers.rotary_frequencies(64, 10000.0, dict(kind="ramp", factor=8.0, original_context=1024))
    g, _ = layers.rotary_frequencies(64, 10000.0)
    assert r[0] == g[0] and abs(r[-1] * 8 / g[-1] - 1) < 1e-12 and abs(m - (0.1 * math.log(8.0) + 1)) < 1e-12
    assert all(a <= b for a, b in zip(r, g))
    assert layers.rotary_frequencies(0) == ([], 1.0)
    for bad in (dict(kind="cubic"), dict(kind="linear", factor=0.5), dict(kind="ramp", factor=2.0)):
        with pytest.raises(ValueError):
            layers.rotary_frequencies(8, 10000.0, bad)
    with pytest.raises(ValueError):
        layers.rotary_frequencies(7)


def test_parameter_blocks_have_the_size_of_the_structs(tmp_path):
    import subprocess
    src = tmp_path / "sizes.c"
    src.write_text('#include <stdio.h>\n#include "rikfad.h"\nint main(void) { printf("%zu %zu", '
                   'sizeof(rikfad_residual_norm), sizeof(rikfad_rotary)); return 0; }\n')
    exe = tmp_path / "sizes"
    subprocess.run(["gcc", "-I", pkg_build.INCLUDE, str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout
    assert out.split() == [str(layers._NORM.size), str(layers._ROTARY.size)]


@pytest.mark.parametrize("kw", [dict(numels=[3], dtypes="f64"), dict(numels=[3, 4], dtypes=["f32"]),
                                dict(numels=[3], dtypes=[["f32"]])])
def test_clipper_types_are_checked(kw):
    from paper_2609_30342_gb300.gradients import GradientClipper
    with pytest.raises(ValueError):
        GradientClipper(**kw)
