"""Build the R-iKFAD CUDA library in-tree for sm_103a.

``python -m paper_2609_30342_gb300.build`` (or ``build()``) compiles
``csrc/*.cu`` and ``csrc/*.cpp`` with nvcc into
``paper_2609_30342_gb300/librikfad.so``.  The CUDA runtime is linked
statically, so the library needs only the driver at run time.
"""
import os
import shutil
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(PKG, "librikfad.so")
OBJDIR = os.path.join(PKG, "_build")
# The checked build: every kernel verifies its plan indices and offsets
# before each access (RIKFAD_CHECKED; see csrc/rikfad_checks.cuh).
LIB_CHECKED = os.path.join(PKG, "librikfad_checked.so")
OBJDIR_CHECKED = os.path.join(PKG, "_build_checked")

ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
NVCC_FLAGS = ["-O3", "-std=c++17", "-lineinfo", "-Xcompiler", "-fPIC", "-Xcompiler",
              "-fvisibility=hidden", "-I", INCLUDE, "-I", CSRC]


def nvcc():
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: the CUDA toolkit is required to build librikfad.so")


# Sources without device-side plan checks: both builds link the same objects.
UNCHECKED = ("rikfad_norm", "rikfad_clip", "rikfad_rotary", "rikfad_embed", "rikfad_distill")


def sources():
    """The translation units, the longest compilations first."""
    names = [f for f in os.listdir(CSRC) if f.endswith((".cu", ".cpp"))]
    return [os.path.join(CSRC, f) for f in sorted(names, key=lambda f: ("norm_backward" not in f, "norm" not in f, f))]


def _stale(lib=LIB):
    """Whether a library or object is missing or older than any source."""
    if not os.path.exists(lib):
        return True
    t = os.path.getmtime(lib)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(INCLUDE, "rikfad.h")]
    return any(os.path.getmtime(d) > t for d in deps)


def build(force=False, verbose=False, extra_flags=(), checked=False):
    """Compile the library if it is missing or older than its sources; return
    its path.  checked=True builds librikfad_checked.so instead, with the
    device-side plan checks compiled in."""
    lib = LIB_CHECKED if checked else LIB
    objdir = OBJDIR_CHECKED if checked else OBJDIR
    if not force and not _stale(lib):
        return lib
    os.makedirs(objdir, exist_ok=True)
    cc = nvcc()
    flags = NVCC_FLAGS + list(extra_flags)

    def compile_one(src):
        name = os.path.basename(src)
        obj = os.path.join(objdir, name + ".o")
        mine = flags + (["-DRIKFAD_CHECKED"] if checked else [])
        if checked and name.startswith(UNCHECKED):
            os.makedirs(OBJDIR, exist_ok=True)
            obj, mine = os.path.join(OBJDIR, name + ".o"), flags
            if not force and not _stale(obj):
                return obj
        cmd = [cc] + ARCH + mine + ["-c", src, "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError("nvcc failed on %s:\n%s%s" % (src, r.stdout, r.stderr))
        if verbose and (r.stdout or r.stderr):
            print(r.stdout + r.stderr, flush=True)
        return obj

    with ThreadPoolExecutor(max_workers=min(16, os.cpu_count() or 4)) as ex:
        objs = list(ex.map(compile_one, sources()))
    tmp = lib + ".tmp%d" % os.getpid()
    cmd = [cc] + ARCH + ["-shared", "-Xcompiler", "-fPIC", "-o", tmp] + objs
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("nvcc link failed:\n%s%s" % (r.stdout, r.stderr))
    os.replace(tmp, lib)
    return lib


if __name__ == "__main__":
    v = "-v" in sys.argv
    extra = ["-Xptxas", "-v"] if "--ptxas" in sys.argv else []
    print(build(force=True, verbose=v or bool(extra), extra_flags=extra, checked="--checked" in sys.argv))
