"""Norm of a gradient list and clipping, before the optimiser's step.

``GradientClipper(numels, dtypes, out_dtypes)`` plans a fixed list, as ``rikfad.RIKFAD`` does; ``norm`` gives the
2-norm of every gradient and of all of them, ``clip`` also scales the gradients to a largest total norm, in place or
into other tensors, of another type if need be (fp32 gradients summed over micro-batches to the bf16 ones that a handle
takes).  Argument marshalling only: the work runs in the kernels behind ``rikfad_clip_run``.
"""
import contextlib
import ctypes

import torch

from . import rikfad

_TORCH = {torch.float32: rikfad.F32, torch.bfloat16: rikfad.BF16, torch.float16: rikfad.F16}
_NAMES = {**rikfad.DTYPE_CODES, **_TORCH}


def _codes(dtypes, n):
    each = [dtypes] * n if isinstance(dtypes, (str, torch.dtype)) else list(dtypes)
    if len(each) != n:
        raise ValueError("need one dtype per tensor")
    try:
        return [_NAMES[d] for d in each]
    except (KeyError, TypeError):
        raise ValueError("dtypes must be 'f32', 'bf16', 'f16' or the torch types") from None


class ClipPointers:
    """Checked, packed pointers of one set of gradients and outputs."""

    def __init__(self, grads, out, grad_array, out_array):
        self.keep = (grads, out)
        self.grads, self.out = grad_array, out_array
        self.device = next((t.device for t in grads if t.is_cuda), None)
        if self.device is None:
            self.device = torch.device("cuda", torch.cuda.current_device())


class GradientClipper:
    """``numels``: elements of each tensor; ``dtypes``: "f32", "bf16" or "f16", one for all or one each;
    ``out_dtypes``: those of the clipped gradients (default: the same); ``device``: where the gradients are (default: the
    current device)."""

    def __init__(self, numels, dtypes="bf16", out_dtypes=None, device=None):
        self.numels = [int(n) for n in numels]
        n = len(self.numels)
        self._in = _codes(dtypes, n)
        self._out = self._in if out_dtypes is None else _codes(out_dtypes, n)
        h = ctypes.c_void_p()
        self._h = None
        with contextlib.nullcontext() if device is None else torch.cuda.device(device):
            rikfad._check(rikfad.lib().rikfad_clip_create((ctypes.c_int64 * max(n, 1))(*self.numels),
                                                          (ctypes.c_int * max(n, 1))(*self._in),
                                                          (ctypes.c_int * max(n, 1))(*self._out), n, ctypes.byref(h)))
        self._h = h

    @property
    def handle(self):
        if self._h is None:
            raise RuntimeError("clipper is closed")
        return self._h

    def close(self):
        if getattr(self, "_h", None) is not None:
            rikfad.lib().rikfad_clip_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def workspace_bytes(self):
        return rikfad.lib().rikfad_clip_workspace_bytes(self.handle)

    def _packed(self, tensors, codes, what):
        tensors = list(tensors)
        if len(tensors) != len(self.numels):
            raise ValueError("need one %s per tensor of the plan" % what)
        if list(map(torch.Tensor.numel, tensors)) != self.numels:
            raise ValueError("a %s has another number of elements than planned" % what)
        if [_TORCH.get(t.dtype) for t in tensors] != codes:
            raise ValueError("a %s has another dtype than planned" % what)
        if not all(map(torch.Tensor.is_contiguous, tensors)):
            raise ValueError("every %s must be contiguous" % what)
        for t in tensors:
            if not (t.is_cuda or t.is_pinned()):
                raise ValueError("every %s must be a CUDA tensor or page-locked" % what)
        return tensors, rikfad.pointer_array(tensors)

    def pack(self, grads, out=None):
        """Check and pack one set of tensors, for loops that pass the same ones every time."""
        grads, g = self._packed(grads, self._in, "gradient")
        if out is None:
            return ClipPointers(grads, None, g, None)
        out, o = self._packed(out, self._out, "output")
        return ClipPointers(grads, out, g, o)

    def _run(self, ptrs, out, max_norm, stream):
        device = ptrs.device
        if stream is not None:
            with rikfad._streaming(stream, device.index):
                return self._run(ptrs, out, max_norm, None)
        total = torch.empty((), dtype=torch.float32, device=device)
        norms = torch.empty(len(self.numels), dtype=torch.float32, device=device)
        run = rikfad.lib().rikfad_clip_run
        args = (self.handle, ptrs.grads, out, max_norm, norms.data_ptr(), total.data_ptr(),
                rikfad._raw_stream(device.index))
        code = run(*args)
        if code == rikfad.ERR_STATE:        # another device is current: nothing was enqueued
            with torch.cuda.device(device):
                code = run(*args)
        rikfad._check(code)
        return total, norms

    def norm(self, grads=None, stream=None, ptrs=None):
        """(total, norms): the 2-norm of all gradients (a scalar CUDA tensor) and of each, enqueued on ``stream``."""
        return self._run(self.pack(grads) if ptrs is None else ptrs, None, 0.0, stream)

    def clip(self, max_norm, grads=None, out=None, stream=None, ptrs=None):
        """(total, norms) as ``norm`` gives them, and the gradients times ``max_norm / total`` where the total is
        larger (and finite), into ``out`` (in place by default)."""
        if ptrs is None:
            grads = list(grads)
            ptrs = self.pack(grads, grads if out is None else out)
        elif ptrs.out is None:
            raise ValueError("the packed pointers have no outputs")
        return self._run(ptrs, ptrs.out, float(max_norm), stream)
