"""Losses of rows of logits, with their gradients.

``DistillationLoss``   against a teacher's top logits and a label; without a teacher the cross entropy

It has explicit calls on CUDA tensors (``forward``, ``loss_and_gradient``, ``backward``) and is callable inside autograd.
Argument checks and marshalling only: the work runs in the kernels behind ``rikfad_distillation_forward`` and
``rikfad_distillation_backward``, enqueued on the current stream of the tensors' device (or ``stream``, to which what the
call allocates then belongs; the inputs have to be ready on it).  A tensor given as ``out`` counts as changed in autograd.
"""
import math
import struct

import torch

from . import rikfad
from .layers import _F32, _TORCH, _matrix, _streaming

# struct rikfad_distillation: sizes, types, weights, (pointer, stride) pairs of the inputs, labels, results, dlogits
_DISTILLATION = struct.Struct("=2q 6i 4d 6q q 3q 2q")
_INTS = {torch.int32: 4, torch.int64: 8}


def _rows_of(name, t, cols, device, rows):
    """A tensor as ``rows`` rows of ``cols`` contiguous elements: (pointer, row stride)."""
    if t.get_device() != device:
        raise ValueError("%s must be a CUDA tensor on the device of the logits" % name)
    if t.dim() != 2:
        t = _matrix(name, t, cols)
    n, c = t.shape
    if n != rows or c != cols:
        raise ValueError("%s is %d rows of %d columns, expected %d of %d" % (name, n, c, rows, cols))
    s0, s1 = t.stride()
    if n and s1 != 1 and cols > 1 or s0 < cols and n > 1:       # without elements strides say nothing
        raise ValueError("the rows of %s must be contiguous and not overlap" % name)
    return t.data_ptr(), s0 if n > 1 else cols


class DistillationLoss:
    """Of every row of logits s, against K logits t of a teacher at indices i (its largest, say) and against a label:

        p = softmax(t / T)
        loss = teacher_weight T^2 sum_k p_k (log p_k - log softmax(s / T)[i_k]) - label_weight log softmax(s)[label]

    Teacher entries whose index is outside [0, vocab) or whose logit is -inf are absent, and so are labels outside
    [0, vocab); a row with neither has a loss and a gradient of 0.  Either of teacher and labels may be None.  Entries
    that name one element add up.  K is 1024 at most.

    Logits are [..., vocab] in float32, bfloat16 or float16, the teacher's [..., K] in any of them, ``index`` [..., K] and
    ``labels`` [...] int32 or int64.  Rows are contiguous and evenly spaced, labels contiguous.  Losses are float32, one a
    row.  Only the logits have a gradient."""

    def __init__(self, temperature=1.0, teacher_weight=1.0, label_weight=0.0):
        self.temperature, self.teacher_weight, self.label_weight = float(temperature), float(teacher_weight), float(label_weight)
        if not 1e-3 <= self.temperature <= 1e3:
            raise ValueError("temperature must be in [0.001, 1000]")
        for w in (self.teacher_weight, self.label_weight):
            if not abs(w) <= 1e30:
                raise ValueError("weights must be in [-1e30, 1e30]")

    def _inputs(self, logits, teacher, index, labels):
        """The parameter block up to the logits' rows, the others' and the labels, and (rows, vocab, device)."""
        for t in (logits, teacher, index, labels):
            if t is not None and not isinstance(t, torch.Tensor):
                raise ValueError("inputs must be tensors")
        device = logits.get_device()
        if device < 0 or logits.dtype not in _TORCH or logits.dim() == 0:
            raise ValueError("logits must be a CUDA tensor [..., vocab] of float32, bfloat16 or float16")
        lead, vocab = logits.shape[:-1], logits.shape[-1]
        if not 1 <= vocab <= 1 << 24:
            raise ValueError("the vocabulary must be in [1, 2^24]")
        rows = math.prod(lead)
        if (teacher is None) != (index is None):
            raise ValueError("teacher and index belong together")
        if teacher is None and labels is None:
            raise ValueError("need a teacher or labels")
        pl, sl = _rows_of("logits", logits, vocab, device, rows)
        k = pt = st = pi = si = py = 0
        tt, ib, yb = rikfad.F32, 8, 8
        if teacher is not None:
            if teacher.dtype not in _TORCH:
                raise ValueError("teacher must be float32, bfloat16 or float16")
            if index.dtype not in _INTS:
                raise ValueError("index must be int32 or int64")
            if teacher.dim() == 0 or teacher.shape[:-1] != lead or index.shape != teacher.shape:
                raise ValueError("teacher and index must be [..., K] with the leading sizes of the logits")
            k, tt, ib = teacher.shape[-1], _TORCH[teacher.dtype], _INTS[index.dtype]
            if not 0 <= k <= 1024:
                raise ValueError("K must be at most 1024")
            if k:
                pt, st = _rows_of("teacher", teacher, k, device, rows)
                pi, si = _rows_of("index", index, k, device, rows)
        if labels is not None:
            if labels.dtype not in _INTS or labels.get_device() != device or labels.shape != lead or not labels.is_contiguous():
                raise ValueError("labels must be contiguous int32 or int64, one for every row, on the device of the logits")
            py, yb = labels.data_ptr(), _INTS[labels.dtype]
        head = (rows, vocab, k, _TORCH[logits.dtype], tt, ib, yb, 0, self.temperature, self.teacher_weight, self.label_weight)
        return head, (pl, sl, pt, st, pi, si, py), lead, rows, vocab, device

    @staticmethod
    def _gradient(logits, out, rows, vocab, device):
        """The tensor for the gradient, and its (pointer, row stride)."""
        if out is None:
            out = torch.empty_like(logits, memory_format=torch.contiguous_format)
            return out, (out.data_ptr(), vocab)
        if not isinstance(out, torch.Tensor) or out.dtype is not logits.dtype or out.shape != logits.shape:
            raise ValueError("out must have the shape and type of the logits")
        return out, _rows_of("out", out, vocab, device, rows)

    @staticmethod
    def _per_row(dloss, lead, device):
        if not isinstance(dloss, torch.Tensor) or dloss.dtype is not _F32 or dloss.get_device() != device \
                or dloss.shape != lead or not dloss.is_contiguous():
            raise ValueError("dloss must be contiguous float32, one for every row, on the device of the logits")
        return dloss.data_ptr()

    def forward(self, logits, teacher=None, index=None, labels=None, need_stats=True, stream=None):
        """(loss, stats).  ``stats`` (None without ``need_stats``) is what ``backward`` needs besides the inputs."""
        if stream is not None:
            with _streaming(stream, logits):
                return self.forward(logits, teacher, index, labels, need_stats)
        head, inputs, lead, rows, _, device = self._inputs(logits, teacher, index, labels)
        loss = torch.empty(lead, dtype=_F32, device=logits.device)
        stats = torch.empty(rows, 4, dtype=_F32, device=logits.device) if need_stats else None
        block = _DISTILLATION.pack(*head, 1.0, *inputs, loss.data_ptr(), 0 if stats is None else stats.data_ptr(), 0, 0, 0)
        rikfad._call_on(device, rikfad.lib().rikfad_distillation_forward, block, rikfad._raw_stream(device))
        return loss, stats

    def loss_and_gradient(self, logits, teacher=None, index=None, labels=None, grad_scale=1.0, dloss=None, out=None,
                          stream=None):
        """(loss, gradient of the logits) in one pass: that of ``grad_scale`` times the sum of the losses, each times its
        ``dloss`` if given.  ``out`` to write the gradient to; the logits themselves for in place."""
        if stream is not None:
            with _streaming(stream, logits):
                return self.loss_and_gradient(logits, teacher, index, labels, grad_scale, dloss, out)
        head, inputs, lead, rows, vocab, device = self._inputs(logits, teacher, index, labels)
        per_row = 0 if dloss is None else self._per_row(dloss, lead, device)
        loss = torch.empty(lead, dtype=_F32, device=logits.device)
        given = out
        out, to = self._gradient(logits, out, rows, vocab, device)
        block = _DISTILLATION.pack(*head, float(grad_scale), *inputs, loss.data_ptr(), 0, per_row, *to)
        rikfad._call_on(device, rikfad.lib().rikfad_distillation_forward, block, rikfad._raw_stream(device))
        if given is not None:
            rikfad._written(given)
        return loss, out

    def backward(self, dloss, logits, teacher=None, index=None, labels=None, stats=None, grad_scale=1.0, out=None,
                 stream=None):
        """The gradient of the logits, from that of the losses (None: 1) and the forward call's ``stats``."""
        if stream is not None:
            with _streaming(stream, logits):
                return self.backward(dloss, logits, teacher, index, labels, stats, grad_scale, out)
        head, inputs, lead, rows, vocab, device = self._inputs(logits, teacher, index, labels)
        per_row = 0 if dloss is None else self._per_row(dloss, lead, device)
        if not isinstance(stats, torch.Tensor) or stats.dtype is not _F32 or stats.shape != (rows, 4) \
                or not stats.is_contiguous() or stats.get_device() != device:
            raise ValueError("stats must be what forward returned for these inputs")
        given = out
        out, to = self._gradient(logits, out, rows, vocab, device)
        block = _DISTILLATION.pack(*head, float(grad_scale), *inputs, 0, stats.data_ptr(), per_row, *to)
        rikfad._call_on(device, rikfad.lib().rikfad_distillation_backward, block, rikfad._raw_stream(device))
        if given is not None:
            rikfad._written(given)
        return out

    def __call__(self, logits, teacher=None, index=None, labels=None):
        """The rows' losses inside autograd."""
        return _DistillationFunction.apply(self, logits, teacher, index, labels)


class _DistillationFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, op, logits, teacher, index, labels):
        loss, stats = op.forward(logits, teacher, index, labels)
        ctx.op = op
        ctx.save_for_backward(logits, teacher, index, labels, stats)
        return loss

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dloss):
        return None, ctx.op.backward(dloss.contiguous(), *ctx.saved_tensors), None, None, None
