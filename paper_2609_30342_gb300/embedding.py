"""Token embedding: rows of a table by id, scaled, and the table's dense gradient from the tokens sorted by id.

``TokenEmbedding`` has explicit calls on CUDA tensors (``forward``, ``backward``) and is callable inside autograd.
Argument checks and marshalling only: the work runs in the kernels behind ``rikfad_embedding_forward`` and
``rikfad_embedding_backward``, enqueued on the current stream of the tensors' device (or ``stream``, to which what the
call allocates then belongs; the inputs have to be ready on it).  A tensor given as ``out`` counts as changed in autograd.
"""
import math
import struct

import torch

from . import rikfad
from .layers import _TORCH, _rows, _streaming

# struct rikfad_embedding: sizes, types, scale, ids, (pointer, stride) pairs, workspace
_EMBEDDING = struct.Struct("=3q 4i d q 4q qQ")


class TokenEmbedding:
    """out = scale * weight[ids], a row of zeros where an id is outside [0, vocab) (padding).

    weight and rows are float32, bfloat16 or float16, in any combination; ids int32 or int64 of any shape, contiguous."""

    def __init__(self, vocab, width, scale=1.0):
        self.vocab, self.width, self.scale = int(vocab), int(width), float(scale)
        if not 0 <= self.vocab <= 1 << 30:
            raise ValueError("vocab must be in [0, 2^30]")
        if not 1 <= self.width <= 1 << 20:
            raise ValueError("width must be in [1, 2^20]")
        if not math.isfinite(self.scale) or abs(self.scale) > 3e38:
            raise ValueError("scale must be finite in float32")
        self._workspace = {}        # bytes by sizes and types

    def _ids(self, ids, device):
        """(address, bytes of an id, tokens)."""
        if not isinstance(ids, torch.Tensor) or ids.dtype not in (torch.int32, torch.int64):
            raise ValueError("ids must be an int32 or int64 tensor")
        if ids.get_device() != device:
            raise ValueError("ids must be on the device of the other tensors")
        if not ids.is_contiguous():
            raise ValueError("ids must be contiguous")
        return ids.data_ptr(), ids.element_size(), ids.numel()

    @staticmethod
    def _device(t):
        if not isinstance(t, torch.Tensor) or not t.is_cuda:
            raise ValueError("inputs must be CUDA tensors")
        if t.dtype not in _TORCH:
            raise ValueError("weight and rows must be float32, bfloat16 or float16")
        return t.get_device()

    @staticmethod
    def _dtype(dtype, default):
        if dtype is not None and dtype not in _TORCH:
            raise ValueError("dtype must be float32, bfloat16 or float16")
        return default if dtype is None else dtype

    def forward(self, weight, ids, dtype=None, out=None, stream=None):
        """Rows of shape ids.shape + (width,), of ``dtype`` (default weight's); ``out`` to write to."""
        if stream is not None:
            with _streaming(stream, weight):
                return self.forward(weight, ids, dtype, out)
        device, width = self._device(weight), self.width
        at, id_bytes, tokens = self._ids(ids, device)
        pw, sw = _rows("weight", weight, width, weight.dtype, device, self.vocab)
        fresh = out is None
        if fresh:
            out = torch.empty(*ids.shape, width, dtype=self._dtype(dtype, weight.dtype), device=weight.device)
            po, so = out.data_ptr(), width
        else:
            if self._device(out) != device or out.shape != (*ids.shape, width):
                raise ValueError("out must have the shape of ids and %d columns, on the device of weight" % width)
            po, so = _rows("out", out, width, self._dtype(dtype, out.dtype), device, tokens)
        block = _EMBEDDING.pack(tokens, self.vocab, width, _TORCH[weight.dtype], _TORCH[out.dtype], id_bytes, 0, self.scale,
                                at, pw, sw, po, so, 0, 0)
        rikfad._call_on(device, rikfad.lib().rikfad_embedding_forward, block, rikfad._raw_stream(device))
        if not fresh:
            rikfad._written(out)
        return out

    def backward(self, dout, ids, dtype=None, out=None, accumulate=False, stream=None):
        """The gradient of weight, [vocab, width] of ``dtype`` (default dout's), from that of the rows.  ``out`` to write
        to, or with ``accumulate`` to add to: rows without a token are then left alone."""
        if stream is not None:
            with _streaming(stream, dout):
                return self.backward(dout, ids, dtype, out, accumulate)
        device, width, vocab = self._device(dout), self.width, self.vocab
        at, id_bytes, tokens = self._ids(ids, device)
        if dout.shape != (*ids.shape, width):
            raise ValueError("dout must have the shape of ids and %d columns" % width)
        pd, sd = _rows("dout", dout, width, dout.dtype, device, tokens)
        fresh = out is None
        if fresh:
            if accumulate:
                raise ValueError("accumulate needs out")
            out = torch.empty(vocab, width, dtype=self._dtype(dtype, dout.dtype), device=dout.device)
            po, so = out.data_ptr(), width
        else:
            if self._device(out) != device:
                raise ValueError("out must be on the device of dout")
            po, so = _rows("out", out, width, self._dtype(dtype, out.dtype), device, vocab)
        lib = rikfad.lib()
        body = (tokens, vocab, width, _TORCH[out.dtype], _TORCH[dout.dtype], id_bytes, 1 if accumulate else 0, self.scale,
                at, po, so, pd, sd)
        pw = nbytes = 0
        if tokens:
            shape = body[:5]            # the size of the workspace goes by sizes and types alone
            nbytes = self._workspace.get(shape)
            if not nbytes:              # 0: this call is refused below, and later ones may not be
                nbytes = lib.rikfad_embedding_workspace(_EMBEDDING.pack(*body, 0, 0))
                if len(self._workspace) >= 64:
                    self._workspace.clear()
                self._workspace[shape] = nbytes
            work = torch.empty(nbytes, dtype=torch.uint8, device=dout.device)
            pw = work.data_ptr()
        rikfad._call_on(device, lib.rikfad_embedding_backward, _EMBEDDING.pack(*body, pw, nbytes), rikfad._raw_stream(device))
        if not fresh:
            rikfad._written(out)
        return out

    def __call__(self, weight, ids, dtype=None):
        """The rows inside autograd."""
        return _TokenEmbeddingFunction.apply(self, weight, ids, dtype)


class _TokenEmbeddingFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, op, weight, ids, dtype):
        ctx.op, ctx.dtype = op, weight.dtype
        ctx.save_for_backward(ids)
        return op.forward(weight, ids, dtype)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dout):
        ids, = ctx.saved_tensors
        return None, ctx.op.backward(dout.contiguous(), ids, ctx.dtype), None, None
