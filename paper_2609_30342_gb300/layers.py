"""Row operators of a transformer block: the residual sum with the norms around it, and rotary positions.

``ResidualNorm``   u = residual_scale x + branch_scale gate * post(z),  h = pre(u), and all gradients
``Rotary``         heads turned by their token's position, and back
``RotaryNorm``     heads normed, then turned, in one pass, and all gradients

Each has explicit calls on CUDA tensors (``forward``/``backward``, ``rotate``) and is callable inside autograd.
Argument checks and marshalling only: the work runs in the kernels behind ``rikfad_residual_norm_forward`` and
``_backward``, ``rikfad_rotary_apply`` and ``rikfad_rotary_norm_forward`` and ``_backward``, enqueued on the current stream
of the tensors' device (or ``stream``, to which what the call allocates then belongs; the inputs have to be ready on it).
"""
import ctypes
import math
import struct
from collections import namedtuple

import torch

from . import rikfad

_TORCH = {torch.float32: rikfad.F32, torch.bfloat16: rikfad.BF16, torch.float16: rikfad.F16}
_KINDS = {None: 0, "rms": 1, "layer": 2}
_F32 = torch.float32

# struct rikfad_residual_norm: sizes, types, scales, then (pointer, stride) pairs and pointers
_NORM = struct.Struct("=3q 4i 2i 4d 6q 4q 4q q 4q 6q 4q qQ")
# struct rikfad_rotary: sizes, types, pointers, magnitude, two sets of heads
_ROTARY = struct.Struct("=2q 4i qq2q 2i 2i d 18q")

# struct rikfad_rotary_norm: sizes, types, pointers, positions, magnitude and eps, two sets of heads, workspace
_ROTARY_NORM = struct.Struct("=2q 4i qq2q 2i 2i 2d 30q qQ")

_DENSE = torch.contiguous_format
_NO_BACKWARD = (0,) * 16
_NO_HEADS = (0,) * 9
_NO_NORM_HEADS = (0,) * 15

ResidualNormGrads = namedtuple("ResidualNormGrads", "x z gate post_weight post_bias pre_weight pre_bias")
RotaryNormGrads = namedtuple("RotaryNormGrads", "q k q_weight k_weight")


def _streaming(stream, t):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError("inputs must be CUDA tensors")
    return rikfad._streaming(stream, t.get_device())


def _rows(name, t, cols, dtype, device, rows):
    """A tensor as ``rows`` rows of ``cols`` contiguous elements: (pointer, row stride)."""
    if t.dtype is not dtype:
        raise ValueError("%s must be %s, not %s" % (name, dtype, t.dtype))
    if t.get_device() != device:
        raise ValueError("%s must be a CUDA tensor on the device of x" % name)
    if t.dim() != 2:
        t = _matrix(name, t, cols)
    n, c = t.shape
    if c != cols or n != rows:
        raise ValueError("%s is %d rows of %d columns, expected %d of %d" % (name, n, c, rows, cols))
    s0, s1 = t.stride()
    if n and s1 != 1 and cols > 1 or s0 < cols and n > 1:       # without elements strides say nothing
        raise ValueError("the rows of %s must be contiguous and not overlap" % name)
    return t.data_ptr(), s0 if n > 1 else cols


def _matrix(name, t, cols):
    if t.dim() == 0 or t.shape[-1] != cols:
        raise ValueError("%s must have %d columns" % (name, cols))
    try:
        return t.view(-1, cols)
    except RuntimeError:
        raise ValueError("the rows of %s must be evenly spaced" % name) from None


class ResidualNorm:
    """u = residual_scale x + branch_scale gate * post(z) and h = pre(u), over rows of ``cols`` elements.

    ``post``, ``pre``: None, "rms" or "layer"; weights and biases are arguments of the calls (absent: 1 and 0).
    x, u and their gradients are float32 or of z's type; weights and biases float32 or of z's type; a gate float32 or of
    z's type, with one row per row of z or one for every run of rows (its row count divides theirs)."""

    def __init__(self, cols, post=None, pre="rms", post_eps=1e-6, pre_eps=1e-6, residual_scale=1.0, branch_scale=1.0):
        if not 1 <= int(cols) <= 32768:
            raise ValueError("cols must be in [1, 32768]")
        if post not in _KINDS or pre not in _KINDS:
            raise ValueError("post and pre must be None, 'rms' or 'layer'")
        for v in (post_eps, pre_eps):
            if not (math.isfinite(v) and v >= 0):
                raise ValueError("eps must be finite and >= 0")
        for v in (residual_scale, branch_scale):
            if not math.isfinite(v):
                raise ValueError("scales must be finite")
        self.cols, self.post, self.pre = int(cols), post, pre
        self.post_eps, self.pre_eps = float(post_eps), float(pre_eps)
        self.residual_scale, self.branch_scale = float(residual_scale), float(branch_scale)
        self._kinds = (_KINDS[post], _KINDS[pre])
        self._scales = (self.post_eps, self.pre_eps, self.residual_scale, self.branch_scale)
        self._workspace = {}        # bytes by sizes, types and what is there

    def _vector(self, name, v, dtype, device):
        if v is None:
            return 0
        if v.dtype is not dtype or v.get_device() != device or v.dim() != 1 or v.shape[0] != self.cols or \
                not v.is_contiguous():
            raise ValueError("%s must be %d contiguous elements of %s on the device of x" % (name, self.cols, dtype))
        return v.data_ptr()

    def _inputs(self, x, z, gate, weights, dtype):
        """The head of the parameter block up to the weights, and (rows, type of z, device)."""
        cols = self.cols
        for t in (x, z, gate) + weights:
            if t is not None and not isinstance(t, torch.Tensor):
                raise ValueError("inputs must be tensors")
        device = x.get_device()
        if device < 0:
            raise ValueError("x must be a CUDA tensor")
        rt = x.dtype
        dt = z.dtype if z is not None else (rt if dtype is None else dtype)
        w2, b2, w1, b1 = weights
        first = w2 if w2 is not None else w1 if w1 is not None else b2 if b2 is not None else b1
        pt = _F32 if first is None else first.dtype
        gt = _F32 if gate is None else gate.dtype
        if dt not in _TORCH:
            raise ValueError("z must be float32, bfloat16 or float16")
        if (rt is not _F32 and rt is not dt) or (pt is not _F32 and pt is not dt) or (gt is not _F32 and gt is not dt):
            raise ValueError("x, weights, biases and gate must be float32 or %s" % dt)
        rows = x.shape[0] if x.dim() == 2 else _matrix("x", x, cols).shape[0]
        px, sx = _rows("x", x, cols, rt, device, rows)
        pz = sz = pg = sg = 0
        per = 1
        if z is not None:
            pz, sz = _rows("z", z, cols, dt, device, rows)
        elif gate is not None or self.post is not None:
            raise ValueError("a post norm or a gate needs z")
        if gate is not None:
            n = gate.shape[0] if gate.dim() == 2 else _matrix("gate", gate, cols).shape[0]
            if n == 0 and rows or n and rows % n:
                raise ValueError("the gate's rows must divide those of x")
            pg, sg = _rows("gate", gate, cols, gt, device, n)
            per = rows // n if n and rows else 1
        if self.post is None and (w2 is not None or b2 is not None):
            raise ValueError("post_weight and post_bias need a post norm")
        if self.pre is None and (w1 is not None or b1 is not None):
            raise ValueError("pre_weight and pre_bias need a pre norm")
        vector = self._vector
        head = (rows, cols, per, _TORCH[dt], _TORCH[rt], _TORCH[pt], _TORCH[gt], *self._kinds, *self._scales,
                px, sx, pz, sz, pg, sg, vector("post_weight", w2, pt, device), vector("post_bias", b2, pt, device),
                vector("pre_weight", w1, pt, device), vector("pre_bias", b1, pt, device))
        return head, rows, dt, device

    def forward(self, x, z=None, gate=None, post_weight=None, post_bias=None, pre_weight=None, pre_bias=None,
                need_stats=True, dtype=None, out=None, stream=None):
        """(u, h, stats).  ``stats`` (None without ``need_stats``) is what ``backward`` needs besides the inputs.
        Without z, u = residual_scale x and ``dtype`` gives h's type (default x's).  ``out``: (u, h) to write to; u may
        be x and h may be z; None for one that is not wanted."""
        weights = (post_weight, post_bias, pre_weight, pre_bias)
        if stream is not None:
            with _streaming(stream, x):
                return self.forward(x, z, gate, *weights, need_stats=need_stats, dtype=dtype, out=out)
        head, rows, dt, device = self._inputs(x, z, gate, weights, dtype)
        cols = self.cols
        if out is None:
            u = torch.empty_like(x, memory_format=torch.contiguous_format)
            h = torch.empty_like(x, dtype=dt, memory_format=torch.contiguous_format)
            pu, ph = u.data_ptr(), h.data_ptr()
            su = sh = cols
        else:
            u, h = out
            pu, su = (0, 0) if u is None else _rows("u", u, cols, x.dtype, device, rows)
            ph, sh = (0, 0) if h is None else _rows("h", h, cols, dt, device, rows)
        stats = torch.empty(rows, 4, dtype=_F32, device=x.device) if need_stats else None
        block = _NORM.pack(*head, pu, su, ph, sh, 0 if stats is None else stats.data_ptr(), *_NO_BACKWARD)
        rikfad._call_on(device, rikfad.lib().rikfad_residual_norm_forward, block, rikfad._raw_stream(device))
        return u, h, stats

    def backward(self, du, dh, x, z=None, gate=None, post_weight=None, post_bias=None, pre_weight=None, pre_bias=None,
                 stats=None, stream=None, dtype=None):
        """``ResidualNormGrads`` of the forward call's inputs (None where the input is None), from the gradients of u
        and h (either may be None).  Without z and dh, ``dtype`` is h's type as in the forward call (default x's)."""
        weights = (post_weight, post_bias, pre_weight, pre_bias)
        if stream is not None:
            with _streaming(stream, x):
                return self.backward(du, dh, x, z, gate, *weights, stats=stats, dtype=dtype)
        head, rows, dt, device = self._inputs(x, z, gate, weights, dtype if dtype is not None or dh is None else dh.dtype)
        cols = self.cols
        pdu, sdu = (0, 0) if du is None else _rows("du", du, cols, x.dtype, device, rows)
        pdh, sdh = (0, 0) if dh is None else _rows("dh", dh, cols, dt, device, rows)
        if stats is None or stats.dtype is not _F32 or stats.shape != (rows, 4) or not stats.is_contiguous() \
                or stats.get_device() != device:
            raise ValueError("stats must be what forward returned for these inputs")
        dense = torch.contiguous_format
        dx = torch.empty_like(x, memory_format=dense)
        dz = None if z is None else torch.empty_like(z, memory_format=dense)
        # a gate of no rows of x gets no gradient from them
        dgate = None if gate is None else (torch.empty_like if rows else torch.zeros_like)(gate, memory_format=dense)
        dw = [None if w is None else torch.empty_like(w) for w in weights]
        outputs = (dx.data_ptr(), cols, 0 if z is None else dz.data_ptr(), cols, 0 if gate is None else dgate.data_ptr(),
                   cols, *[0 if w is None else w.data_ptr() for w in dw])
        body = (*head, 0, 0, 0, 0, stats.data_ptr(), pdu, sdu, pdh, sdh, *outputs)
        lib = rikfad.lib()
        # the size of the workspace goes by sizes, types and what is there alone
        shape = (*head[:9], z is None, du is None, dh is None, *[w is None for w in dw])
        nbytes = self._workspace.get(shape)
        if nbytes is None:
            nbytes = lib.rikfad_residual_norm_workspace(_NORM.pack(*body, 0, 0))
            if len(self._workspace) >= 64:
                self._workspace.clear()
            self._workspace[shape] = nbytes
        pw = 0
        if nbytes:
            work = torch.empty(nbytes, dtype=torch.uint8, device=x.device)
            pw = work.data_ptr()
        rikfad._call_on(device, lib.rikfad_residual_norm_backward, _NORM.pack(*body, pw, nbytes),
                        rikfad._raw_stream(device))
        return ResidualNormGrads(dx, dz, dgate, *dw)

    def __call__(self, x, z=None, gate=None, post_weight=None, post_bias=None, pre_weight=None, pre_bias=None,
                 dtype=None):
        """(u, h) inside autograd."""
        return _ResidualNormFunction.apply(self, dtype, x, z, gate, post_weight, post_bias, pre_weight, pre_bias)


class _ResidualNormFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, op, dtype, x, *rest):
        u, h, stats = op.forward(x, *rest, dtype=dtype)
        ctx.op, ctx.dtype = op, h.dtype
        ctx.set_materialize_grads(False)
        ctx.save_for_backward(x, *rest, stats)
        return u, h

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, du, dh):
        x, *rest, stats = ctx.saved_tensors
        du, dh = (None if g is None else g.contiguous() for g in (du, dh))
        return (None, None, *ctx.op.backward(du, dh, x, *rest, stats=stats, dtype=ctx.dtype))


def rotary_frequencies(rotary_dim, base=10000.0, scaling=None):
    """(radians per position of every pair, magnitude of the rotated values), in double precision.

    Pair i turns by base^(-2 i / rotary_dim).  ``scaling``: None, or a dict with "kind" and "factor":
      linear  every frequency divided by the factor
      base    the base times factor^(rotary_dim / (rotary_dim - 2)): the fastest pair keeps its frequency, the slowest
              one's is divided by the factor
      ramp    pairs that turn more than "fast" (32) times within "original_context" keep their frequency, those that turn
              less than "slow" (1) times are divided by the factor, with a straight ramp between; the magnitude is
              0.1 ln(factor) + 1"""
    factor = 1.0
    kind = None
    if scaling is not None:
        kind, factor = scaling.get("kind"), float(scaling.get("factor", 1.0))
        if kind not in ("linear", "base", "ramp"):
            raise ValueError("scaling kind must be 'linear', 'base' or 'ramp'")
        if not (math.isfinite(factor) and factor >= 1.0):
            raise ValueError("the scaling factor must be >= 1")
    if not (math.isfinite(base) and base > 0):
        raise ValueError("base must be > 0")
    if rotary_dim % 2 or rotary_dim < 0:
        raise ValueError("rotary_dim must be even and >= 0")
    if kind == "base" and rotary_dim > 2:
        base = base * factor ** (rotary_dim / (rotary_dim - 2))
    f = [base ** (-2.0 * i / rotary_dim) for i in range(rotary_dim // 2)]
    if kind == "linear":
        return [v / factor for v in f], 1.0
    if kind != "ramp":
        return f, 1.0
    original, fast, slow = scaling.get("original_context"), scaling.get("fast", 32.0), scaling.get("slow", 1.0)
    if not original or original <= 0 or not fast > slow:
        raise ValueError("ramp scaling needs original_context > 0 and fast > slow")
    keep = [min(1.0, max(0.0, (original * v / (2.0 * math.pi) - slow) / (fast - slow))) for v in f]
    return [v * (k + (1.0 - k) / factor) for v, k in zip(f, keep)], 0.1 * math.log(factor) + 1.0


class Rotary:
    """Rotary positions of heads of ``head_dim`` elements, the first ``rotary_dim`` (all by default) of which turn, as
    pairs (i, i + rotary_dim / 2) ("half") or (2 i, 2 i + 1) ("interleaved").  ``scaling`` as for
    ``rotary_frequencies``, or ``frequencies`` (radians per position) with ``magnitude``."""

    def __init__(self, head_dim, rotary_dim=None, base=10000.0, layout="half", scaling=None, frequencies=None,
                 magnitude=None, device="cuda"):
        self.head_dim = int(head_dim)
        self.rotary_dim = self.head_dim if rotary_dim is None else int(rotary_dim)
        if not 1 <= self.head_dim <= 4096:
            raise ValueError("head_dim must be in [1, 4096]")
        if self.rotary_dim % 2 or not 0 <= self.rotary_dim <= self.head_dim:
            raise ValueError("rotary_dim must be even and in [0, head_dim]")
        if layout not in ("half", "interleaved"):
            raise ValueError("layout must be 'half' or 'interleaved'")
        self.layout = layout
        if frequencies is None:
            frequencies, m = rotary_frequencies(self.rotary_dim, float(base), scaling)
        else:
            frequencies, m = [float(v) for v in frequencies], 1.0
        self.magnitude = m if magnitude is None else float(magnitude)
        n = self.rotary_dim // 2
        if len(frequencies) != n:
            raise ValueError("need rotary_dim / 2 frequencies")
        turns = (ctypes.c_uint64 * max(n, 1))()
        rikfad._check(rikfad.lib().rikfad_rotary_turns((ctypes.c_double * max(n, 1))(*frequencies), n, turns))
        self.frequencies = frequencies
        signed = [v - (1 << 64) if v >= 1 << 63 else v for v in turns[:n]]
        self.turns = torch.tensor(signed, dtype=torch.int64).to(device)
        self._layout = 0 if layout == "half" else 1

    @property
    def turns(self):
        """The frequencies as the kernel takes them: turns per position in units of 2^-64, int64 bits."""
        return self._turns

    @turns.setter
    def turns(self, turns):
        if turns.dtype is not torch.int64 or turns.shape != (self.rotary_dim // 2,) or not turns.is_contiguous():
            raise ValueError("turns must be rotary_dim / 2 contiguous int64 values")
        self._turns = turns

    def _heads(self, name, t, lead, dtype, device):
        """(pointer, heads, batch, token and head strides) of a [tokens, heads, head_dim] or
        [batch, tokens, heads, head_dim] tensor."""
        if t.dtype is not dtype:
            raise ValueError("%s must be %s, not %s" % (name, dtype, t.dtype))
        if t.get_device() != device:
            raise ValueError("%s must be a CUDA tensor on the device of q" % name)
        shape, s = t.shape, t.stride()
        if shape[:-2] != lead or shape[-1] != self.head_dim:
            raise ValueError("%s must be [tokens, heads, %d] or [batch, tokens, heads, %d], with the tokens of q"
                             % (name, self.head_dim, self.head_dim))
        if s[-1] != 1 and self.head_dim > 1 and t.numel():      # without elements strides say nothing
            raise ValueError("the heads of %s must be contiguous" % name)
        if len(s) == 3:
            return t.data_ptr(), shape[1], 0, s[0], s[1]
        return t.data_ptr(), shape[2], s[0], s[1], s[2]

    def _lead(self, q):
        """(device, type, leading sizes, batch, tokens) of q."""
        device, dtype = q.get_device(), q.dtype
        if device < 0 or device != self._turns.get_device():
            raise ValueError("q must be on %s, the device of the frequencies" % self._turns.device)
        if dtype not in _TORCH:
            raise ValueError("q must be float32, bfloat16 or float16")
        lead = q.shape[:-2]
        if len(lead) == 1:
            return device, dtype, lead, 1, lead[0]
        if len(lead) == 2:
            return device, dtype, lead, *lead
        raise ValueError("q must be [tokens, heads, head_dim] or [batch, tokens, heads, head_dim]")

    @staticmethod
    def _positions(positions, lead, tokens, device):
        """(pointer, batch stride, bytes of a position)."""
        if positions is None:
            return 0, 0, 8
        width = 4 if positions.dtype is torch.int32 else 8
        if positions.get_device() != device or width == 8 and positions.dtype is not torch.int64:
            raise ValueError("positions must be an int32 or int64 CUDA tensor on the device of q")
        per_batch = 0
        if len(lead) == 2 and positions.shape == lead:
            per_batch = positions.stride(0)
        elif positions.shape != (tokens,):
            raise ValueError("positions must be [tokens] or [batch, tokens]")
        if tokens > 1 and positions.stride(-1) != 1:
            raise ValueError("positions must be contiguous along the tokens")
        return positions.data_ptr(), per_batch, width

    def rotate(self, q, k=None, positions=None, start=0, inverse=False, out=None, stream=None):
        """(q', k') of queries and keys [tokens, heads, head_dim] or [batch, tokens, heads, head_dim] (k' None without
        k).  ``positions``: int32 or int64 CUDA tensor [tokens] or [batch, tokens]; default ``start`` + 0, 1, ...
        ``inverse`` turns back: the gradient of the rotation.  ``out``: (q', k') to write to; q and k themselves
        rotate in place."""
        if stream is not None:
            with _streaming(stream, q):
                return self.rotate(q, k, positions, start, inverse, out)
        for t in (q, k, positions):
            if t is not None and not isinstance(t, torch.Tensor):
                raise ValueError("inputs must be tensors")
        device, dtype, lead, batch, tokens = self._lead(q)
        at, per_batch, width = self._positions(positions, lead, tokens, device)
        if out is None:
            dense = torch.contiguous_format
            out = (torch.empty_like(q, memory_format=dense),
                   None if k is None else torch.empty_like(k, memory_format=dense))
        lists = []
        for name, src, dst in (("q", q, out[0]), ("k", k, out[1])):
            if src is None:
                lists += _NO_HEADS
                continue
            ps, heads, *from_ = self._heads(name, src, lead, dtype, device)
            pd, to_heads, *to = self._heads(name, dst, lead, dtype, device)
            if to_heads != heads:
                raise ValueError("the output of %s must have its shape" % name)
            lists += (ps, pd, heads, *from_, *to)
        block = _ROTARY.pack(batch, tokens, self.head_dim, self.rotary_dim, self._layout, _TORCH[dtype],
                             self._turns.data_ptr(), at, per_batch, start, width, 1 if inverse else 0,
                             1 if k is None else 2, 0,
                             self.magnitude, *lists)
        rikfad._call_on(device, rikfad.lib().rikfad_rotary_apply, block, rikfad._raw_stream(device))
        return out[0], (None if k is None else out[1])

    def __call__(self, q, k, positions=None, start=0):
        """(q', k') inside autograd."""
        return _RotaryFunction.apply(self, q, k, positions, start)


class _RotaryFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, op, q, k, positions, start):
        ctx.op, ctx.start = op, start
        ctx.set_materialize_grads(False)
        ctx.save_for_backward(*([] if positions is None else [positions]))
        return op.rotate(q, k, positions=positions, start=start)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dq, dk):
        positions = ctx.saved_tensors[0] if ctx.saved_tensors else None
        if dq is None:
            dk, _ = ctx.op.rotate(dk.contiguous(), positions=positions, start=ctx.start, inverse=True)
        else:
            dq, dk = ctx.op.rotate(dq.contiguous(), None if dk is None else dk.contiguous(), positions=positions,
                                   start=ctx.start, inverse=True)
        return None, dq, dk, None, None


class RotaryNorm(Rotary):
    """Heads divided by their root mean square (of all ``head_dim`` elements, with ``eps``), times a weight per element,
    then turned as ``Rotary`` turns them: out = R(position) (x / sqrt(mean(x^2) + eps) * weight).

    Queries and keys have weights of their own, float32 or of the heads' type, arguments of the calls (absent: 1)."""

    def __init__(self, head_dim, rotary_dim=None, base=10000.0, layout="half", scaling=None, frequencies=None,
                 magnitude=None, eps=1e-6, device="cuda"):
        if not 1 <= int(head_dim) <= 512:
            raise ValueError("head_dim must be in [1, 512]")
        if not (math.isfinite(eps) and eps >= 0):
            raise ValueError("eps must be finite and >= 0")
        super().__init__(head_dim, rotary_dim, base, layout, scaling, frequencies, magnitude, device)
        self.eps = float(eps)
        self._workspace = 0         # bytes, when a call has asked for them

    def _dense(self, tokens, heads):
        """Batch, token and head strides of a contiguous tensor."""
        return tokens * heads * self.head_dim, heads * self.head_dim, self.head_dim

    def _weights(self, weights, dtype, device):
        """The weights' type, and their addresses."""
        given = next((w for w in weights if w is not None), None)
        if given is None:
            return _F32, (0, 0)
        pt = given.dtype
        if pt is not _F32 and pt is not dtype:
            raise ValueError("weights must be float32 or %s" % dtype)
        for w in weights:
            if w is not None and (w.dtype is not pt or w.get_device() != device or w.shape != (self.head_dim,)
                                  or not w.is_contiguous()):
                raise ValueError("weights must be %d contiguous elements of one type on the device of q" % self.head_dim)
        return pt, tuple(0 if w is None else w.data_ptr() for w in weights)

    def _block(self, first, positions, start, pt, lists, work=(0, 0)):
        device, dtype, lead, batch, tokens = first
        at, per_batch, width = self._positions(positions, lead, tokens, device)
        return _ROTARY_NORM.pack(batch, tokens, self.head_dim, self.rotary_dim, self._layout, _TORCH[dtype],
                                 self._turns.data_ptr(), at, per_batch, start, width, _TORCH[pt], len(lists) // 15, 0,
                                 self.magnitude, self.eps, *lists, *(_NO_NORM_HEADS if len(lists) == 15 else ()), *work)

    def forward(self, q, k=None, q_weight=None, k_weight=None, positions=None, start=0, out=None, stream=None):
        """(q', k') of queries and keys [tokens, heads, head_dim] or [batch, tokens, heads, head_dim] (k' None without k),
        with positions as for ``rotate``.  ``out``: (q', k') to write to; q and k themselves for in place.  Tensors given as
        ``out`` count as changed in autograd: a graph that holds them refuses its backward pass."""
        if stream is not None:
            with _streaming(stream, q):
                return self.forward(q, k, q_weight, k_weight, positions, start, out)
        for t in (q, k, q_weight, k_weight, positions):
            if t is not None and not isinstance(t, torch.Tensor):
                raise ValueError("inputs must be tensors")
        first = device, dtype, lead, batch, tokens = self._lead(q)
        if k is None and k_weight is not None:
            raise ValueError("k_weight needs k")
        pt, weights = self._weights((q_weight, k_weight), dtype, device)
        lists, fresh = [], out is None
        if fresh:
            out = (torch.empty_like(q, memory_format=_DENSE), None if k is None else torch.empty_like(k, memory_format=_DENSE))
        for name, src, dst, weight in (("q", q, out[0], weights[0]), ("k", k, out[1], weights[1])):
            if src is None:
                continue
            px, heads, *from_ = self._heads(name, src, lead, dtype, device)
            if fresh:
                po, to = dst.data_ptr(), self._dense(tokens, heads)
            else:
                po, to_heads, *to = self._heads(name, dst, lead, dtype, device)
                if to_heads != heads:
                    raise ValueError("the output of %s must have its shape" % name)
            lists += (px, 0, weight, po, 0, heads, *from_, *to, 0, 0, 0)
        rikfad._call_on(device, rikfad.lib().rikfad_rotary_norm_forward, self._block(first, positions, start, pt, lists),
                        rikfad._raw_stream(device))
        if not fresh:
            rikfad._written(out[0], None if k is None else out[1])
        return out[0], (None if k is None else out[1])

    def backward(self, dq, dk, q, k=None, q_weight=None, k_weight=None, positions=None, start=0, stream=None):
        """``RotaryNormGrads`` of the forward call's inputs (None where the input is None), from the gradients of its
        outputs.  Either of them may be None, with no gradients of that input and its weight then."""
        if stream is not None:
            with _streaming(stream, q):
                return self.backward(dq, dk, q, k, q_weight, k_weight, positions, start)
        for t in (dq, dk, q, k, q_weight, k_weight, positions):
            if t is not None and not isinstance(t, torch.Tensor):
                raise ValueError("inputs must be tensors")
        first = device, dtype, lead, batch, tokens = self._lead(q)
        if k is None and (dk is not None or k_weight is not None):
            raise ValueError("dk and k_weight need k")
        pt, weights = self._weights((q_weight, k_weight), dtype, device)
        lists, grads = [], []
        for name, x, d, weight, pw in (("q", q, dq, q_weight, weights[0]), ("k", k, dk, k_weight, weights[1])):
            if d is None:
                grads += (None, None)
                continue
            px, heads, *from_ = self._heads(name, x, lead, dtype, device)
            pd, d_heads, *d_from = self._heads("d" + name, d, lead, dtype, device)
            if d_heads != heads:
                raise ValueError("d%s must have the shape of %s" % (name, name))
            dx, dw = torch.empty_like(x, memory_format=_DENSE), None if weight is None else torch.empty_like(weight)
            grads += (dx, dw)
            lists += (px, pd, pw, dx.data_ptr(), 0 if dw is None else dw.data_ptr(), heads, *from_,
                      *self._dense(tokens, heads), *d_from)
        if lists:
            lib = rikfad.lib()
            work = (0, 0)
            if grads[1] is not None or grads[-1] is not None:
                nbytes = self._workspace
                if not nbytes:              # it goes by head_dim alone; 0: this call's sizes are refused below
                    nbytes = self._workspace = lib.rikfad_rotary_norm_workspace(
                        self._block(first, positions, start, pt, lists))
                buffer = torch.empty(nbytes, dtype=torch.uint8, device=q.device)
                work = (buffer.data_ptr(), nbytes)
            rikfad._call_on(device, lib.rikfad_rotary_norm_backward, self._block(first, positions, start, pt, lists, work),
                            rikfad._raw_stream(device))
        return RotaryNormGrads(grads[0], grads[2], grads[1], grads[3])

    def __call__(self, q, k=None, q_weight=None, k_weight=None, positions=None, start=0):
        """(q', k') inside autograd."""
        return _RotaryNormFunction.apply(self, q, k, q_weight, k_weight, positions, start)


class _RotaryNormFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, op, q, k, q_weight, k_weight, positions, start):
        ctx.op, ctx.start = op, start
        ctx.set_materialize_grads(False)
        ctx.save_for_backward(q, k, q_weight, k_weight, positions)
        return op.forward(q, k, q_weight, k_weight, positions, start)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dq, dk):
        dq, dk = (None if g is None else g.contiguous() for g in (dq, dk))
        q, k, q_weight, k_weight, positions = ctx.saved_tensors
        g = ctx.op.backward(dq, dk, q, k, q_weight, k_weight, positions, ctx.start)
        return None, g.q, g.k, g.q_weight, g.k_weight, None, None
