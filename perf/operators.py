"""Performance cases of the operators of a training step that stand between a model's matrix products and the
optimiser: the rows' norms, gates and residual sums, the rotation of heads by position, and the global norm of the
gradients with clipping.

``listed()`` are the cases that are timed, ``draw(rng)`` gives more of the same ranges, ``prepare(case, seed)`` makes
what a program has in hand before the call, ``run(state)`` is one pass, ``work(case)`` what that pass cannot do
without, and ``exact(case, seed)`` the results in 64 bits.  With ``own`` false a pass is computed in elementary torch
operations in 32 bits, with ``own`` true by the package's operators.

The operators ("op" of a case):

  clip    the 2-norm of every gradient of a list and of all of them, and the gradients scaled to a largest norm, out of
          place (a training loop keeps its accumulated gradients and hands the optimiser the clipped ones, in the type
          that its handle takes); with "clip" false only the norms
              total = sqrt(sum g^2),  out = g min(1, max_norm / total)
  norm    the residual sum of a transformer block and the norms around it
              u = residual_scale x + branch_scale gate post(z),   h = pre(u)
          post and pre are RMS or layer norms with weight and bias, or absent; a gate row is shared by ``gate_rows``
          consecutive rows.  "train" adds the gradients of everything from du and dh.
  rotary  heads rotated by their token's position; pair i of a head turns by position x frequency i.  "train" adds the
          gradients (the inverse rotation).
"""
import math

import torch

own = False
DEVICE = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ALIGN = 64          # elements: every gradient of a flat buffer starts on 256 bytes (128 for 16-bit types)


# ------------------------------------------------------------------ cases

def _clip(name, **kw):
    return dict(dict(name=name, op="clip", clip=True, grad_std=1e-3), **kw)


def _norm(name, **kw):
    return dict(dict(name=name, op="norm", train=True, gate="none", gate_rows=1, residual="same",
                     params="f32", residual_scale=1.0, branch_scale=1.0, eps=1e-6), **kw)


def _rotary(name, **kw):
    return dict(dict(name=name, op="rotary", train=False, fused=False, base=10000.0, scaling="none", factor=1.0,
                     original=1024), **kw)


def listed():
    return [
        # The smallest list: one layer's matrix and bias, fp32 gradients; latency and launches.
        _clip("clip-layer-f32", params="matrix", rows=256, cols=512, grad="f32", out="f32", max_norm=0.2),
        # A small model's list (100 tensors, 30M parameters) in mixed precision; it fits the L2 cache.
        _clip("clip-nano-bf16", params="gpt2", layers=6, width=384, vocab=50304, ctx=256, grad="bf16", out="bf16",
              max_norm=1.0),
        # The benchmark's list (196 tensors, 124M parameters): fp32 gradients summed over micro-batches, handed to the
        # optimiser in bf16.
        _clip("clip-gpt2s-f32-bf16", params="gpt2", layers=12, width=768, vocab=50257, ctx=1024, grad="f32",
              out="bf16", max_norm=1.0),
        # The largest: 1557.6M parameters.
        _clip("clip-gpt2xl-bf16", params="gpt2", layers=48, width=1600, vocab=50257, ctx=1024, grad="bf16", out="bf16",
              max_norm=1.0),
        # A token being generated: one row through the sandwich norms of a block; latency.
        _norm("norm-token-768", train=False, rows=1, cols=768, dtype="bf16", post="rms", pre="rms"),
        # A training step's batch (16 sequences of 1024) at the benchmark's width: residual sum and layer norm, fp32
        # residual stream and parameters.
        _norm("norm-train-768", rows=16384, cols=768, dtype="bf16", residual="f32", post="none", pre="layer"),
        # The widest of the benchmark's models, norms before and after, a gate for every row, scaled branch.
        _norm("norm-train-1600-gated", rows=8192, cols=1600, dtype="bf16", post="rms", pre="rms", gate="rows",
              branch_scale=0.5),
        # An odd width, half precision, a learned gate per sequence (6 of 683), layer norms on both sides.
        _norm("norm-train-odd", rows=4098, cols=1001, dtype="f16", residual="f32", post="layer", pre="layer",
              gate="shared", gate_rows=683, residual_scale=1.2),
        # The largest: a long batch at width 4096.
        _norm("norm-train-4096", rows=32768, cols=4096, dtype="bf16", post="rms", pre="rms", gate="rows"),
        # Tokens being generated for 8 requests, late in long contexts; latency.
        _rotary("rotary-tokens", tokens=8, q_heads=12, k_heads=12, head_dim=64, rotary_dim=64, dtype="bf16",
                layout="half", positions="random"),
        # A training step's batch of packed sequences, queries and keys inside the fused projection's output, with
        # the gradients.
        _rotary("rotary-train-768", train=True, tokens=16384, q_heads=12, k_heads=12, head_dim=64, rotary_dim=64,
                dtype="bf16", layout="half", positions="packed", fused=True),
        # The largest: a long prompt, grouped heads, half of each head rotated, frequencies stretched for the context.
        _rotary("rotary-long", tokens=131072, q_heads=32, k_heads=8, head_dim=128, rotary_dim=64, dtype="bf16",
                layout="interleaved", positions="prompt", scaling="ramp", factor=8.0, original=16384),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Half of them multiples of 64, the others any number."""
    n = _log_int(rng, lo, hi)
    return max(64, n // 64 * 64) if rng.random() < 0.5 else n


def _draw_clip(rng):
    if rng.random() < 0.5:
        cols = _width(rng, 24, 16384)
        p = dict(params="matrix", cols=cols, rows=_log_int(rng, 16, max(17, min(65536, 200_000_000 // cols))))
    else:
        p = dict(params="gpt2", layers=rng.randint(1, 24), width=32 * rng.randint(2, 40),
                 vocab=_log_int(rng, 500, 51000), ctx=rng.choice((128, 256, 512, 1024)))
    grad = rng.choice(("bf16", "f32", "f32", "f16"))
    out = "bf16" if grad == "f32" and rng.random() < 0.5 else grad
    std = 1e-3 if grad != "f16" else 1e-2
    # from gradients that are let through to a strong cut
    n = sum(_numel(s) for s in _shapes(p))
    max_norm = float("%.4g" % (std * math.sqrt(n) * math.exp(rng.uniform(math.log(0.05), math.log(2.0)))))
    return dict(op="clip", clip=rng.random() < 0.8, grad=grad, out=out, grad_std=std, max_norm=max_norm, **p)


def _draw_norm(rng):
    cols = _width(rng, 48, 8192)
    gate = rng.choice(("none", "rows", "shared"))
    rows = _log_int(rng, 1, max(2, min(32768, 100_000_000 // cols)))
    gate_rows = 1
    if gate == "shared":
        gate_rows = _log_int(rng, 1, rows)
        rows = max(1, rows // gate_rows) * gate_rows
    return dict(op="norm", train=rng.random() < 0.75, rows=rows, cols=cols, dtype=rng.choice(("bf16", "bf16", "f16", "f32")),
                residual=rng.choice(("same", "f32")), params=rng.choice(("f32", "f32", "same")),
                post=rng.choice(("none", "rms", "layer")), pre=rng.choice(("rms", "layer")),
                gate=gate, gate_rows=gate_rows, residual_scale=rng.choice((1.0, 1.0, 1.2)),
                branch_scale=rng.choice((1.0, 0.5)), eps=rng.choice((1e-5, 1e-6)))


def _draw_rotary(rng):
    head_dim = rng.choice((32, 64, 64, 80, 96, 128, 128, 256, 2 * rng.randint(9, 100)))
    rotary_dim = head_dim if rng.random() < 0.5 else 2 * rng.randint(2, head_dim // 2)
    k_heads = _log_int(rng, 1, 16)
    q_heads = k_heads * rng.choice((1, 1, 2, 4, 8))
    tokens = _log_int(rng, 1, max(2, min(131072, 300_000_000 // ((q_heads + k_heads) * head_dim))))
    scaling = rng.choice(("none", "none", "linear", "base", "ramp"))
    return dict(op="rotary", train=rng.random() < 0.5, tokens=tokens, q_heads=q_heads, k_heads=k_heads, head_dim=head_dim,
                rotary_dim=rotary_dim, dtype=rng.choice(("bf16", "bf16", "f16", "f32")),
                layout=rng.choice(("half", "interleaved")), positions=rng.choice(("prompt", "packed", "random")),
                fused=rng.random() < 0.5, base=rng.choice((10000.0, 500000.0)), scaling=scaling,
                factor=1.0 if scaling == "none" else rng.choice((2.0, 8.0, 32.0)), original=rng.choice((1024, 8192)))


def draw(rng):
    return rng.choice((_draw_clip, _draw_norm, _draw_rotary))(rng)


# ----------------------------------------------------------------- inputs

def _numel(shape):
    return math.prod(shape)


def _shapes(case):
    """A matrix and a vector (a layer and its bias), or the tensors of a GPT-2-shaped model (separate q, k, v)."""
    if case["params"] == "matrix":
        return [(case["rows"], case["cols"]), (case["cols"],)]
    d = case["width"]
    out = [(case["vocab"], d), (case["ctx"], d)]
    for _ in range(case["layers"]):
        out += [(d,), (d,)] + [(d, d), (d,)] * 4 + [(d,), (d,), (4 * d, d), (4 * d,), (d, 4 * d), (d,)]
    return out + [(d,), (d,)]


def _views(flat, shapes):
    out, at = [], 0
    for s in shapes:
        n = _numel(s)
        out.append(flat[at:at + n].view(s))
        at += -(-n // ALIGN) * ALIGN
    return out


def _flat_size(shapes):
    return sum(-(-_numel(s) // ALIGN) * ALIGN for s in shapes)


class _State:
    """What a program keeps between passes."""


def _gen(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _clip_inputs(case, seed):
    shapes, gen = _shapes(case), _gen(seed)
    flat = torch.empty(_flat_size(shapes), dtype=DTYPES[case["grad"]], device=DEVICE)
    step = 1 << 26
    for at in range(0, flat.numel(), step):
        part = flat[at:at + step]
        part.copy_(torch.randn(part.numel(), generator=gen, device=DEVICE).mul_(case["grad_std"]))
    return shapes, flat


def _norm_inputs(case, seed):
    """A residual stream with a few strong channels, a branch's output of smaller size, gates in (0, 1) for rows and
    about zero when shared, weights about one."""
    gen, rows, cols = _gen(seed), case["rows"], case["cols"]
    dt = DTYPES[case["dtype"]]
    rt = torch.float32 if case["residual"] == "f32" else dt
    pt = torch.float32 if case["params"] == "f32" else dt

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=DEVICE)

    t = {}
    channel = 1.0 + 4.0 * (torch.rand(cols, generator=gen, device=DEVICE) < 0.02)
    t["x"] = ((normal(rows, cols) + 0.2 * normal(cols)) * channel).to(rt)
    t["z"] = (0.6 * normal(rows, cols) + 0.1 * normal(cols)).to(dt)
    if case["gate"] == "rows":
        t["gate"] = torch.rand(rows, cols, generator=gen, device=DEVICE).to(dt)
    elif case["gate"] == "shared":
        t["gate"] = (0.5 * normal(rows // case["gate_rows"], cols)).to(pt)
    for side in ("post", "pre"):
        if case[side] != "none":
            t[side + "_weight"] = (1.0 + 0.1 * normal(cols)).to(pt)
        if case[side] == "layer":
            t[side + "_bias"] = (0.1 * normal(cols)).to(pt)
    if case["train"]:
        t["du"] = (0.05 * normal(rows, cols)).to(rt)
        t["dh"] = (0.05 * normal(rows, cols)).to(dt)
    return t


def _rotary_inputs(case, seed):
    gen, tokens, d = _gen(seed), case["tokens"], case["head_dim"]
    dt, hq, hk = DTYPES[case["dtype"]], case["q_heads"], case["k_heads"]

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=DEVICE).to(dt)

    t = {}
    if case["fused"]:               # queries, keys and values side by side, as a projection leaves them
        qkv = normal(tokens, (hq + 2 * hk) * d)
        t["q"] = qkv[:, :hq * d].unflatten(1, (hq, d))
        t["k"] = qkv[:, hq * d:(hq + hk) * d].unflatten(1, (hk, d))
    else:
        t["q"], t["k"] = normal(tokens, hq, d), normal(tokens, hk, d)
    if case["positions"] == "prompt":
        t["positions"] = torch.arange(tokens, device=DEVICE)
    elif case["positions"] == "packed":     # sequences of different lengths, one after the other
        start = torch.rand(tokens, generator=gen, device=DEVICE) < 1.0 / min(700, tokens)
        at = torch.arange(tokens, device=DEVICE)
        t["positions"] = at - torch.cummax(torch.where(start, at, torch.zeros_like(at)), 0).values
    else:                                   # requests at any point of contexts of up to a million tokens
        t["positions"] = torch.randint(0, 1 << 20, (tokens,), generator=gen, device=DEVICE)
    if case["train"]:
        t["dq"], t["dk"] = normal(tokens, hq, d), normal(tokens, hk, d)
    return t


def _frequencies(case):
    """Radians per position of every pair, and the factor on the rotated values.

    linear: every frequency divided by the factor.  base: the base stretched so that the slowest pair slows by the
    factor.  ramp: pairs that turn more than 32 times within the original context keep their frequency, those that turn
    less than once are divided by the factor, with a straight ramp between; the values grow by 0.1 ln(factor) + 1."""
    rot, base, factor = case["rotary_dim"], case["base"], case["factor"]
    if case["scaling"] == "base" and rot > 2:
        base *= factor ** (rot / (rot - 2))
    f = [base ** (-2.0 * i / rot) for i in range(rot // 2)]
    if case["scaling"] == "linear":
        f = [v / factor for v in f]
    if case["scaling"] != "ramp":
        return f, 1.0
    keep = [min(1.0, max(0.0, (case["original"] * v / (2 * math.pi) - 1.0) / 31.0)) for v in f]
    return [v * (k + (1.0 - k) / factor) for v, k in zip(f, keep)], 0.1 * math.log(factor) + 1.0


# ------------------------------------------------------------ prepare, run

def prepare(case, seed):
    s = _State()
    s.case = case
    if case["op"] == "clip":
        s.shapes, s.flat = _clip_inputs(case, seed)
        s.grads = _views(s.flat, s.shapes)
        if case["clip"]:
            s.out = torch.zeros(s.flat.numel(), dtype=DTYPES[case["out"]], device=DEVICE)
            s.outs = _views(s.out, s.shapes)
        if own:
            from paper_2609_30342_gb300 import gradients
            s.clipper = gradients.GradientClipper([_numel(v) for v in s.shapes], case["grad"],
                                                  case["out"] if case["clip"] else None)
            s.ptrs = s.clipper.pack(s.grads, s.outs if case["clip"] else None)
    elif case["op"] == "norm":
        s.t = _norm_inputs(case, seed)
        if own:
            from paper_2609_30342_gb300 import layers
            s.op = layers.ResidualNorm(case["cols"], post=None if case["post"] == "none" else case["post"],
                                       pre=case["pre"], post_eps=case["eps"], pre_eps=case["eps"],
                                       residual_scale=case["residual_scale"], branch_scale=case["branch_scale"])
    else:
        s.t = _rotary_inputs(case, seed)
        freq, s.magnitude = _frequencies(case)
        if own:
            from paper_2609_30342_gb300 import layers
            scaling = None if case["scaling"] == "none" else dict(kind=case["scaling"], factor=case["factor"],
                                                                  original_context=case["original"])
            s.op = layers.Rotary(case["head_dim"], case["rotary_dim"], base=case["base"], layout=case["layout"],
                                 scaling=scaling, device=DEVICE)
        else:
            s.freq = torch.tensor(freq, dtype=torch.float64, device=DEVICE)
    return s


def _run_clip(s):
    case = s.case
    if own:
        if case["clip"]:
            total, norms = s.clipper.clip(case["max_norm"], ptrs=s.ptrs)
        else:
            total, norms = s.clipper.norm(ptrs=s.ptrs)
    else:
        norms = torch.stack([(g.float() * g.float()).sum().sqrt() for g in s.grads])
        total = (norms * norms).sum().sqrt()
        if case["clip"]:
            scale = torch.clamp(case["max_norm"] / total, max=1.0)
            for g, o in zip(s.grads, s.outs):
                o.copy_(g.float() * scale)
    return {"total": total, "norms": norms, "out": s.out} if case["clip"] else {"total": total, "norms": norms}


def _plain_norm(v, kind, eps):
    """The normed rows before weight and bias, and 1 / (root mean square or standard deviation)."""
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    r = torch.rsqrt((v * v).mean(1, keepdim=True) + eps)
    return v * r, r


def _plain_norm_grad(dy, weight, y, r, kind):
    """The gradient of the norm's input from its output's."""
    g = dy * weight
    dv = g - y * (g * y).mean(1, keepdim=True)
    if kind == "layer":
        dv = dv - g.mean(1, keepdim=True)
    return dv * r


def _run_norm(s):
    case, t = s.case, s.t
    weights = {k: t.get(k) for k in ("gate", "post_weight", "post_bias", "pre_weight", "pre_bias")}
    if own:
        u, h, stats = s.op.forward(t["x"], t["z"], need_stats=case["train"], **weights)
        if not case["train"]:
            return {"u": u, "h": h}
        g = s.op.backward(t["du"], t["dh"], t["x"], t["z"], stats=stats, **weights)
        out = {"u": u, "h": h, "dx": g.x, "dz": g.z}
        out.update({"d" + k: getattr(g, k) for k, v in weights.items() if v is not None})
        return out
    rt, dt = t["x"].dtype, t["z"].dtype
    rows, cols, per = case["rows"], case["cols"], case["gate_rows"]
    w = {k: None if v is None else v.float() for k, v in weights.items()}
    x, n = t["x"].float(), t["z"].float()
    if case["post"] != "none":
        y2, r2 = _plain_norm(n, case["post"], case["eps"])
        n = y2 * w["post_weight"]
        if w["post_bias"] is not None:
            n = n + w["post_bias"]
    gate = None if w["gate"] is None else w["gate"].repeat_interleave(per, 0)
    a, b = case["residual_scale"], case["branch_scale"]
    u = a * x + b * (n if gate is None else gate * n)
    y1, r1 = _plain_norm(u, case["pre"], case["eps"])
    h = y1 * w["pre_weight"]
    if w["pre_bias"] is not None:
        h = h + w["pre_bias"]
    out = {"u": u.to(rt), "h": h.to(dt)}
    if not case["train"]:
        return out
    dh = t["dh"].float()
    du = t["du"].float() + _plain_norm_grad(dh, w["pre_weight"], y1, r1, case["pre"])
    out["dx"] = (a * du).to(rt)
    dn = b * du if gate is None else b * gate * du
    grads = {"pre_weight": (dh * y1).sum(0), "pre_bias": dh.sum(0)}
    if gate is not None:
        grads["gate"] = (b * du * n).view(rows // per, per, cols).sum(1)
    if case["post"] != "none":
        grads["post_weight"], grads["post_bias"] = (dn * y2).sum(0), dn.sum(0)
        dn = _plain_norm_grad(dn, w["post_weight"], y2, r2, case["post"])
    out["dz"] = dn.to(dt)
    out.update({"d" + k: grads[k].to(v.dtype) for k, v in weights.items() if v is not None})
    return out


def _plain_rotate(v, cos, sin, case):
    rot, d = case["rotary_dim"], case["head_dim"]
    f = v.float()
    if case["layout"] == "half":
        a, b = f[..., :rot // 2], f[..., rot // 2:rot]
        r = torch.cat((a * cos - b * sin, b * cos + a * sin, f[..., rot:]), -1)
    else:
        a, b = f[..., 0:rot:2], f[..., 1:rot:2]
        r = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
        r = torch.cat((r, f[..., rot:]), -1)
    return r.to(v.dtype)


def _run_rotary(s):
    case, t = s.case, s.t
    if own:
        q, k = s.op.rotate(t["q"], t["k"], positions=t["positions"])
        if not case["train"]:
            return {"q": q, "k": k}
        dq, dk = s.op.rotate(t["dq"], t["dk"], positions=t["positions"], inverse=True)
        return {"q": q, "k": k, "dq": dq, "dk": dk}
    # The angle is reduced to one turn in 64 bits: as a 32-bit product it is off by 0.06 rad at position 1e6.
    angle = torch.remainder(t["positions"].double()[:, None] * s.freq, 2 * math.pi).float()[:, None, :]
    cos, sin = torch.cos(angle) * s.magnitude, torch.sin(angle) * s.magnitude
    out = {"q": _plain_rotate(t["q"], cos, sin, case), "k": _plain_rotate(t["k"], cos, sin, case)}
    if case["train"]:
        out["dq"], out["dk"] = (_plain_rotate(t[n], cos, -sin, case) for n in ("dq", "dk"))
    return out


def run(s):
    return {"clip": _run_clip, "norm": _run_norm, "rotary": _run_rotary}[s.case["op"]](s)


# ------------------------------------------------------------------- work

_BYTES = {"f32": 4, "bf16": 2, "f16": 2}


def work(case):
    """Every input read once, every output written once; a square root, an exponential or a sine counts as one
    operation."""
    if case["op"] == "clip":
        shapes = _shapes(case)
        n = sum(_numel(v) for v in shapes)
        out = _BYTES[case["out"]] if case["clip"] else 0
        return {"bytes": n * (_BYTES[case["grad"]] + out) + 4 * (len(shapes) + 1), "flops": n * (3 if case["clip"] else 2)}
    if case["op"] == "norm":
        rows, cols = case["rows"], case["cols"]
        a = _BYTES[case["dtype"]]
        r = 4 if case["residual"] == "f32" else a
        p = 4 if case["params"] == "f32" else a
        vectors = sum({"none": 0, "rms": 1, "layer": 2}[case[k]] for k in ("post", "pre"))
        gate = {"none": 0, "rows": rows * a, "shared": rows // case["gate_rows"] * p}[case["gate"]]
        nbytes = cols * (rows * (2 * r + 2 * a) + gate + vectors * p)       # x, z, gate, weights; u, h
        flops = rows * cols * (3 + 6 * sum(case[k] != "none" for k in ("post", "pre")))
        if case["train"]:
            nbytes += cols * (rows * (2 * r + 2 * a) + gate + vectors * p)  # du, dh; dx, dz, gradients of the rest
            flops += rows * cols * (6 + 9 * sum(case[k] != "none" for k in ("post", "pre")))
        return {"bytes": nbytes, "flops": flops}
    heads = case["q_heads"] + case["k_heads"]
    passes = 2 if case["train"] else 1
    n = case["tokens"] * heads
    return {"bytes": passes * 2 * n * case["head_dim"] * _BYTES[case["dtype"]] + 8 * case["tokens"],
            "flops": passes * 3 * n * case["rotary_dim"] + 3 * case["tokens"] * case["rotary_dim"] // 2}


# ------------------------------------------------------------------ exact

def _exact_clip(case, seed):
    shapes, flat = _clip_inputs(case, seed)
    grads = _views(flat, shapes)
    squares = [float(torch.dot(v, v)) for v in (g.reshape(-1).double() for g in grads)]
    total = math.sqrt(math.fsum(squares))
    res = {"total": torch.tensor(total, dtype=torch.float64),
           "norms": torch.tensor([math.sqrt(v) for v in squares], dtype=torch.float64)}
    if case["clip"]:
        out = torch.zeros(flat.numel(), dtype=torch.float64, device=DEVICE)
        for g, o in zip(grads, _views(out, shapes)):
            o.copy_(g.double() * (case["max_norm"] / total if total > case["max_norm"] else 1.0))
        res["out"] = out
    return res


def _exact_norm(case, seed):
    """The definition in 64 bits; the gradients by automatic differentiation."""
    t = {k: v.double() for k, v in _norm_inputs(case, seed).items()}
    du, dh = t.pop("du", None), t.pop("dh", None)
    for v in t.values():
        v.requires_grad_(case["train"])

    def normed(v, side):
        if case[side] == "none":
            return v
        centred = v - v.mean(-1, keepdim=True) if case[side] == "layer" else v
        y = centred / torch.sqrt((centred ** 2).mean(-1, keepdim=True) + case["eps"]) * t[side + "_weight"]
        return y + t[side + "_bias"] if case[side] == "layer" else y

    branch = normed(t["z"], "post")
    if case["gate"] != "none":
        groups = t["gate"].shape[0]
        branch = (branch.reshape(groups, -1, case["cols"]) * t["gate"][:, None]).reshape(case["rows"], case["cols"])
    u = case["residual_scale"] * t["x"] + case["branch_scale"] * branch
    h = normed(u, "pre")
    out = {"u": u, "h": h}
    if case["train"]:
        grads = torch.autograd.grad((u, h), list(t.values()), (du, dh))
        out.update({"d" + k: g for k, g in zip(t, grads)})
        order = ("u", "h", "dx", "dz", "dgate", "dpost_weight", "dpost_bias", "dpre_weight", "dpre_bias")
        out = {k: out[k].detach() for k in order if k in out}
    return out


def _exact_rotary(case, seed):
    """A head's pairs as complex numbers, turned by multiplication."""
    t = _rotary_inputs(case, seed)
    freq, magnitude = _frequencies(case)
    angle = torch.outer(t["positions"].double(), torch.tensor(freq, dtype=torch.float64, device=DEVICE))
    turn = torch.polar(torch.full_like(angle, magnitude), angle)[:, None, :]
    rot = case["rotary_dim"]

    def rotate(v, by):
        out = v.double().contiguous()
        pairs = out[..., :rot].reshape(*v.shape[:2], *((2, rot // 2) if case["layout"] == "half" else (rot // 2, 2)))
        if case["layout"] == "half":
            pairs = pairs.transpose(-1, -2)
        turned = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * by)
        if case["layout"] == "half":
            turned = turned.transpose(-1, -2)
        out[..., :rot] = turned.reshape(*v.shape[:2], rot)
        return out

    out = {"q": rotate(t["q"], turn), "k": rotate(t["k"], turn)}
    if case["train"]:
        out["dq"], out["dk"] = (rotate(t[n], turn.conj()) for n in ("dq", "dk"))
    return out


def exact(case, seed):
    return {"clip": _exact_clip, "norm": _exact_norm, "rotary": _exact_rotary}[case["op"]](case, seed)
