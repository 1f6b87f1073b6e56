"""Performance cases of the operators at the ends of a training step and in its heads: the token embedding and its
gradient, the norms of queries and keys with the rotation by position, and the loss against a teacher's top logits and
the labels, with its gradient.

``listed()`` are the cases that are timed, ``draw(rng)`` gives more of the same ranges, ``prepare(case, seed)`` makes
what a program has in hand before the call, ``run(state)`` is one pass, ``work(case)`` what that pass cannot do
without, and ``exact(case, seed)`` the results in 64 bits.  With ``own`` false a pass is computed in elementary torch
operations in 32 bits, with ``own`` true by the package's operators.

The operators ("op" of a case):

  embed    out_t = scale W[id_t], a row of zeros for an id outside the vocabulary (padding).  "train" adds the dense
           gradient of the table, dW_v = scale sum over the tokens with id v of dout_t.
  heads    every head of queries and keys divided by its root mean square, times a weight per element, then turned by
           its token's position:
               out = R(position) (x / sqrt(mean(x^2) + eps) * weight)
           "train" adds the gradients of heads and weights.
  distill  rows of logits s against K logits t of a teacher at the indices i, at temperature T, and a label:
               p = softmax(t / T),  loss = a T^2 sum_k p_k (log p_k - log softmax(s / T)[i_k]) - b log softmax(s)[label]
           Teacher entries whose index is negative and labels that are negative are absent; so is a term with nothing
           left.  "train" adds the gradient of the losses' sum times grad_scale with respect to the logits.
"""
import math

import numpy as np
import torch

own = False
DEVICE = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
INTS = {4: torch.int32, 8: torch.int64}


# ------------------------------------------------------------------ cases

def _embed(name, **kw):
    return dict(dict(name=name, op="embed", train=True, scale=1.0, ids="zipf", id_bytes=8, padded=0.0), **kw)


def _heads(name, **kw):
    return dict(dict(name=name, op="heads", train=True, fused=False, base=10000.0, scaling="none", factor=1.0,
                     original=1024, params="f32", eps=1e-6), **kw)


def _distill(name, **kw):
    return dict(dict(name=name, op="distill", train=True, temperature=1.0, teacher_weight=1.0, label_weight=0.0,
                     teacher="same", index_bytes=8, absent=0.0), **kw)


def listed():
    return [
        # Tokens being generated for 8 requests: latency.
        _embed("embed-tokens", train=False, tokens=8, vocab=50257, width=768, weight="bf16", out="bf16"),
        # A training step's batch (16 sequences of 1024) at the benchmark's table: fp32 parameters and residual stream.
        _embed("embed-train-768", tokens=16384, vocab=50257, width=768, weight="f32", out="f32"),
        # An odd width, half precision, padded sequences, rows scaled by the root of the width, few tokens a row.
        _embed("embed-train-odd", tokens=4099, vocab=8191, width=1001, weight="f16", out="f16", scale=31.64, ids="uniform",
               id_bytes=4, padded=0.15),
        # The largest: a long batch and a large table.
        _embed("embed-train-4096", tokens=65536, vocab=131072, width=4096, weight="bf16", out="bf16"),
        # Tokens being generated for 8 requests, late in long contexts: latency.
        _heads("heads-tokens", train=False, tokens=8, q_heads=12, k_heads=12, head_dim=64, rotary_dim=64, dtype="bf16",
               layout="half", positions="random"),
        # A training step's batch of packed sequences, queries and keys inside the fused projection's output.
        _heads("heads-train-768", tokens=16384, q_heads=12, k_heads=12, head_dim=64, rotary_dim=64, dtype="bf16",
               layout="half", positions="packed", fused=True),
        # Grouped heads of an odd size, half of each turned, half precision.
        _heads("heads-train-odd", tokens=3001, q_heads=9, k_heads=3, head_dim=80, rotary_dim=40, dtype="f16",
               layout="interleaved", positions="packed", params="same"),
        # The largest: long sequences, grouped heads, frequencies stretched for the context.
        _heads("heads-train-long", tokens=65536, q_heads=32, k_heads=8, head_dim=128, rotary_dim=128, dtype="bf16",
               layout="half", positions="prompt", scaling="ramp", factor=8.0, original=8192),
        # The losses of a few tokens, no gradient: latency.
        _distill("distill-rows", train=False, rows=8, vocab=50257, k=16, dtype="bf16"),
        # A training step's rows at the benchmark's vocabulary: a softened teacher and the labels together.
        _distill("distill-train-50257", rows=8192, vocab=50257, k=64, dtype="bf16", temperature=2.0, label_weight=0.5),
        # fp32 logits of an odd vocabulary, few entries, some rows without a teacher or a label.
        _distill("distill-train-odd", rows=1021, vocab=32003, k=7, dtype="f32", label_weight=0.5, teacher="bf16",
                 index_bytes=4, absent=0.2),
        # The largest: a vocabulary of 131072, the teacher alone.
        _distill("distill-train-131072", rows=8192, vocab=131072, k=128, dtype="bf16", temperature=2.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Half of them multiples of 64, the others any number."""
    n = _log_int(rng, lo, hi)
    return max(64, n // 64 * 64) if rng.random() < 0.5 else n


def _draw_embed(rng):
    width = _width(rng, 48, 8192)
    vocab = _log_int(rng, 16, max(17, min(262144, 400_000_000 // width)))
    tokens = _log_int(rng, 1, max(2, min(131072, 200_000_000 // width)))
    weight = rng.choice(("f32", "bf16", "bf16", "f16"))
    return dict(op="embed", train=rng.random() < 0.8, tokens=tokens, vocab=vocab, width=width, weight=weight,
                out=rng.choice((weight, "f32", "bf16")), scale=rng.choice((1.0, float("%.4g" % math.sqrt(width)))),
                ids=rng.choice(("zipf", "zipf", "uniform", "few")), id_bytes=rng.choice((4, 8, 8)),
                padded=rng.choice((0.0, 0.0, 0.15)))


def _draw_heads(rng):
    head_dim = rng.choice((32, 64, 64, 80, 96, 128, 128, 256, rng.randint(17, 200)))
    rotary_dim = head_dim // 2 * 2 if rng.random() < 0.5 else 2 * rng.randint(2, head_dim // 2)
    k_heads = _log_int(rng, 1, 16)
    q_heads = k_heads * rng.choice((1, 1, 2, 4, 8))
    tokens = _log_int(rng, 1, max(2, min(131072, 250_000_000 // ((q_heads + k_heads) * head_dim))))
    scaling = rng.choice(("none", "none", "linear", "base", "ramp"))
    return dict(op="heads", train=rng.random() < 0.75, tokens=tokens, q_heads=q_heads, k_heads=k_heads, head_dim=head_dim,
                rotary_dim=rotary_dim, dtype=rng.choice(("bf16", "bf16", "f16", "f32")),
                layout=rng.choice(("half", "interleaved")), positions=rng.choice(("prompt", "packed", "random")),
                fused=rng.random() < 0.5, base=rng.choice((10000.0, 500000.0)), scaling=scaling,
                factor=1.0 if scaling == "none" else rng.choice((2.0, 8.0, 32.0)), original=rng.choice((1024, 8192)),
                params=rng.choice(("f32", "f32", "same")), eps=rng.choice((1e-5, 1e-6)))


def _draw_distill(rng):
    vocab = _log_int(rng, 100, 262144)
    vocab = vocab // 64 * 64 if vocab > 640 and rng.random() < 0.5 else vocab
    k = 0 if rng.random() < 0.15 else _log_int(rng, 1, min(256, vocab // 2))
    rows = _log_int(rng, 1, max(2, min(16384, 600_000_000 // vocab)))
    label = 1.0 if k == 0 else rng.choice((0.0, 0.5, 0.1))
    return dict(op="distill", train=rng.random() < 0.8, rows=rows, vocab=vocab, k=k,
                dtype=rng.choice(("bf16", "bf16", "f16", "f32")), temperature=rng.choice((1.0, 2.0, round(rng.uniform(0.7, 4.0), 2))),
                teacher_weight=0.0 if k == 0 else rng.choice((1.0, 0.9)), label_weight=label,
                teacher=rng.choice(("same", "bf16", "f32")), index_bytes=rng.choice((4, 8)), absent=rng.choice((0.0, 0.0, 0.2)))


def draw(rng):
    return rng.choice((_draw_embed, _draw_heads, _draw_distill))(rng)


# ----------------------------------------------------------------- inputs

class _State:
    """What a program keeps between passes."""


def _gen(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _shares(case):
    """The share of every id in a text: frequencies fall with the rank, and ids are numbered about by frequency; or all
    alike; or a handful of ids."""
    vocab = case["vocab"]
    if case["ids"] == "uniform":
        return np.full(vocab, 1.0 / vocab)
    n = min(vocab, 5) if case["ids"] == "few" else vocab
    p = np.zeros(vocab)
    p[:n] = 1.0 / (np.arange(n) + 2.7)
    return p / p.sum()


def _normal(gen, shape, dtype, scale=1.0):
    return torch.randn(*shape, generator=gen, device=DEVICE).mul_(scale).to(dtype)


def _embed_inputs(case, seed):
    gen, tokens = _gen(seed), case["tokens"]
    ends = torch.from_numpy(np.cumsum(_shares(case))).to(DEVICE)
    u = torch.rand(tokens, generator=gen, device=DEVICE, dtype=torch.float64)
    ids = torch.searchsorted(ends, u, right=True).clamp_(max=case["vocab"] - 1)
    if case["padded"]:                      # the ends of sequences in a padded batch
        at = torch.arange(tokens, device=DEVICE) % 128
        ids = torch.where(at >= 128 * (1.0 - case["padded"]), torch.full_like(ids, -1), ids)
    t = {"ids": ids.to(INTS[case["id_bytes"]]),
         "weight": _normal(gen, (case["vocab"], case["width"]), DTYPES[case["weight"]], 0.02)}
    if case["train"]:
        t["dout"] = _normal(gen, (tokens, case["width"]), DTYPES[case["out"]], 0.05)
    return t


def _heads_inputs(case, seed):
    """Heads of different sizes, as projections leave them, and weights about one."""
    gen, tokens, d = _gen(seed), case["tokens"], case["head_dim"]
    dt, hq, hk = DTYPES[case["dtype"]], case["q_heads"], case["k_heads"]
    pt = torch.float32 if case["params"] == "f32" else dt
    t = {}
    if case["fused"]:               # queries, keys and values side by side
        qkv = _normal(gen, (tokens, (hq + 2 * hk) * d), dt, 1.5)
        t["q"] = qkv[:, :hq * d].unflatten(1, (hq, d))
        t["k"] = qkv[:, hq * d:(hq + hk) * d].unflatten(1, (hk, d))
    else:
        t["q"], t["k"] = _normal(gen, (tokens, hq, d), dt, 1.5), _normal(gen, (tokens, hk, d), dt, 0.7)
    for name in ("q_weight", "k_weight"):
        t[name] = (1.0 + 0.1 * torch.randn(d, generator=gen, device=DEVICE)).to(pt)
    at = torch.arange(tokens, device=DEVICE)
    if case["positions"] == "prompt":
        t["positions"] = at
    elif case["positions"] == "packed":     # sequences of different lengths, one after the other
        start = torch.rand(tokens, generator=gen, device=DEVICE) < 1.0 / min(700, tokens)
        t["positions"] = at - torch.cummax(torch.where(start, at, torch.zeros_like(at)), 0).values
    else:                                   # requests at any point of contexts of up to a million tokens
        t["positions"] = torch.randint(0, 1 << 20, (tokens,), generator=gen, device=DEVICE)
    if case["train"]:
        t["dq"], t["dk"] = _normal(gen, (tokens, hq, d), dt, 0.1), _normal(gen, (tokens, hk, d), dt, 0.1)
    return t


def _frequencies(case):
    """Radians per position of every pair, and the factor on the turned values.

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


def _distill_inputs(case, seed):
    """Logits of a model that is some way to its teacher: the entries that the teacher ranks highest stand out."""
    gen, rows, vocab, k = _gen(seed), case["rows"], case["vocab"], case["k"]
    dt = DTYPES[case["dtype"]]
    logits = torch.empty(rows, vocab, dtype=dt, device=DEVICE)
    step = max(1, (1 << 26) // vocab)
    for r in range(0, rows, step):
        logits[r:r + step].copy_(torch.randn(logits[r:r + step].shape, generator=gen, device=DEVICE).mul_(2.0))
    t = {}
    first = torch.randint(0, vocab, (rows, 1), generator=gen, device=DEVICE)
    if k:
        gap = 1 + (torch.rand(rows, 1, generator=gen, device=DEVICE) * (vocab // k)).long().clamp_(max=max(0, vocab // k - 1))
        index = (first + gap * torch.arange(k, device=DEVICE)) % vocab      # distinct: k gap <= vocab
        fall = torch.rand(rows, k, generator=gen, device=DEVICE).cumsum(1) * (12.0 / k)
        t["teacher"] = (14.0 - fall).to(dt if case["teacher"] == "same" else DTYPES[case["teacher"]])
        lift = logits.gather(1, index).float() + 9.0 - fall
        logits.scatter_(1, index, lift.to(dt))
        if case["absent"]:                  # fewer entries than K, down to none
            left = (torch.rand(rows, 1, generator=gen, device=DEVICE) / (1.0 - case["absent"]) * k).long()
            index = torch.where(torch.arange(k, device=DEVICE) < left, index, torch.full_like(index, -1))
        t["index"] = index.to(INTS[case["index_bytes"]])
    if case["label_weight"]:
        labels = first[:, 0]
        if case["absent"]:
            gone = torch.rand(rows, generator=gen, device=DEVICE) < case["absent"]
            labels = torch.where(gone, torch.full_like(labels, -100), labels)
        t["labels"] = labels
    t["logits"] = logits
    return t


# ------------------------------------------------------------ prepare, run

_INPUTS = {"embed": _embed_inputs, "heads": _heads_inputs, "distill": _distill_inputs}


def _grad_scale(case):
    """The gradient of the rows' mean; float16 ones are scaled up, as a float16 training loop's loss is."""
    return (4096.0 if case["dtype"] == "f16" else 1.0) / case["rows"]


def prepare(case, seed):
    s = _State()
    s.case, s.t = case, _INPUTS[case["op"]](case, seed)
    if case["op"] == "embed":
        if own:
            from paper_2609_30342_gb300 import embedding
            s.op = embedding.TokenEmbedding(case["vocab"], case["width"], scale=case["scale"])
    elif case["op"] == "heads":
        freq, s.magnitude = _frequencies(case)
        if own:
            from paper_2609_30342_gb300 import layers
            scaling = None if case["scaling"] == "none" else dict(kind=case["scaling"], factor=case["factor"],
                                                                  original_context=case["original"])
            s.op = layers.RotaryNorm(case["head_dim"], case["rotary_dim"], base=case["base"], layout=case["layout"],
                                     scaling=scaling, eps=case["eps"], device=DEVICE)
        else:
            s.freq = torch.tensor(freq, dtype=torch.float64, device=DEVICE)
    elif own:
        from paper_2609_30342_gb300 import losses
        s.op = losses.DistillationLoss(temperature=case["temperature"], teacher_weight=case["teacher_weight"],
                                       label_weight=case["label_weight"])
    return s


def _run_embed(s):
    case, t = s.case, s.t
    if own:
        out = {"out": s.op.forward(t["weight"], t["ids"], dtype=DTYPES[case["out"]])}
        if case["train"]:
            out["dweight"] = s.op.backward(t["dout"], t["ids"], dtype=t["weight"].dtype)
        return out
    vocab, ids = case["vocab"], t["ids"].long()
    inside = (ids >= 0) & (ids < vocab)
    rows = t["weight"][torch.where(inside, ids, torch.zeros_like(ids))].float() * case["scale"]
    out = {"out": torch.where(inside[:, None], rows, torch.zeros_like(rows)).to(DTYPES[case["out"]])}
    if case["train"]:
        dw = torch.zeros(vocab + 1, case["width"], dtype=torch.float32, device=DEVICE)      # the last row: padding
        dw.index_add_(0, torch.where(inside, ids, torch.full_like(ids, vocab)), t["dout"].float())
        out["dweight"] = (dw[:vocab] * case["scale"]).to(t["weight"].dtype)
    return out


def _plain_turn(f, cos, sin, case):
    rot = case["rotary_dim"]
    if case["layout"] == "half":
        a, b = f[..., :rot // 2], f[..., rot // 2:rot]
        return torch.cat((a * cos - b * sin, b * cos + a * sin, f[..., rot:]), -1)
    a, b = f[..., 0:rot:2], f[..., 1:rot:2]
    return torch.cat((torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2), f[..., rot:]), -1)


def _run_heads(s):
    case, t = s.case, s.t
    if own:
        q, k = s.op.forward(t["q"], t["k"], t["q_weight"], t["k_weight"], positions=t["positions"])
        out = {"q": q, "k": k}
        if case["train"]:
            g = s.op.backward(t["dq"], t["dk"], t["q"], t["k"], t["q_weight"], t["k_weight"], positions=t["positions"])
            out.update(dq=g.q, dk=g.k, dq_weight=g.q_weight, dk_weight=g.k_weight)
        return out
    # The angle is reduced to one turn in 64 bits: as a 32-bit product it is off by 0.06 rad at position 1e6.
    angle = torch.remainder(t["positions"].double()[:, None] * s.freq, 2 * math.pi).float()[:, None, :]
    cos, sin = torch.cos(angle) * s.magnitude, torch.sin(angle) * s.magnitude
    out = {}
    for n in ("q", "k"):
        x, w = t[n].float(), t[n + "_weight"].float()
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + case["eps"])
        y = x * r
        out[n] = _plain_turn(y * w, cos, sin, case).to(t[n].dtype)
        if case["train"]:
            dy = _plain_turn(t["d" + n].float(), cos, -sin, case)
            g = dy * w
            out["d" + n] = (r * (g - y * (g * y).mean(-1, keepdim=True))).to(t[n].dtype)
            out["d" + n + "_weight"] = (dy * y).sum((0, 1)).to(t[n + "_weight"].dtype)
    return out


def _run_distill(s):
    case, t = s.case, s.t
    logits, teacher, index, labels = t["logits"], t.get("teacher"), t.get("index"), t.get("labels")
    scale = _grad_scale(case)
    if own:
        if not case["train"]:
            return {"loss": s.op.forward(logits, teacher, index, labels)[0]}
        loss, dlogits = s.op.loss_and_gradient(logits, teacher, index, labels, grad_scale=scale)
        return {"loss": loss, "dlogits": dlogits}
    x, T = logits.float(), case["temperature"]
    loss = torch.zeros(case["rows"], dtype=torch.float32, device=DEVICE)
    grad = None
    if teacher is not None:
        a = case["teacher_weight"]
        there, at = index >= 0, index.long().clamp(min=0)
        some = there.any(1, keepdim=True)
        e = torch.exp((teacher.float() - teacher.float().max(1, keepdim=True).values) / T) * there
        p = e / e.sum(1, keepdim=True).clamp(min=1e-30)
        top = x.max(1, keepdim=True).values
        e = torch.exp((x - top) / T)
        total = e.sum(1, keepdim=True)
        log_q = (x.gather(1, at) - top) / T - torch.log(total)
        loss = loss + a * T * T * (torch.where(p > 0, p * (torch.log(p.clamp(min=1e-38)) - log_q), torch.zeros_like(p))).sum(1)
        if case["train"]:
            grad = e * (some * (a * T * scale) / total)
            grad.scatter_add_(1, at, p * (-a * T * scale))
    if labels is not None:
        b = case["label_weight"]
        there, at = (labels >= 0)[:, None], labels.clamp(min=0)[:, None]
        top = x.max(1, keepdim=True).values
        e = torch.exp(x - top)
        total = e.sum(1, keepdim=True)
        loss = loss - b * (there * (x.gather(1, at) - top - torch.log(total)))[:, 0]
        if case["train"]:
            e = e * (there * (b * scale) / total)
            grad = e if grad is None else grad + e
            grad.scatter_add_(1, at, there * torch.full_like(total, -b * scale))
    return {"loss": loss, "dlogits": grad.to(logits.dtype)} if case["train"] else {"loss": loss}


def run(s):
    return {"embed": _run_embed, "heads": _run_heads, "distill": _run_distill}[s.case["op"]](s)


# ------------------------------------------------------------------- work

_BYTES = {"f32": 4, "bf16": 2, "f16": 2}


def work(case):
    """Every input read once (of the table, the rows that occur), every output written once; a root, an exponential, a
    logarithm or a sine counts as one operation."""
    if case["op"] == "embed":
        tokens, width, vocab = case["tokens"], case["width"], case["vocab"]
        inside = tokens * (1.0 - case["padded"])
        distinct = float(-np.expm1(inside * np.log1p(-np.minimum(_shares(case), 1 - 1e-12))).sum())
        w, o = _BYTES[case["weight"]], _BYTES[case["out"]]
        passes = 2 if case["train"] else 1
        nbytes = passes * (tokens * case["id_bytes"] + tokens * width * o) + distinct * width * w
        if case["train"]:
            nbytes += vocab * width * w
        return {"bytes": int(nbytes), "flops": int(passes * inside * width)}
    if case["op"] == "heads":
        n = case["tokens"] * (case["q_heads"] + case["k_heads"])
        d, rot, b = case["head_dim"], case["rotary_dim"], _BYTES[case["dtype"]]
        p = 4 if case["params"] == "f32" else b
        nbytes = 2 * n * d * b + 8 * case["tokens"] + 2 * d * p
        flops = n * (4 * d + 3 * rot) + 3 * case["tokens"] * rot // 2
        if case["train"]:
            nbytes += 2 * n * d * b + 2 * d * p     # the heads are read once for both directions
            flops += n * (9 * d + 3 * rot)
        return {"bytes": nbytes, "flops": flops}
    n, k, b = case["rows"] * case["vocab"], case["rows"] * case["k"], _BYTES[case["dtype"]]
    softmaxes = 2 if case["k"] and case["label_weight"] and case["temperature"] != 1.0 else 1
    t = b if case["teacher"] == "same" else _BYTES[case["teacher"]]
    nbytes = n * b + k * (t + case["index_bytes"]) + case["rows"] * (4 + (8 if case["label_weight"] else 0))
    flops = n * (1 + 3 * softmaxes) + 8 * k
    if case["train"]:
        nbytes += n * b
        flops += n * 2 * softmaxes + 2 * k
    return {"bytes": nbytes, "flops": flops}


# ------------------------------------------------------------------ exact

def _exact_embed(case, seed):
    """A product with the matrix that has scale at (token, id), and with its transpose."""
    t = _embed_inputs(case, seed)
    tokens, vocab = case["tokens"], case["vocab"]
    at = torch.nonzero(t["ids"] >= 0)[:, 0]
    ids = t["ids"].long()[at]
    out = torch.zeros(tokens, case["width"], dtype=torch.float64, device=DEVICE)
    out[at] = t["weight"][ids].double() * case["scale"]
    res = {"out": out}
    if case["train"]:
        dw = torch.zeros(vocab, case["width"], dtype=torch.float64, device=DEVICE)
        dw.index_put_((ids,), t["dout"][at].double() * case["scale"], accumulate=True)
        res["dweight"] = dw
    return res


def _exact_heads(case, seed):
    """A head's pairs as complex numbers, turned by multiplication; the gradients by automatic differentiation."""
    t = _heads_inputs(case, seed)
    freq, magnitude = _frequencies(case)
    angle = torch.outer(t["positions"].double(), torch.tensor(freq, dtype=torch.float64, device=DEVICE))
    turn = torch.polar(torch.full_like(angle, magnitude), angle)[:, None, :]
    rot, half = case["rotary_dim"], case["layout"] == "half"
    res = {}
    for n in ("q", "k"):
        total, outs, grads = None, [], []
        step = max(1, (1 << 27) // (t[n].shape[1] * case["head_dim"]))
        w = t[n + "_weight"].double().requires_grad_(case["train"])
        for i in range(0, case["tokens"], step):
            x = t[n][i:i + step].double().requires_grad_(case["train"])
            y = x / torch.sqrt((x ** 2).mean(-1, keepdim=True) + case["eps"]) * w
            pairs = y[..., :rot].unflatten(-1, (2, rot // 2) if half else (rot // 2, 2))
            pairs = pairs.transpose(-1, -2) if half else pairs
            turned = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn[i:i + step])
            turned = turned.transpose(-1, -2) if half else turned
            out = torch.cat((turned.flatten(-2), y[..., rot:]), -1)
            outs.append(out.detach())
            if case["train"]:
                dx, dw = torch.autograd.grad(out, (x, w), t["d" + n][i:i + step].double())
                grads.append(dx)
                total = dw if total is None else total + dw
        res[n] = torch.cat(outs)
        if case["train"]:
            res["d" + n], res["d" + n + "_weight"] = torch.cat(grads), total
    return {n: res[n] for n in ("q", "k", "dq", "dq_weight", "dk", "dk_weight") if n in res}


def _exact_distill(case, seed):
    """The definition by rows' log-softmax in 64 bits; the gradient by automatic differentiation."""
    t, T = _distill_inputs(case, seed), case["temperature"]
    step = max(1, (1 << 26) // case["vocab"])
    losses, grads = [], []
    for i in range(0, case["rows"], step):
        x = t["logits"][i:i + step].double().requires_grad_(case["train"])
        loss = torch.zeros(x.shape[0], dtype=torch.float64, device=DEVICE)
        if case["k"]:
            index = t["index"][i:i + step].long()
            there = index >= 0
            soft = (t["teacher"][i:i + step].double() / T).masked_fill(~there, -math.inf)
            soft = torch.where(there.any(1, keepdim=True), soft, torch.zeros_like(soft)).log_softmax(1)
            log_q = torch.log_softmax(x / T, 1).gather(1, index.clamp(min=0))
            kl = torch.where(there, soft.exp() * (soft.masked_fill(~there, 0.0) - log_q), torch.zeros_like(soft))
            loss = loss + case["teacher_weight"] * T ** 2 * kl.sum(1)
        if case["label_weight"]:
            labels = t["labels"][i:i + step]
            nll = -torch.log_softmax(x, 1).gather(1, labels.clamp(min=0)[:, None])[:, 0]
            loss = loss + case["label_weight"] * torch.where(labels >= 0, nll, torch.zeros_like(nll))
        if case["train"]:
            grads.append(torch.autograd.grad(loss.sum() * _grad_scale(case), x)[0])
        losses.append(loss.detach())
    return {"loss": torch.cat(losses), "dlogits": torch.cat(grads)} if case["train"] else {"loss": torch.cat(losses)}


def exact(case, seed):
    return {"embed": _exact_embed, "heads": _exact_heads, "distill": _exact_distill}[case["op"]](case, seed)
