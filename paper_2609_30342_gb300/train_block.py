"""A small language model trained with the library's operators around its matrix products.

    python -m paper_2609_30342_gb300.train_block [--steps 60] [--layers 2] [--width 256]

Transformer blocks with norms before and after each branch and a learned gate per channel (``layers.ResidualNorm``),
rotary positions over packed sequences (``layers.Rotary``), the gradients clipped to a largest global norm
(``RIKFADOptimizer.clip_grad_norm``) and the R-iKFAD step.  Activations are bfloat16, the residual stream and the
parameters float32.  The data are synthetic: every token is a fixed function of the two before it, with some noise.
"""
import argparse

import torch
from torch import nn

from .layers import ResidualNorm, Rotary
from .optim import RIKFADOptimizer


class Block(nn.Module):
    """Attention and a two-layer perceptron.  ``forward`` takes the residual stream and its normed rows and gives both
    for what follows."""

    def __init__(self, width, heads, norm, rotary):
        super().__init__()
        self.heads, self.norm, self.rotary = heads, norm, rotary
        self.qkv, self.out = nn.Linear(width, 3 * width, bias=False), nn.Linear(width, width, bias=False)
        self.up, self.down = nn.Linear(width, 4 * width, bias=False), nn.Linear(4 * width, width, bias=False)
        for name in ("attention", "mlp"):
            self.register_parameter(name + "_gate", nn.Parameter(torch.ones(1, width)))
            self.register_parameter(name + "_post", nn.Parameter(torch.ones(width)))
            self.register_parameter(name + "_pre", nn.Parameter(torch.ones(width)))

    def attend(self, h, positions, mask):
        tokens, width = h.shape
        q, k, v = torch.nn.functional.linear(h, self.qkv.weight.to(h.dtype)).view(tokens, 3, self.heads, -1).unbind(1)
        q, k = self.rotary(q, k, positions=positions)
        scores = torch.einsum("ihd,jhd->hij", q, k).float() * q.shape[-1] ** -0.5
        weights = torch.softmax(scores.masked_fill(~mask, float("-inf")), -1).to(h.dtype)
        mixed = torch.einsum("hij,jhd->ihd", weights, v).reshape(tokens, width)
        return torch.nn.functional.linear(mixed, self.out.weight.to(h.dtype))

    def perceptron(self, h):
        up = torch.nn.functional.linear(h, self.up.weight.to(h.dtype))
        return torch.nn.functional.linear(torch.nn.functional.gelu(up), self.down.weight.to(h.dtype))

    def forward(self, x, h, positions, mask):
        x, h = self.norm(x, self.attend(h, positions, mask), self.attention_gate, post_weight=self.attention_post,
                         pre_weight=self.attention_pre)
        return self.norm(x, self.perceptron(h), self.mlp_gate, post_weight=self.mlp_post, pre_weight=self.mlp_pre)


class Model(nn.Module):
    def __init__(self, vocab=512, width=256, layers=2, heads=4, dtype=torch.bfloat16, norm=None, first=None, rotary=None):
        super().__init__()
        self.dtype = dtype
        self.embed = nn.Embedding(vocab, width)
        nn.init.normal_(self.embed.weight, std=0.02)
        self.first = ResidualNorm(width, pre="rms") if first is None else first
        norm = ResidualNorm(width, post="rms", pre="rms", branch_scale=(2 * layers) ** -0.5) if norm is None else norm
        rotary = Rotary(width // heads) if rotary is None else rotary
        self.blocks = nn.ModuleList([Block(width, heads, norm, rotary) for _ in range(layers)])
        self.scale = nn.Parameter(torch.ones(width))

    def forward(self, tokens, positions):
        """Logits of packed sequences: ``positions`` starts again at 0 with each of them."""
        sequence = torch.cumsum(positions == 0, 0)
        at = torch.arange(tokens.numel(), device=tokens.device)
        mask = (sequence[:, None] == sequence[None]) & (at[:, None] >= at[None])
        x, h = self.first(self.embed(tokens), pre_weight=self.scale, dtype=self.dtype)
        for block in self.blocks:
            x, h = block(x, h, positions, mask)
        return torch.nn.functional.linear(h, self.embed.weight.to(h.dtype)).float()


def batch(step, vocab, lengths, device="cuda"):
    """(tokens, positions) of packed sequences of the given lengths."""
    gen = torch.Generator()
    gen.manual_seed(step)
    tokens, positions = [], []
    for n in lengths:
        s = torch.randint(0, vocab, (2,), generator=gen).tolist()
        noise = torch.rand(n, generator=gen)
        other = torch.randint(0, vocab, (n,), generator=gen)
        for i in range(2, n + 1):
            s.append(int(other[i - 2]) if noise[i - 2] < 0.02 else (3 * s[-1] + s[-2] + 7) % 17)
        tokens.append(torch.tensor(s[:n]))
        positions.append(torch.arange(n))
    return torch.cat(tokens).to(device), torch.cat(positions).to(device)


def loss_of(model, tokens, positions):
    """Mean cross entropy of every token but the sequences' first."""
    logits = model(tokens, positions)
    follows = positions[1:] > 0
    return torch.nn.functional.cross_entropy(logits[:-1][follows], tokens[1:][follows])


def train(steps=60, vocab=512, width=256, layers=2, lengths=(200, 57, 1, 254), max_norm=1.0, lr=0.05, alpha=0.1, mu=1e-2,
          seed=0, report=None):
    """Train on synthetic sequences; returns the losses and gradient norms of the steps."""
    torch.manual_seed(seed)
    model = Model(vocab, width, layers).cuda()
    opt = RIKFADOptimizer(model.parameters(), lr=lr, alpha=alpha, mu=mu)
    history = []
    for step in range(steps):
        tokens, positions = batch(step, vocab, lengths)
        opt.zero_grad()
        loss = loss_of(model, tokens, positions)
        loss.backward()
        norm = opt.clip_grad_norm(max_norm)
        opt.step()
        history.append((loss.detach(), norm))
        if report and (step % 10 == 0 or step == steps - 1):
            report("step %4d  loss %.4f  gradient norm %.4f" % (step, float(loss.detach()), float(norm)))
    opt.check_finite()
    opt.close()
    return [float(v) for v, _ in history], [float(n) for _, n in history]


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--steps", type=int, default=60)
    p.add_argument("--layers", type=int, default=2)
    p.add_argument("--width", type=int, default=256)
    p.add_argument("--max-norm", type=float, default=1.0)
    a = p.parse_args()
    train(a.steps, layers=a.layers, width=a.width, max_norm=a.max_norm, report=print)


if __name__ == "__main__":
    main()
