"""Recovering what quantization lost: ``python -m paper_2512_02010_amd.recover``.

A small example that runs the package's pieces as they are meant to be used together.  A feed-forward model with random
weights is the teacher, in full precision.  Its weights quantized to NVFP4 are the student, which stays frozen; beside each of its layers
stand low-rank adapters, one for each of two tasks.  Every step distils the teacher's top logits into the adapters of the tokens'
tasks (``finetune.nvfp4_distill_step``, ``adapted_fprop``, ``adapted_backward``).  At the end one batch mixes both tasks and tokens without an
adapter, as a server's does.
"""
from __future__ import annotations

import torch

from . import finetune as F
from . import linear as L


class AdaptedLinear:
    """A quantized, frozen weight [N][K] with an adapter of rank r for each of several tasks; fp32 master copies, Adam."""

    def __init__(self, weight: torch.Tensor, adapters: int, rank: int, generator: torch.Generator):
        n, k = weight.shape
        self.quantized = L.quantize_weight(weight)
        a = torch.randn((adapters, rank, k), generator=generator, device=weight.device) / k ** 0.5
        self.master = [a, torch.zeros((adapters, n, rank), device=weight.device)]          # B = 0: no change at first
        self.moments = [(torch.zeros_like(t), torch.zeros_like(t)) for t in self.master]
        self.scales = torch.ones(adapters, device=weight.device)
        self.cast()

    def cast(self):
        self.a, self.b = (t.bfloat16() for t in self.master)

    def forward(self, x, which, keep: bool):
        y, h = F.adapted_fprop(x, self.quantized, self.a, self.b, which, self.scales, want_h=True)
        if keep:
            self.kept = (x, h, which)
        return y

    def backward(self, dy, seed: int, want_dx: bool = True):
        x, h, which = self.kept
        dx, *self.grads = F.adapted_backward(dy, x, h, self.quantized, self.a, self.b, which, self.scales, seed, want_dx=want_dx)
        return dx

    def update(self, step: int, rate: float):
        for t, g, (m, v) in zip(self.master, self.grads, self.moments):
            m.lerp_(g, 0.1)
            v.lerp_(g.square(), 0.01)
            t.sub_(rate * (m / (1 - 0.9 ** step)) / ((v / (1 - 0.99 ** step)).sqrt() + 1e-12))
        self.cast()


def run(steps: int = 60, tokens: int = 512, width: int = 256, hidden: int = 512, vocab: int = 2048, rank: int = 16, top: int = 32,
        seed: int = 0, rate: float = 2e-3, say=lambda *a: None):
    """Returns (mean loss of every step, mean loss with adapters and without in the last, mixed batch)."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    shapes = ((hidden, width), (width, hidden), (vocab, width))
    weights = [normal(*s) * (1.6 / s[1] ** 0.5) for s in shapes]
    words = normal(vocab, width)
    layers = [AdaptedLinear(w, 2, rank, g) for w in weights]

    def teacher(x):
        x = x.float()
        z = torch.relu(x @ weights[0].T) @ weights[1].T @ weights[2].T
        return z.topk(top, dim=1)

    def student(x, which, keep=False):
        y = layers[0].forward(x, which, keep)
        r = torch.relu(y)
        return y, layers[2].forward(layers[1].forward(r, which, keep), which, keep)

    losses = []
    for step in range(1, steps + 1):
        x = words[torch.randint(0, vocab, (tokens,), generator=g, device="cuda")].bfloat16()
        which = torch.randint(0, 2, (tokens,), generator=g, device="cuda", dtype=torch.int32)
        values, index = teacher(x)
        y, logits = student(x, which, keep=True)
        loss, d = F.nvfp4_distill_step(logits, values, index, torch.full((tokens,), 1.0 / tokens, device="cuda"), out=logits)
        d = layers[1].backward(layers[2].backward(d, 3 * step), 3 * step + 1)
        layers[0].backward(d * (y > 0), 3 * step + 2, want_dx=False)
        for layer in layers:
            layer.update(step, rate)
        losses.append(loss.mean())
        if step % 20 == 0:
            say(f"step {step}: loss {float(losses[-1]):.5f}")

    # one batch of both tasks and of tokens without an adapter, in any order
    x = words[torch.randint(0, vocab, (tokens,), generator=g, device="cuda")].bfloat16()
    which = torch.randint(-1, 2, (tokens,), generator=g, device="cuda", dtype=torch.int32)
    values, index = teacher(x)
    loss, _ = F.nvfp4_distill_forward(student(x, which)[1], values, index)
    adapted, plain = float(loss[which >= 0].mean()), float(loss[which < 0].mean())
    say(f"mixed batch: loss {adapted:.5f} with adapters, {plain:.5f} without")
    return [float(v) for v in losses], adapted, plain


if __name__ == "__main__":
    run(say=print)
