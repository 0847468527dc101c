"""A small language model trained by Distributed Lion with the layer operators making its gradients:

    python -m paper_2404_00438_b200.example [--steps 60] [--workers 4]

Residual MLP blocks over the current token's (fixed) embedding and a head over the vocabulary, learning the next word
of a synthetic chain.  Every worker has its own batch; the blocks keep their inputs and pre-activations in 8 bits; every
weight and bias gradient is written straight into the worker's slice of the optimizer's arena, which the
step then reads.  The workers are slices of one GPU, as in the library's benchmark.
"""
from __future__ import annotations

import argparse
from typing import Dict, List, Tuple

import torch

from . import dlion, inputs, layers

BF16 = torch.bfloat16


class Model:
    """Parameter shapes, their place in the arena, and one forward and backward pass."""

    def __init__(self, words: int, width: int, hidden: int, blocks: int):
        self.words, self.width, self.blocks = words, width, blocks
        self.shapes: Dict[str, Tuple[int, ...]] = {}
        for i in range(blocks):
            self.shapes.update({f"w1.{i}": (width, hidden), f"b1.{i}": (hidden,),
                                f"w2.{i}": (hidden, width), f"b2.{i}": (width,)})
        self.shapes["head"] = (words, width)
        numels = [torch.Size(s).numel() for s in self.shapes.values()]
        self.segments, self.d_pad = inputs.layout(numels)

    def views(self, arena: torch.Tensor) -> Dict[str, torch.Tensor]:
        """The parameters' (or gradients') tensors in a flat arena."""
        return {name: arena[o:o + n].view(shape) for (name, shape), (o, n) in zip(self.shapes.items(), self.segments)}

    def initial(self, device, seed: int = 0) -> torch.Tensor:
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        x = torch.zeros(self.d_pad, device=device)
        for name, t in self.views(x).items():
            if t.dim() == 2:
                fan_in = t.shape[1] if name == "head" else t.shape[0]
                t.copy_(torch.randn(t.shape, generator=g, device=device) * fan_in ** -0.5)
        return x

    def loss_and_gradients(self, p: Dict[str, torch.Tensor], g: Dict[str, torch.Tensor], x: torch.Tensor,
                           targets: torch.Tensor) -> torch.Tensor:
        """Mean loss of a batch of embeddings ``x`` (bf16 [m, width]); the gradients of the bf16 parameters ``p``
        are written to ``g``, whose type is the arena's."""
        kept: List[Tuple[layers.Checkpoint8, layers.Checkpoint8]] = []
        for i in range(self.blocks):
            x8 = layers.checkpoint8(x)
            h, z8 = layers.linear_forward(x, p[f"w1.{i}"], p[f"b1.{i}"], act="gelu", keep="8bit")
            x = layers.linear_forward(h, p[f"w2.{i}"], p[f"b2.{i}"], residual=x)
            kept.append((x8, z8))
        grad_dtype = g["head"].dtype
        r = layers.lm_loss(x, p["head"], targets, grad_dtype=grad_dtype, dw=g["head"])
        dx = r.dx
        for i in reversed(range(self.blocks)):
            x8, z8 = kept[i]
            dz, _, _ = layers.linear_backward(dx, p[f"w2.{i}"], z8, act="gelu", grad_dtype=grad_dtype,
                                              dw=g[f"w2.{i}"], db=g[f"b2.{i}"])
            dx, _, _ = layers.linear_backward(dz, p[f"w1.{i}"], x8, residual=dx, grad_dtype=grad_dtype,
                                              dw=g[f"w1.{i}"], db=g[f"b1.{i}"])
        return r.loss


def batch(step: int, worker: int, rows: int, words: int, device) -> Tuple[torch.Tensor, torch.Tensor]:
    """Words and the words that follow them in the chain next = 5 word + 3."""
    g = torch.Generator(device=device)
    g.manual_seed(1 + step * 1009 + worker)
    now = torch.randint(0, words, (rows,), generator=g, device=device)
    return now, (5 * now + 3) % words


def train(steps: int = 60, workers: int = 4, rows: int = 512, words: int = 1000, width: int = 256, hidden: int = 1024,
          blocks: int = 2, lr: float = 1e-3, mode: int = dlion.MAJORITY, report=print) -> List[float]:
    """Losses, averaged over the workers, of every step."""
    device = torch.device("cuda", torch.cuda.current_device())
    model = Model(words, width, hidden, blocks)
    x = model.initial(device)
    table = torch.randn(words, width, generator=torch.Generator(device=device).manual_seed(7), device=device).to(BF16)
    grads = torch.zeros(workers, model.d_pad, dtype=BF16, device=device)
    m = torch.zeros(workers, model.d_pad, device=device)
    packed = torch.zeros(workers, model.d_pad // 32, dtype=torch.int32, device=device)
    opt = dlion.Dlion(model.segments, model.d_pad, workers, lr=lr, weight_decay=0.01, mode=mode, gdtype=dlion.GRAD_BF16)
    losses = []
    for step in range(steps):
        weights = model.views(x.to(BF16))               # every worker holds the same parameters
        total = torch.zeros((), device=device)
        for i in range(workers):
            now, following = batch(step, i, rows, words, device)
            total += model.loss_and_gradients(weights, model.views(grads[i]), table[now], following)
        opt.worker_step(-1, grads, m, packed)
        opt.aggregate_apply(packed, x)
        losses.append(float(total) / workers)
        layers.check()                                  # a kernel whose wait ran out leaves its outputs undefined
        if step % 10 == 0 or step == steps - 1:
            report(f"step {step}: loss {losses[-1]:.3f}")
    opt.destroy()
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--workers", type=int, default=4)
    a = ap.parse_args()
    train(a.steps, a.workers)
