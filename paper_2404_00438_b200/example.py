"""A small language model trained by Distributed Lion with the layer operators making its gradients:

    python -m paper_2404_00438_b200.example [--steps 60] [--workers 4] [--attention]

Residual MLP blocks over the current token's (fixed) embedding and a head over the vocabulary, learning the next word
of a synthetic chain; with ``--attention`` blocks of layer norm, causal attention over packed sequences and MLP, learning a chain
in which the next word depends on the last two.  Every worker has its own batch; the blocks keep their inputs and pre-activations in 8 bits; every
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


class Decoder(Model):
    """Blocks x + attention(norm(x)), then x + mlp(norm(x)), with grouped heads, over sequences packed one behind the other."""

    def __init__(self, words: int, width: int, hidden: int, blocks: int, heads: int, kv_heads: int):
        self.words, self.width, self.blocks, self.heads, self.kv_heads = words, width, blocks, heads, kv_heads
        self.dim = width // heads
        mixed = (heads + 2 * kv_heads) * self.dim
        self.shapes = {}
        for i in range(blocks):
            self.shapes.update({f"n1.{i}": (width,), f"c1.{i}": (width,), f"qkv.{i}": (width, mixed), f"bqkv.{i}": (mixed,),
                                f"out.{i}": (width, width), f"bout.{i}": (width,), f"n2.{i}": (width,), f"c2.{i}": (width,),
                                f"w1.{i}": (width, hidden), f"b1.{i}": (hidden,), f"w2.{i}": (hidden, width), f"b2.{i}": (width,)})
        self.shapes.update({"n": (width,), "c": (width,), "head": (words, width)})
        self.segments, self.d_pad = inputs.layout([torch.Size(s).numel() for s in self.shapes.values()])

    def initial(self, device, seed: int = 0) -> torch.Tensor:
        x = super().initial(device, seed)
        for name, t in self.views(x).items():
            if name.split(".")[0] in ("n", "n1", "n2"):
                t.fill_(1.0)
        return x

    def _split(self, t: torch.Tensor):
        """q, k and v in a product's output (or their gradients' places in its gradient)."""
        t = t.view(t.shape[0], self.heads + 2 * self.kv_heads, self.dim)
        return t[:, :self.heads], t[:, self.heads:self.heads + self.kv_heads], t[:, self.heads + self.kv_heads:]

    def loss_and_gradients(self, p: Dict[str, torch.Tensor], g: Dict[str, torch.Tensor], x: torch.Tensor, targets: torch.Tensor,
                           offsets: torch.Tensor = None) -> torch.Tensor:
        """As :meth:`Model.loss_and_gradients`; ``offsets`` says where the sequences begin and end.  Rows behind the last one
        should have no target: attention neither reads nor makes anything there."""
        m = x.shape[0]
        kept = []
        for i in range(self.blocks):
            a, s1 = layers.norm_forward(x, p[f"n1.{i}"], p[f"c1.{i}"])
            mixed = layers.linear_forward(a, p[f"qkv.{i}"], p[f"bqkv.{i}"])
            o, lse = layers.attention_forward(*self._split(mixed), offsets=offsets)
            y = layers.linear_forward(o.view(m, self.width), p[f"out.{i}"], p[f"bout.{i}"], residual=x)
            b, s2 = layers.norm_forward(y, p[f"n2.{i}"], p[f"c2.{i}"])
            h, z8 = layers.linear_forward(b, p[f"w1.{i}"], p[f"b1.{i}"], act="gelu", keep="8bit")
            kept.append((x, s1, a, mixed, o, lse, y, s2, b, z8))
            x = layers.linear_forward(h, p[f"w2.{i}"], p[f"b2.{i}"], residual=y)
        a, s = layers.norm_forward(x, p["n"], p["c"])
        dt = g["head"].dtype
        r = layers.lm_loss(a, p["head"], targets, grad_dtype=dt, dw=g["head"])
        dx, _, _ = layers.norm_backward(r.dx, x, p["n"], s, grad_dtype=dt, dw=g["n"], db=g["c"])
        for i in reversed(range(self.blocks)):
            x, s1, a, mixed, o, lse, y, s2, b, z8 = kept[i]
            dz, _, _ = layers.linear_backward(dx, p[f"w2.{i}"], z8, act="gelu", grad_dtype=dt, dw=g[f"w2.{i}"], db=g[f"b2.{i}"])
            db, _, _ = layers.linear_backward(dz, p[f"w1.{i}"], b, grad_dtype=dt, dw=g[f"w1.{i}"], db=g[f"b1.{i}"])
            dy, _, _ = layers.norm_backward(db, y, p[f"n2.{i}"], s2, residual=dx, grad_dtype=dt, dw=g[f"n2.{i}"], db=g[f"c2.{i}"])
            do, _, _ = layers.linear_backward(dy, p[f"out.{i}"], o.view(m, self.width), grad_dtype=dt, dw=g[f"out.{i}"], db=g[f"bout.{i}"])
            dmixed = torch.empty_like(mixed)
            dq, dk, dv = self._split(dmixed)
            layers.attention_backward(do.view(o.shape), *self._split(mixed), o, lse, offsets=offsets, dq=dq, dk=dk, dv=dv, zero_rest=True)
            da, _, _ = layers.linear_backward(dmixed, p[f"qkv.{i}"], a, grad_dtype=dt, dw=g[f"qkv.{i}"], db=g[f"bqkv.{i}"])
            dx, _, _ = layers.norm_backward(da, x, p[f"n1.{i}"], s1, residual=dy, grad_dtype=dt, dw=g[f"n1.{i}"], db=g[f"c1.{i}"])
        return r.loss


def documents(step: int, worker: int, rows: int, words: int, device) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """Sequences of 40 to 79 words in ``rows`` rows, in which a word is the sum of the last two; the words, those that follow them
    (-100 for a sequence's first word, after which anything may come, and behind the last sequence) and the offsets."""
    g = torch.Generator()
    g.manual_seed(1 + step * 1009 + worker)
    now, following, offsets = torch.zeros(rows, dtype=torch.int64), torch.full((rows,), -100), [0]
    while offsets[-1] + 80 <= rows:
        n = int(torch.randint(40, 80, (1,), generator=g))
        a, b = (int(v) for v in torch.randint(0, words, (2,), generator=g))
        at = offsets[-1]
        for i in range(n):
            now[at + i] = a
            if i > 0:
                following[at + i] = b
            a, b = b, (a + b) % words
        offsets.append(at + n)
    return now.to(device), following.to(device), torch.tensor(offsets, device=device)


def batch(step: int, worker: int, rows: int, words: int, device) -> Tuple[torch.Tensor, torch.Tensor]:
    """Words and the words that follow them in the chain next = 5 word + 3."""
    g = torch.Generator(device=device)
    g.manual_seed(1 + step * 1009 + worker)
    now = torch.randint(0, words, (rows,), generator=g, device=device)
    return now, (5 * now + 3) % words


def train(steps: int = 60, workers: int = 4, rows: int = 512, words: int = 1000, width: int = 256, hidden: int = 1024,
          blocks: int = 2, lr: float = 1e-3, mode: int = dlion.MAJORITY, report=print, attention: bool = False) -> List[float]:
    """Losses, averaged over the workers, of every step."""
    device = torch.device("cuda", torch.cuda.current_device())
    model = Decoder(words, width, hidden, blocks, heads=width // 64, kv_heads=width // 128) if attention else Model(words, width, hidden, blocks)
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
            if attention:
                now, following, offsets = documents(step, i, rows, words, device)
                total += model.loss_and_gradients(weights, model.views(grads[i]), table[now], following, offsets)
            else:
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
    ap.add_argument("--attention", action="store_true", help="a decoder over packed sequences instead of MLP blocks")
    a = ap.parse_args()
    train(a.steps, a.workers, words=100 if a.attention else 1000, attention=a.attention)
