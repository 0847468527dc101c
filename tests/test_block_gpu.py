"""Norm, attention, products and loss together, as a decoder's training step uses them."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
F64 = torch.float64


@pytest.fixture(scope="module")
def ex():
    assert torch.cuda.is_available(), "this test needs a CUDA device"
    from paper_2404_00438_b200 import build
    build.build()
    from paper_2404_00438_b200 import example
    return example


def reference(model, p, x, targets, lengths):
    """The loss in 64 bits."""
    m, w = x.shape

    def norm(t, weight, bias):
        return torch.nn.functional.layer_norm(t, (w,), weight, bias, 1e-5)

    for i in range(model.blocks):
        mixed = norm(x, p[f"n1.{i}"], p[f"c1.{i}"]) @ p[f"qkv.{i}"] + p[f"bqkv.{i}"]
        q, k, v = model._split(mixed)
        group = model.heads // model.kv_heads
        outs, at = [], 0
        for n in lengths:
            s = torch.einsum("ihc,jhc->hij", q[at:at + n], k[at:at + n].repeat_interleave(group, 1)) / math.sqrt(model.dim)
            s = s.masked_fill(torch.ones(n, n, dtype=torch.bool, device=x.device).triu(1), -math.inf)
            outs.append(torch.einsum("hij,jhc->ihc", torch.softmax(s, 2), v[at:at + n].repeat_interleave(group, 1)).reshape(n, w))
            at += n
        outs.append(torch.zeros(m - at, w, dtype=x.dtype, device=x.device))
        x = x + torch.cat(outs) @ p[f"out.{i}"] + p[f"bout.{i}"]
        h = torch.nn.functional.gelu(norm(x, p[f"n2.{i}"], p[f"c2.{i}"]) @ p[f"w1.{i}"] + p[f"b1.{i}"], approximate="tanh")
        x = x + h @ p[f"w2.{i}"] + p[f"b2.{i}"]
    return torch.nn.functional.cross_entropy(norm(x, p["n"], p["c"]) @ p["head"].t(), targets)


def test_gradients_in_the_arena(ex):
    """Operands rounded some twenty times on the way to the first block (2^-9 each on average) and pre-activations in 8 bits (2^-7
    of an element) leave each tensor's gradient within 5 % in the 2-norm; the arena's padding stays untouched, and rows
    behind the last sequence take no part.  The keys' bias shifts a row's scores alike, so its gradient is 0 but for
    rounding: it is left out."""
    dev = torch.device("cuda:0")
    model = ex.Decoder(words=300, width=256, hidden=512, blocks=2, heads=4, kv_heads=2)
    x = model.initial(dev)
    gen = torch.Generator(device=dev).manual_seed(5)
    for t in model.views(x).values():
        if t.dim() == 1:
            t.add_(torch.randn(t.shape, generator=gen, device=dev) * 0.1)
    p = model.views(x.to(torch.bfloat16))
    lengths = [100, 1, 150, 37]
    rows = sum(lengths) + 12
    inp = torch.randn(rows, 256, generator=gen, device=dev).to(torch.bfloat16)
    targets = (torch.arange(rows, device=dev) * 7) % 300
    targets[-12:] = -100
    offsets = torch.tensor([0] + lengths, device=dev).cumsum(0)
    for dtype in (torch.bfloat16, torch.float32):
        arena = torch.full((model.d_pad,), 3.0, dtype=dtype, device=dev)
        g = model.views(arena)
        loss = model.loss_and_gradients(p, g, inp, targets, offsets)
        q = {k: v.to(F64).requires_grad_() for k, v in p.items()}
        want = reference(model, q, inp.to(F64), targets, lengths)
        want.backward()
        assert abs(float(loss) - float(want.detach())) <= 0.01 * float(want.detach())
        for name in g:
            got, ref = g[name].to(F64), q[name].grad
            if name.startswith("bqkv"):
                keep = torch.ones_like(ref, dtype=torch.bool)
                keep[256:384] = False
                got, ref = got[keep], ref[keep]
            rel = float((got - ref).norm() / ref.norm())
            assert rel <= 0.05, (name, rel)
        mask = torch.ones(model.d_pad, dtype=torch.bool, device=dev)
        for o, n in model.segments:
            mask[o:o + n] = False
        assert bool((arena[mask] == 3.0).all())


def test_a_few_steps_run(ex):
    losses = ex.train(steps=4, workers=2, rows=400, words=50, width=128, hidden=256, blocks=1, report=lambda s: None, attention=True)
    assert len(losses) == 4 and all(math.isfinite(v) for v in losses)


def test_a_step_captured_beside_an_eager_one(ex):
    """Forward and backward of a block captured into a graph and replayed with other inputs, while an eager pass's tensors live."""
    from paper_2404_00438_b200 import layers
    dev = torch.device("cuda:0")
    model = ex.Decoder(words=100, width=128, hidden=256, blocks=1, heads=2, kv_heads=1)
    p = model.views(model.initial(dev).to(torch.bfloat16))
    x = torch.randn(300, 128, device=dev).to(torch.bfloat16)
    targets = torch.arange(300, device=dev) % 100
    offsets = torch.tensor([0, 120, 300], device=dev)
    eager, captured = torch.zeros(model.d_pad, device=dev), torch.zeros(model.d_pad, device=dev)
    first = model.loss_and_gradients(p, model.views(eager), x, targets, offsets)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss = model.loss_and_gradients(p, model.views(captured), x, targets, offsets)
    for seed in (3, 4):
        x.copy_(torch.randn(300, 128, generator=torch.Generator(device=dev).manual_seed(seed), device=dev))
        offsets.copy_(torch.tensor([0, 60 * seed, 300], device=dev))
        graph.replay()
        again = model.loss_and_gradients(p, model.views(eager), x, targets, offsets)
        torch.cuda.synchronize()
        assert torch.equal(loss, again) and torch.equal(captured, eager)
    assert float(first) > 0
    layers.check()
