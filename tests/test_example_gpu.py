"""The layer operators and the optimizer step together: the example's gradients against autograd in 64 bits, and
that it learns."""
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


def test_gradients_in_the_arena(ex):
    """Rounded operands (2^-9 each on average, some seven of them on the way to the first block) and 8-bit
    activations (about 2^-7 of an element, in the weights' gradients and in the slopes) leave each tensor's gradient
    within 5 % in the 2-norm; padding stays untouched."""
    dev = torch.device("cuda:0")
    model = ex.Model(words=700, width=96, hidden=200, blocks=2)
    x = model.initial(dev)
    for name, t in model.views(x).items():
        if t.dim() == 1:
            t.normal_(0, 0.1, generator=torch.Generator(device=dev).manual_seed(5))
    p = model.views(x.to(torch.bfloat16))
    inp = torch.randn(150, 96, generator=torch.Generator(device=dev).manual_seed(1), device=dev).to(torch.bfloat16)
    targets = torch.arange(150, device=dev) * 3
    for dtype in (torch.bfloat16, torch.float32):
        arena = torch.full((model.d_pad,), 3.0, dtype=dtype, device=dev)
        g = model.views(arena)
        loss = model.loss_and_gradients(p, g, inp, targets)
        q = {k: v.to(F64).requires_grad_() for k, v in p.items()}
        h = inp.to(F64)
        for i in range(2):
            z = torch.nn.functional.gelu(h @ q[f"w1.{i}"] + q[f"b1.{i}"], approximate="tanh")
            h = z @ q[f"w2.{i}"] + q[f"b2.{i}"] + h
        want = torch.nn.functional.cross_entropy(h @ q["head"].t(), targets)
        want.backward()
        assert abs(float(loss) - float(want.detach())) <= 0.01 * float(want.detach())
        for name in g:
            rel = float((g[name].to(F64) - q[name].grad).norm() / q[name].grad.norm())
            assert rel <= 0.05, (name, rel)
        mask = torch.ones(model.d_pad, dtype=torch.bool, device=dev)
        for o, n in model.segments:
            mask[o:o + n] = False
        assert bool((arena[mask] == 3.0).all())


def test_it_learns(ex):
    losses = ex.train(steps=40, workers=3, rows=256, words=200, width=128, hidden=256, blocks=1, report=lambda s: None)
    assert all(math.isfinite(v) for v in losses)
    assert losses[0] > 0.8 * math.log(200) and losses[-1] < 0.5 * losses[0]
