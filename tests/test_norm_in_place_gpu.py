"""Layer norm with results over inputs, in every form that a call may take: y over x, dx over dy, dx over the skip's gradient.
Each call gives the bits that it gives with results of its own, dw and db among them."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
DEV = "cuda:0"

# few and many rows; up to 768 columns, 2048, 8192, 16384, 32768 and beyond, on and off the 16-byte grid
SHAPES = [(45, 256), (3, 768), (700, 768), (5003, 768), (37, 1001), (4801, 1001), (5, 2048), (4750, 2047), (9, 4096), (1201, 4096), (1250, 4450), (3, 8192),
          (603, 8192), (5, 8199), (7, 8200), (301, 9001), (4, 9001), (9, 12289), (3, 14000), (300, 14000), (130, 16384), (2, 20000), (3, 32769), (70, 40000)]


@pytest.fixture(scope="module")
def L():
    assert torch.cuda.is_available(), "this test needs a CUDA device"
    from paper_2404_00438_b200 import build
    build.build()
    from paper_2404_00438_b200 import layers
    return layers


def normal(seed, *shape, std=1.0, mean=0.0, dtype=BF):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return (torch.randn(*shape, generator=g, device=DEV) * std + mean).to(dtype)


@pytest.mark.parametrize("m,n", SHAPES)
@pytest.mark.parametrize("stream", [BF, F32])
def test_forward(L, m, n, stream):
    x, w, b = normal(1, m, n, std=2.0, mean=0.5, dtype=stream), normal(2, n, std=0.3, mean=1.0), normal(3, n)
    y, stats = L.norm_forward(x, w, b, out_dtype=stream)
    over = x.clone()
    got = L.norm_forward(over, w, b, out=over)
    assert got.out is over and torch.equal(over, y) and torch.equal(got.stats, stats)


@pytest.mark.parametrize("m,n", SHAPES)
@pytest.mark.parametrize("stream", [BF, F32])
def test_backward(L, m, n, stream):
    x, w = normal(1, m, n, std=2.0, mean=0.5, dtype=stream), normal(2, n, std=0.3, mean=1.0)
    dy, r = normal(4, m, n, dtype=stream), normal(5, m, n, dtype=stream)
    _, stats = L.norm_forward(x, w)
    for skip in (None, r):
        want = L.norm_backward(dy, x, w, stats, residual=skip, grad_dtype=F32)
        over = dy.clone()
        got = L.norm_backward(over, x, w, stats, residual=skip, dx=over, grad_dtype=F32)
        assert got[0] is over
        for name, a, c in zip(("dx", "dw", "db"), got, want):
            assert torch.equal(a, c), f"dx over dy: {name}"
    over = r.clone()
    got = L.norm_backward(dy, x, w, stats, residual=over, dx=over, grad_dtype=F32)
    assert got[0] is over
    for name, a, c in zip(("dx", "dw", "db"), got, want):
        assert torch.equal(a, c), f"dx over the skip's gradient: {name}"
    for need in (dict(need_dw=False), dict(need_db=False)):       # one of the sums alone
        over = dy.clone()
        for a, c in zip(L.norm_backward(over, x, w, stats, residual=r, dx=over, grad_dtype=F32, **need), want):
            assert a is None or torch.equal(a, c)
