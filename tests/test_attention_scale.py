"""The ends of the attention's scale: scale times log2(e), by which the kernels multiply, is finite."""
import ctypes

import pytest
import torch

from paper_2404_00438_b200 import build as dl_build

P = 1 << 20      # an aligned address that is never read
BF = torch.bfloat16


@pytest.fixture(scope="module")
def L():
    dl_build.build()
    from paper_2404_00438_b200 import layers
    return layers


@pytest.mark.parametrize("scale", [2.1e38, 2.4e38, 3.3e38])
def test_refused(L, scale):
    """Before anything is launched, by the library and by its binding."""
    a = dict(rows=100, heads=4, kv_heads=4, dim=64, lse=P, lse_ld=100, causal=1, scale=scale)
    for t in ("q", "k", "v", "out", "dout", "dq", "dk", "dv"):
        a.update({t: P, t + "_rs": 256, t + "_hs": 64})
    forward = L._AttentionForward(**{n: a[n] for n, _ in L._AttentionForward._fields_ if n in a})
    backward = L._AttentionBackward(**{n: a[n] for n, _ in L._AttentionBackward._fields_ if n in a})
    assert L._lib.dlion_attention_forward(ctypes.byref(forward), P, 1 << 40, None) == 1
    assert L._lib.dlion_attention_backward(ctypes.byref(backward), P, 1 << 40, None) == 1
    with pytest.raises(ValueError, match="scale"):
        L._scale(scale, 64)


@pytest.mark.gpu
@pytest.mark.parametrize("dim", [64, 128])
def test_ends(L, dim):
    """Scores of 0, at any scale: every key's weight is the same.  At the smallest scale all scores are as good as 0: |q . k| is below
    300 here, a score below 3e-40, and a row of one key has it as its lse, where the others' is 0."""
    dev = "cuda:0"
    g = torch.Generator(device=dev)
    g.manual_seed(dim)
    q, k, v, do = (torch.randn(200, 2, dim, generator=g, device=dev).to(BF) for _ in range(4))
    zero = torch.zeros_like(q)
    want = L.attention_forward(zero, k, v, scale=1.0)
    wanted = L.attention_backward(do, zero, k, v, *want, scale=1.0)
    for query, scale in ((zero, 2e38), (zero, 1e-30), (q, 1e-42)):
        got = L.attention_forward(query, k, v, scale=scale)
        assert torch.equal(got.out, want.out) and float((got.lse - want.lse).abs().max()) <= (1e-39 if query is q else 0.0)
        assert torch.equal(L.attention_backward(do, query, k, v, *got, scale=scale)[2], wanted[2])
    L.check()
