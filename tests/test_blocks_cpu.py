"""Host-side checks of the norm and the attention that need no GPU: structures agree with the header, and malformed arguments are
refused before CUDA is touched."""
import ctypes
import os
import re

import pytest
import torch

from paper_2404_00438_b200 import build as dl_build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20      # an aligned address that is never read
BF = torch.bfloat16


@pytest.fixture(scope="module")
def layers():
    dl_build.build()
    from paper_2404_00438_b200 import layers
    return layers


@pytest.mark.parametrize("struct,cls", [("dlion_norm_fwd", "_NormForward"), ("dlion_norm_bwd", "_NormBackward"),
                                        ("dlion_attention_fwd", "_AttentionForward"), ("dlion_attention_bwd", "_AttentionBackward")])
def test_structures_match_header(layers, struct, cls):
    header = open(os.path.join(ROOT, "include", "dlion_layers.h")).read()
    body = re.sub(r"/\*.*?\*/", "", re.search(r"typedef struct \{([^}]*)\} %s;" % struct, header).group(1), flags=re.S)
    fields = []
    for decl in body.split(";"):
        decl = decl.replace("const", "").strip()
        if decl:
            kind = "ptr" if "*" in decl else decl.split()[0]
            fields += [(n.strip(" *"), kind) for n in decl.replace("*", " ").split(None, 1)[1].split(",")]
    want = {"ptr": ctypes.c_void_p, "int64_t": ctypes.c_int64, "int32_t": ctypes.c_int32, "float": ctypes.c_float}
    assert [(n, want[k]) for n, k in fields] == list(getattr(layers, cls)._fields_)


@pytest.mark.parametrize("kw,status", [
    (dict(m=-1), 1), (dict(n=0), 1), (dict(m=(1 << 30) + 1), 1), (dict(x=None), 1), (dict(y=None), 1), (dict(stats=None), 1), (dict(x_type=2), 1),
    (dict(y_type=-1), 1), (dict(w_type=3), 1), (dict(b=P, b_type=9), 1), (dict(x_ld=15), 1), (dict(y_ld=-1), 1), (dict(eps=-1.0), 1),
    (dict(eps=float("nan")), 1), (dict(eps=float("inf")), 1), (dict(x=P + 1), 2), (dict(y=P + 2), 2), (dict(stats=P + 2), 2), (dict(w=P + 1), 2),
])
def test_norm_forward_refusals(layers, kw, status):
    a = dict(m=4, n=16, x=P, x_ld=16, x_type=1, w=P, w_type=1, eps=1e-5, y=P, y_ld=16, y_type=0, stats=P)
    a.update(kw)
    assert layers._lib.dlion_norm_forward(ctypes.byref(layers._NormForward(**a)), None) == status
    assert layers._lib.dlion_norm_forward(None, None) == 1


@pytest.mark.parametrize("kw,status", [
    (dict(m=-1), 1), (dict(n=0), 1), (dict(dy=None), 1), (dict(x=None), 1), (dict(stats=None), 1), (dict(dy_type=2), 1), (dict(x_type=2), 1),
    (dict(grad_type=2), 1), (dict(dy_ld=15), 1), (dict(x_ld=3), 1), (dict(dx_ld=7), 1), (dict(residual=P, r_ld=3), 1), (dict(dw=P + 2), 2),
    (dict(db=P + 1), 2), (dict(dx=P + 1), 2), (dict(stats=P + 1), 2), (dict(dy=P + 1), 2),
])
def test_norm_backward_refusals(layers, kw, status):
    a = dict(m=4, n=16, dy=P, dy_ld=16, dy_type=1, x=P, x_ld=16, x_type=1, w=P, w_type=1, stats=P, dx=P, dx_ld=16, dw=P, db=P, grad_type=0)
    a.update(kw)
    ref = ctypes.byref(layers._NormBackward(**a))
    assert layers._lib.dlion_norm_backward(ref, P, 1 << 40, None) == status
    assert layers._lib.dlion_norm_backward_workspace(ref) == 0
    assert layers._lib.dlion_norm_backward(None, P, 1 << 40, None) == 1


def test_norm_workspace(layers):
    a = layers._NormBackward(m=4000, n=16, dy=P, dy_ld=16, dy_type=1, x=P, x_ld=16, x_type=1, stats=P, dx=P, dx_ld=16, dw=P, grad_type=0)
    need = layers._lib.dlion_norm_backward_workspace(ctypes.byref(a))
    assert need > 0
    assert layers._lib.dlion_norm_backward(ctypes.byref(a), P, need - 1, None) == 1
    assert layers._lib.dlion_norm_backward(ctypes.byref(a), None, need, None) == 1
    assert layers._lib.dlion_norm_backward(ctypes.byref(a), P + 8, need, None) == 2


def attention(layers, backward, **kw):
    a = dict(rows=100, heads=4, kv_heads=2, dim=64, lse=P, lse_ld=100, causal=1, scale=0.125)
    for t, h in (("q", 4), ("k", 2), ("v", 2), ("out", 4)) + ((("dout", 4), ("dq", 4), ("dk", 2), ("dv", 2)) if backward else ()):
        a.update({t: P, t + "_rs": 64 * h, t + "_hs": 64})
    a.update(kw)
    cls, name = (layers._AttentionBackward, "dlion_attention_backward") if backward else (layers._AttentionForward, "dlion_attention_forward")
    return cls(**a), getattr(layers._lib, name), getattr(layers._lib, name + "_workspace")


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), 1), (dict(rows=(1 << 30) + 1), 1), (dict(heads=0), 1), (dict(kv_heads=0), 1), (dict(kv_heads=3), 1), (dict(heads=65538), 1),
    (dict(dim=0), 1), (dict(dim=12), 1), (dict(dim=136), 1), (dict(causal=2), 1), (dict(scale=0.0), 1), (dict(scale=-1.0), 1),
    (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1), (dict(length=7), 1), (dict(length=-1), 1), (dict(sequences=3), 1),
    (dict(offsets=P, sequences=-1), 1), (dict(offsets=P, sequences=2, length=100), 1), (dict(offsets=P, sequences=2, offsets_64=2), 1),
    (dict(offsets=P + 4, sequences=2, offsets_64=1), 2), (dict(offsets=P + 2, sequences=2), 2), (dict(lse_ld=99), 1), (dict(lse=None), 1), (dict(lse=P + 2), 2),
    (dict(zero_rest=2), 1), (dict(q=None), 1), (dict(k=None), 1), (dict(out=None), 1), (dict(q_rs=252), 1), (dict(k_hs=60), 1), (dict(v_rs=56), 1),
    (dict(out_hs=0), 1), (dict(q=P + 8), 2), (dict(out=P + 2), 2),
])
def test_attention_refusals(layers, kw, status, backward):
    a, call, size = attention(layers, backward, **kw)
    assert call(ctypes.byref(a), P, 1 << 40, None) == status
    assert size(ctypes.byref(a)) == 0
    assert call(None, P, 0, None) == 1


@pytest.mark.parametrize("kw,status", [(dict(dout=None), 1), (dict(dq=None), 1), (dict(dk_rs=100), 1), (dict(dv_hs=4), 1), (dict(dq=P + 8), 2)])
def test_attention_backward_refusals(layers, kw, status):
    a, call, _ = attention(layers, True, **kw)
    assert call(ctypes.byref(a), P, 1 << 40, None) == status


@pytest.mark.parametrize("backward", [False, True])
def test_attention_workspace(layers, backward):
    a, call, size = attention(layers, backward, offsets=P, sequences=9)
    need = size(ctypes.byref(a))
    assert need > 0
    assert call(ctypes.byref(a), P, need - 1, None) == 1
    assert call(ctypes.byref(a), P + 8, need, None) == 2
    a, _, size = attention(layers, backward, offsets=P, sequences=1 << 20)       # no more pieces than rows
    assert size(ctypes.byref(a)) <= (100 * 16 + 256) * 2 + 4 * 400 + 256


def test_host_tensors_never_reach_the_library(layers):
    x, stats = torch.zeros(4, 8, dtype=BF), torch.zeros(2, 4)
    q = torch.zeros(4, 2, 64, dtype=BF)
    for call in (lambda: layers.norm_forward(x), lambda: layers.norm_backward(x, x, None, stats), lambda: layers.attention_forward(q, q, q),
                 lambda: layers.attention_backward(q, q, q, q, q, torch.zeros(2, 4))):
        with pytest.raises(ValueError, match="CUDA tensor"):
            call()
    with pytest.raises(ValueError):
        layers.norm_forward([1.0])
    with pytest.raises(ValueError):
        layers.attention_forward(None, q, q)
