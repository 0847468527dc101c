"""Host-side checks of the layer operators that need no GPU: the header, the exports and the binding's
structures agree, and malformed arguments are refused before CUDA is touched."""
import ctypes
import os
import re

import pytest
import torch

from paper_2404_00438_b200 import build as dl_build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20      # an aligned address that is never read


@pytest.fixture(scope="module")
def layers():
    dl_build.build()
    from paper_2404_00438_b200 import layers
    return layers


def header():
    return open(os.path.join(ROOT, "include", "dlion_layers.h")).read()


def test_exports_match_header(layers):
    declared = set(re.findall(r"^(?:uint64_t|dlion_status) (dlion_[a-z0-9_]+)\s*\(", header(), re.M))
    assert declared == set(layers.EXPORTS)
    raw = ctypes.CDLL(dl_build.LIB)
    for name in declared:
        assert hasattr(raw, name)


@pytest.mark.parametrize("struct,cls", [("dlion_linear_fwd", "_Forward"), ("dlion_linear_bwd", "_Backward"), ("dlion_loss", "_Loss")])
def test_structures_match_header(layers, struct, cls):
    body = re.search(r"typedef struct \{([^}]*)\} %s;" % struct, header()).group(1)
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    fields = []
    for decl in body.split(";"):
        decl = decl.replace("const", "").strip()
        if decl:
            kind = decl.split()[0]
            kind = "ptr" if "*" in decl else kind
            fields += [(n.strip(" *"), kind) for n in decl.replace("*", " ").split(None, 1)[1].split(",")]
    want = {"ptr": ctypes.c_void_p, "int64_t": ctypes.c_int64, "int32_t": ctypes.c_int32, "float": ctypes.c_float}
    assert [(n, want[k]) for n, k in fields] == list(getattr(layers, cls)._fields_)


def forward_args(layers, **kw):
    a = dict(m=4, k=8, n=16, x=P, x_rs=8, x_cs=1, w=P, w_rs=16, w_cs=1, y=P, y_ld=16, y_type=1)
    a.update(kw)
    return layers._Forward(**a)


@pytest.mark.parametrize("kw,status", [
    (dict(m=-1), 1), (dict(k=0), 1), (dict(n=0), 1), (dict(m=(1 << 30) + 1), 1), (dict(x=None), 1), (dict(w=None), 1),
    (dict(y=None), 1), (dict(act=4), 1), (dict(act=-1), 1), (dict(keep=3), 1), (dict(y_type=2), 1), (dict(y_ld=15), 1),
    (dict(x_rs=-8), 1), (dict(bias=P, bias_type=7), 1), (dict(residual=P, r_ld=3), 1), (dict(keep=2, kept=P, kept_ld=16), 1),
    (dict(keep=2, kept=P, kept_ld=16, kept_e_ld=4), 1), (dict(keep=1, kept_ld=16), 1), (dict(x=P + 1), 2), (dict(y=P + 2, y_type=0), 2),
])
def test_forward_refusals(layers, kw, status):
    lib, a = layers._lib, forward_args(layers, **kw)
    assert lib.dlion_linear_forward(ctypes.byref(a), P, 1 << 40, None) == status
    assert lib.dlion_linear_forward_workspace(ctypes.byref(a)) == 0


def test_null_structures_and_workspaces(layers):
    lib = layers._lib
    assert lib.dlion_linear_forward(None, P, 0, None) == 1
    assert lib.dlion_linear_backward(None, P, 0, None) == 1
    assert lib.dlion_lm_loss(None, P, 0, None) == 1
    a = forward_args(layers, x_rs=9, k=8)                 # rows off the 16-byte grid: packed into the workspace
    need = lib.dlion_linear_forward_workspace(ctypes.byref(a))
    assert need >= 4 * 8 * 2
    assert lib.dlion_linear_forward(ctypes.byref(a), P, need - 1, None) == 1
    assert lib.dlion_linear_forward(ctypes.byref(a), None, need, None) == 1
    assert lib.dlion_linear_forward(ctypes.byref(a), P + 8, need, None) == 2


@pytest.mark.parametrize("kw,status", [
    (dict(saved=0), 1), (dict(saved=3), 1), (dict(dy=None), 1), (dict(u=None), 1), (dict(dw_rs=15), 1), (dict(dw_rs=4, dw_cs=4), 1),
    (dict(grad_type=2), 1), (dict(dx_ld=7), 1), (dict(w=None), 1), (dict(saved=2, u_e=None), 1), (dict(dw=P + 2, grad_type=0), 2),
    (dict(db=P + 1), 2),
])
def test_backward_refusals(layers, kw, status):
    a = dict(m=4, k=8, n=16, dy=P, dy_rs=16, dy_cs=1, w=P, w_rs=16, w_cs=1, saved=1, u=P, u_ld=8, u_e_ld=4, dx=P, dx_ld=8, dw=P,
             dw_rs=16, dw_cs=1, db=P, grad_type=1)
    a.update(kw)
    assert layers._lib.dlion_linear_backward(ctypes.byref(layers._Backward(**a)), P, 1 << 40, None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(h=0), 1), (dict(v=0), 1), (dict(m=-1), 1), (dict(dx=None), 1), (dict(loss=None), 1), (dict(rows=None), 1),
    (dict(targets=None), 1), (dict(mean=2), 1), (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1), (dict(piece=-1), 1),
    (dict(dw_ld=7), 1), (dict(grad_type=5), 1), (dict(targets=P + 4), 2), (dict(loss=P + 2), 2),
])
def test_loss_refusals(layers, kw, status):
    a = dict(m=4, h=8, v=16, x=P, x_rs=8, x_cs=1, w=P, w_rs=8, w_cs=1, targets=P, ignore_index=-100, mean=1, scale=1.0, loss=P,
             rows=P, dx=P, dx_ld=8, dw=P, dw_ld=8, grad_type=1)
    a.update(kw)
    assert layers._lib.dlion_lm_loss(ctypes.byref(layers._Loss(**a)), P, 1 << 40, None) == status


def test_checkpoint_refusals(layers):
    lib = layers._lib
    assert lib.dlion_checkpoint8(P, 7, 4, 8, P, 8, P, 4, None) == 1
    assert lib.dlion_checkpoint8(P, 8, 4, 8, P, 8, P, 3, None) == 1 or lib.dlion_checkpoint8(P, 8, 4, 40, P, 40, P, 3, None) == 1
    assert lib.dlion_checkpoint8(None, 8, 4, 8, P, 8, P, 4, None) == 1
    assert lib.dlion_checkpoint8(P + 1, 8, 4, 8, P, 8, P, 4, None) == 2
    assert lib.dlion_restore8(P, 8, P, 4, 4, 0, P, 8, None) == 1
    assert lib.dlion_restore8(P, 8, None, 4, 4, 8, P, 8, None) == 1
    assert lib.dlion_checkpoint8(None, 8, 0, 8, None, 8, None, 0, None) == 0       # no rows: nothing to do


def test_host_tensors_never_reach_the_library(layers):
    x, w = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(8, 16, dtype=torch.bfloat16)
    for call in (lambda: layers.linear_forward(x, w), lambda: layers.linear_backward(torch.zeros(4, 16, dtype=torch.bfloat16), w, x),
                 lambda: layers.checkpoint8(x), lambda: layers.lm_loss(x, w.t(), torch.zeros(4, dtype=torch.int64)),
                 lambda: layers.restore8(layers.Checkpoint8(torch.zeros(4, 8, dtype=torch.int8), torch.zeros(1, 4, dtype=torch.uint8)))):
        with pytest.raises(ValueError, match="CUDA tensor"):
            call()
    with pytest.raises(ValueError):
        layers.linear_forward([1.0], w)
    with pytest.raises(ValueError):
        layers.restore8(x)
