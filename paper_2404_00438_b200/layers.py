"""Layer operators that make the gradients the optimizer step consumes: binding over the C ABI
declared in ``include/dlion_layers.h``.

    y, z8 = linear_forward(x, w, bias, act="gelu", keep="8bit")    # y = act(x w + bias), z kept in 8 bits
    du, dw, db = linear_backward(dy, w2, z8, act="gelu")           # gradients of y2 = act(z) w2 + b2
    x8 = checkpoint8(x); x = restore8(x8)                          # a 33/64 of bf16's bytes
    r = lm_loss(x, w, targets)                                     # r.loss, r.rows, r.dx, r.dw
    y, stats = norm_forward(x, w, b)                               # layer norm
    dx, dw, db = norm_backward(dy, x, w, stats, residual=r)        # its gradients, the skip's added
    out, lse = attention_forward(q, k, v, offsets=offsets)         # of packed sequences
    dq, dk, dv = attention_backward(dout, q, k, v, out, lse, offsets=offsets)

Argument marshalling only, as in ``dlion``: every tensor is checked, becomes a device address, and the
current torch stream becomes the ``cudaStream_t``.  Outputs may be given (``out=``, ``dw=``, ...): a view
into the optimizer's gradient arena is a valid ``dw`` or ``db``.  The workspace comes from torch's
allocator on the current stream unless one is given.  There is no CPU path, and no autograd: tensors that require
gradients are read like any others and results have no graph; the gradients are what the ``_backward`` calls and
``lm_loss`` return.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional, Tuple, Union

import torch

from . import dlion as _dlion
from .dlion import DlionError, GRAD_BF16, GRAD_F32, OK

ACTS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
KEEP_NONE, KEEP_BF16, KEEP_8BIT = 0, 1, 2
KEEPS = {None: KEEP_NONE, "bf16": KEEP_BF16, "8bit": KEEP_8BIT}
BLOCK8 = 32
_TYPES = {torch.float32: GRAD_F32, torch.bfloat16: GRAD_BF16}
_BF16 = torch.bfloat16

EXPORTS = ("dlion_linear_forward_workspace", "dlion_linear_backward_workspace", "dlion_lm_loss_workspace",
           "dlion_linear_forward", "dlion_linear_backward", "dlion_lm_loss", "dlion_checkpoint8",
           "dlion_restore8", "dlion_norm_forward", "dlion_norm_backward_workspace", "dlion_norm_backward",
           "dlion_attention_forward_workspace", "dlion_attention_forward", "dlion_attention_backward_workspace",
           "dlion_attention_backward", "dlion_layers_check")

_i64, _i32, _vp, _f32 = ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p, ctypes.c_float


class _Forward(ctypes.Structure):
    _fields_ = [("m", _i64), ("k", _i64), ("n", _i64), ("x", _vp), ("x_rs", _i64), ("x_cs", _i64),
                ("w", _vp), ("w_rs", _i64), ("w_cs", _i64), ("bias", _vp), ("bias_type", _i32), ("act", _i32),
                ("residual", _vp), ("r_ld", _i64), ("y", _vp), ("y_ld", _i64), ("y_type", _i32), ("keep", _i32),
                ("kept", _vp), ("kept_ld", _i64), ("kept_e", _vp), ("kept_e_ld", _i64)]


class _Backward(ctypes.Structure):
    _fields_ = [("m", _i64), ("k", _i64), ("n", _i64), ("dy", _vp), ("dy_rs", _i64), ("dy_cs", _i64),
                ("w", _vp), ("w_rs", _i64), ("w_cs", _i64), ("act", _i32), ("saved", _i32),
                ("u", _vp), ("u_ld", _i64), ("u_e", _vp), ("u_e_ld", _i64), ("residual", _vp), ("r_ld", _i64),
                ("dx", _vp), ("dx_ld", _i64), ("dw", _vp), ("dw_rs", _i64), ("dw_cs", _i64), ("db", _vp),
                ("grad_type", _i32)]


class _Loss(ctypes.Structure):
    _fields_ = [("m", _i64), ("h", _i64), ("v", _i64), ("x", _vp), ("x_rs", _i64), ("x_cs", _i64),
                ("w", _vp), ("w_rs", _i64), ("w_cs", _i64), ("targets", _vp), ("ignore_index", _i64),
                ("mean", _i32), ("scale", _f32), ("loss", _vp), ("rows", _vp), ("dx", _vp), ("dx_ld", _i64),
                ("dw", _vp), ("dw_ld", _i64), ("grad_type", _i32), ("piece", _i64)]


class _NormForward(ctypes.Structure):
    _fields_ = [("m", _i64), ("n", _i64), ("x", _vp), ("x_ld", _i64), ("x_type", _i32), ("w", _vp), ("w_type", _i32),
                ("b", _vp), ("b_type", _i32), ("eps", _f32), ("y", _vp), ("y_ld", _i64), ("y_type", _i32), ("stats", _vp)]


class _NormBackward(ctypes.Structure):
    _fields_ = [("m", _i64), ("n", _i64), ("dy", _vp), ("dy_ld", _i64), ("dy_type", _i32), ("x", _vp), ("x_ld", _i64),
                ("x_type", _i32), ("w", _vp), ("w_type", _i32), ("stats", _vp), ("residual", _vp), ("r_ld", _i64),
                ("dx", _vp), ("dx_ld", _i64), ("dw", _vp), ("db", _vp), ("grad_type", _i32)]


def _strided(*names):
    return [f for n in names for f in ((n, _vp), (n + "_rs", _i64), (n + "_hs", _i64))]


_ATTENTION_SIZES = [("rows", _i64), ("heads", _i64), ("kv_heads", _i64), ("dim", _i64)]
_ATTENTION_SEQUENCES = [("offsets", _vp), ("offsets_64", _i32), ("sequences", _i64), ("length", _i64), ("causal", _i32), ("scale", _f32)]


class _AttentionForward(ctypes.Structure):
    _fields_ = (_ATTENTION_SIZES + _strided("q", "k", "v") + _ATTENTION_SEQUENCES + _strided("out")
                + [("lse", _vp), ("lse_ld", _i64), ("zero_rest", _i32)])


class _AttentionBackward(ctypes.Structure):
    _fields_ = (_ATTENTION_SIZES + _strided("q", "k", "v", "out", "dout") + [("lse", _vp), ("lse_ld", _i64)] + _ATTENTION_SEQUENCES
                + _strided("dq", "dk", "dv") + [("zero_rest", _i32)])


def _bind(lib):
    for name, struct in (("dlion_linear_forward", _Forward), ("dlion_linear_backward", _Backward), ("dlion_lm_loss", _Loss),
                         ("dlion_norm_backward", _NormBackward), ("dlion_attention_forward", _AttentionForward),
                         ("dlion_attention_backward", _AttentionBackward)):
        size, call = getattr(lib, name + "_workspace"), getattr(lib, name)
        size.argtypes, size.restype = [ctypes.POINTER(struct)], ctypes.c_uint64
        call.argtypes, call.restype = [ctypes.POINTER(struct), _vp, ctypes.c_uint64, _vp], ctypes.c_int
    lib.dlion_norm_forward.argtypes, lib.dlion_norm_forward.restype = [ctypes.POINTER(_NormForward), _vp], ctypes.c_int
    lib.dlion_checkpoint8.argtypes = [_vp, _i64, _i64, _i64, _vp, _i64, _vp, _i64, _vp]
    lib.dlion_checkpoint8.restype = ctypes.c_int
    lib.dlion_restore8.argtypes = [_vp, _i64, _vp, _i64, _i64, _i64, _vp, _i64, _vp]
    lib.dlion_restore8.restype = ctypes.c_int
    lib.dlion_layers_check.argtypes = [_vp]
    lib.dlion_layers_check.restype = ctypes.c_int
    return lib


_lib = _bind(_dlion.lib())

# the current stream's handle and device without the objects and checks around them, where torch offers that
_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda device: torch.cuda.current_stream(device).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_Tensor, _empty = torch.Tensor, torch.empty
_FORWARD = (_lib.dlion_linear_forward_workspace, _lib.dlion_linear_forward)
_BACKWARD = (_lib.dlion_linear_backward_workspace, _lib.dlion_linear_backward)
_LOSS = (_lib.dlion_lm_loss_workspace, _lib.dlion_lm_loss)
_NORM_BACKWARD = (_lib.dlion_norm_backward_workspace, _lib.dlion_norm_backward)
_ATTENTION_FORWARD = (_lib.dlion_attention_forward_workspace, _lib.dlion_attention_forward)
_ATTENTION_BACKWARD = (_lib.dlion_attention_backward_workspace, _lib.dlion_attention_backward)
_ONLY_BF16 = (_BF16,)


class Checkpoint8(NamedTuple):
    """A matrix in 8 bits: value = q * 2^(e - 127), ``e`` shared by 32 values of a row ([ceil(k/32), m])."""
    q: torch.Tensor
    e: torch.Tensor


class Normed(NamedTuple):
    out: torch.Tensor
    stats: torch.Tensor                # float32 [2, m]: the rows' means, then 1 / sqrt(var + eps)


class Attended(NamedTuple):
    out: torch.Tensor                  # bf16 [rows, heads, dim]
    lse: torch.Tensor                  # float32 [heads, rows]: log of the sum of the scores' exponentials


class Loss(NamedTuple):
    loss: torch.Tensor                 # float32 scalar
    rows: torch.Tensor                 # float32 [m]
    dx: Optional[torch.Tensor]
    dw: Optional[torch.Tensor]


def _device(t, name: str) -> int:
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name}: expected a torch.Tensor, got {type(t).__name__}")
    index = t.get_device()
    if index < 0:
        raise ValueError(f"{name}: must be a CUDA tensor (the library has no CPU path)")
    if index != _current_device():
        raise ValueError(f"{name}: is on cuda:{index}, the current device is cuda:{_current_device()}")
    return index


# The checks run on every call, and a small product takes a few microseconds: each is one expression while all is well,
# and _refused finds the words.
def _matrix(t, name: str, device: int, dtypes, shape, adjacent: bool = False) -> None:
    """Raises unless ``t`` is a tensor of ``shape`` and of one of ``dtypes`` on ``device`` (``adjacent``: with
    adjacent columns and rows that do not overlap)."""
    if not (isinstance(t, _Tensor) and t.dtype in dtypes and t.shape == shape and t.get_device() == device):
        _refused(t, name, device, dtypes, shape)
    if adjacent and not t.is_contiguous():
        rs, cs = t.stride()
        if (cs != 1 and shape[1] != 1) or (shape[0] > 1 and rs < shape[1]):
            raise ValueError(f"{name}: needs adjacent columns (got strides {(rs, cs)})")


def _vector(t, name: str, device: int, dtypes, n: int) -> None:
    if not (isinstance(t, _Tensor) and t.dtype in dtypes and t.shape == (n,) and t.get_device() == device):
        _refused(t, name, device, dtypes, (n,))
    if not t.is_contiguous():
        raise ValueError(f"{name}: expected {n} adjacent values, got strides {t.stride()}")


def _refused(t, name: str, device: int, dtypes, shape) -> None:
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name}: expected a torch.Tensor, got {type(t).__name__}")
    if t.get_device() != device:
        raise ValueError(f"{name}: is on {t.device}, the call is on cuda:{device}")
    if t.dtype not in dtypes:
        raise ValueError(f"{name}: dtype {t.dtype}, expected one of {tuple(dtypes)}")
    raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")


def _two_dim(t, name: str) -> Tuple[int, int]:
    shape = t.shape
    if len(shape) != 2:
        raise ValueError(f"{name}: expected a matrix, got {t.dim()} dimensions")
    return shape


def _enumerator(table, value, name: str) -> int:
    try:
        return table[value]
    except (KeyError, TypeError):
        raise ValueError(f"{name}: {value!r}, expected one of {tuple(table)}") from None


def _grad_type(dtype) -> int:
    return _enumerator(_TYPES, dtype, "grad_dtype")


# an empty tensor on each device: its new_empty(n) takes 1.4 us, torch.empty(n, dtype=, device=) 2.3
_bytes = {}


def _space(need: int, device: int) -> torch.Tensor:
    none = _bytes.get(device)
    if none is None:
        none = _bytes[device] = _empty(0, dtype=torch.uint8, device=device)
    return none.new_empty(need)


def _call(calls, args, device: int, workspace: Optional[torch.Tensor]) -> None:
    size, call = calls
    ref = ctypes.byref(args)
    need = size(ref)
    if workspace is None:
        if need:
            workspace = _space(need, device)
    else:
        _dlion.check_tensor(workspace, "workspace", (torch.uint8,), need, device)
    st = call(ref, workspace.data_ptr() if need else None, need, _stream(device))
    if st != OK:
        raise DlionError(st, call.__name__)


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def linear_forward(x: torch.Tensor, w: torch.Tensor, bias: Optional[torch.Tensor] = None, *, act: str = "none",
                   residual: Optional[torch.Tensor] = None, keep: Optional[str] = None,
                   out: Optional[torch.Tensor] = None, out_dtype: torch.dtype = torch.bfloat16,
                   workspace: Optional[torch.Tensor] = None):
    """``y = act(x w + bias) + residual``: ``x`` [m, k] and ``w`` [k, n] bf16 of any strides (a weight stored
    [n, k] is passed as its ``.t()``), ``bias`` [n] bf16 or fp32, ``residual`` [m, n] bf16.  ``keep`` = "bf16" or
    "8bit" also returns what is needed of z = x w + bias for the backward pass of the NEXT product."""
    device = _device(x, "x")
    m, k = _two_dim(x, "x")
    n = _two_dim(w, "w")[1]
    _matrix(x, "x", device, _ONLY_BF16, (m, k))
    _matrix(w, "w", device, _ONLY_BF16, (k, n))
    if bias is not None:
        _vector(bias, "bias", device, _TYPES, n)
    if residual is not None:
        _matrix(residual, "residual", device, _ONLY_BF16, (m, n), True)
    a, how = _enumerator(ACTS, act, "act"), _enumerator(KEEPS, keep, "keep")
    if out is None:
        if out_dtype not in _TYPES:
            raise ValueError(f"out_dtype: {out_dtype}, expected one of {tuple(_TYPES)}")
        out = x.new_empty((m, n)) if out_dtype is _BF16 else x.new_empty((m, n), dtype=out_dtype)
    else:
        _matrix(out, "out", device, _TYPES, (m, n), True)
    kept = None
    q = e = None
    if how == KEEP_8BIT:
        kept = Checkpoint8(x.new_empty((m, n), dtype=torch.int8),
                           x.new_empty((-(-n // BLOCK8), m), dtype=torch.uint8))
        q, e = kept
    elif how == KEEP_BF16:
        q = kept = x.new_empty((m, n))
    xs, ws = x.stride(), w.stride()
    args = _Forward(m, k, n, x.data_ptr(), xs[0], xs[1], w.data_ptr(), ws[0], ws[1], _ptr(bias),
                    0 if bias is None else _TYPES[bias.dtype], a, _ptr(residual),
                    0 if residual is None else residual.stride(0), out.data_ptr(), out.stride(0), _TYPES[out.dtype],
                    how, _ptr(q), n, _ptr(e), m)
    _call(_FORWARD, args, device, workspace)
    return out if kept is None else (out, kept)


def linear_backward(dy: torch.Tensor, w: torch.Tensor, saved: Union[torch.Tensor, Checkpoint8, None], *, act: str = "none",
                    residual: Optional[torch.Tensor] = None, need_dx: bool = True, need_dw: bool = True,
                    need_db: bool = True, grad_dtype: torch.dtype = torch.bfloat16,
                    dx: Optional[torch.Tensor] = None, dw: Optional[torch.Tensor] = None,
                    db: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """Gradients of ``y = act(u) w + b``: ``du = (dy wᵀ) act'(u) + residual`` (bf16 [m, k]),
    ``dw = act(u)ᵀ dy`` ([k, n], in ``w``'s own order when it is not given) and ``db = Σ dy`` ([n]) in
    ``grad_dtype``.  ``saved`` is u: a bf16 [m, k] tensor or a :class:`Checkpoint8`.  With ``act`` = "none" u is
    the layer's input itself.  Returns (du, dw, db), None for what is not needed."""
    device = _device(dy, "dy")
    m, n = _two_dim(dy, "dy")
    k = _two_dim(w, "w")[0]
    _matrix(dy, "dy", device, _ONLY_BF16, (m, n))
    _matrix(w, "w", device, _ONLY_BF16, (k, n))
    a = _enumerator(ACTS, act, "act")
    u = e = None
    u_ld = e_ld = 0
    how = KEEP_BF16
    if isinstance(saved, Checkpoint8):
        how = KEEP_8BIT
        u, e = saved
        _checkpoint(saved, "saved", device, m, k)
        u_ld, e_ld = u.stride(0), e.stride(0)
    elif saved is not None:
        u = saved
        _matrix(u, "saved", device, _ONLY_BF16, (m, k), True)
        u_ld = u.stride(0)
    elif need_dw or (need_dx and a):
        raise ValueError("saved: needed for dw, and for dx behind an activation")
    if residual is not None:
        _matrix(residual, "residual", device, _ONLY_BF16, (m, k), True)
    g = _grad_type(grad_dtype)
    ys, ws = dy.stride(), w.stride()
    gs = (n, 1) if ws[0] >= ws[1] else (1, k)       # of a dw that is not given (or not wanted: dx's bits are the same then)
    if not need_dx:
        dx = None
    elif dx is None:
        dx = dy.new_empty((m, k))
    else:
        _matrix(dx, "dx", device, _ONLY_BF16, (m, k), True)
    if not need_dw:
        dw = None
    elif dw is None:
        dw = dy.new_empty((k, n), dtype=grad_dtype) if ws[0] >= ws[1] else dy.new_empty((n, k), dtype=grad_dtype).t()
    else:
        _matrix(dw, "dw", device, (grad_dtype,), (k, n))
        gs = dw.stride()
        if not ((gs[1] == 1 and (k == 1 or gs[0] >= n)) or (gs[0] == 1 and (n == 1 or gs[1] >= k))):
            raise ValueError(f"dw: needs adjacent rows or columns (got strides {gs})")
    if not need_db:
        db = None
    elif db is None:
        db = dy.new_empty((n,), dtype=grad_dtype)
    else:
        _vector(db, "db", device, (grad_dtype,), n)
    args = _Backward(m, k, n, dy.data_ptr(), ys[0], ys[1], w.data_ptr(), ws[0], ws[1], a, how, _ptr(u), u_ld, _ptr(e), e_ld,
                     _ptr(residual), 0 if residual is None else residual.stride(0), _ptr(dx),
                     0 if dx is None else dx.stride(0), _ptr(dw), gs[0], gs[1], _ptr(db), g)
    _call(_BACKWARD, args, device, workspace)
    return dx, dw, db


def _checkpoint(c: Checkpoint8, name: str, device: int, m: int, k: int) -> None:
    _matrix(c.q, name + ".q", device, (torch.int8,), (m, k), True)
    _matrix(c.e, name + ".e", device, (torch.uint8,), (-(-k // BLOCK8), m), True)


def checkpoint8(x: torch.Tensor, out: Optional[Checkpoint8] = None) -> Checkpoint8:
    """``x`` (bf16 [m, k], adjacent columns) in the 8-bit form."""
    device = _device(x, "x")
    m, k = _two_dim(x, "x")
    _matrix(x, "x", device, _ONLY_BF16, (m, k), True)
    if out is None:
        q, e = x.new_empty((m, k), dtype=torch.int8), x.new_empty((-(-k // BLOCK8), m), dtype=torch.uint8)
        out, q_ld, e_ld = Checkpoint8(q, e), k, m
    else:
        _checkpoint(out, "out", device, m, k)
        q, e = out
        q_ld, e_ld = q.stride(0), e.stride(0)
    st = _lib.dlion_checkpoint8(x.data_ptr(), x.stride(0), m, k, q.data_ptr(), q_ld, e.data_ptr(), e_ld, _stream(device))
    if st != OK:
        raise DlionError(st, "dlion_checkpoint8")
    return out


def restore8(c: Checkpoint8, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The values of a :class:`Checkpoint8`, exact in bf16."""
    if not isinstance(c, Checkpoint8):
        raise ValueError(f"expected a Checkpoint8, got {type(c).__name__}")
    device = _device(c.q, "q")
    m, k = _two_dim(c.q, "q")
    _checkpoint(c, "c", device, m, k)
    if out is None:
        out, x_ld = c.q.new_empty((m, k), dtype=_BF16), k
    else:
        _matrix(out, "out", device, _ONLY_BF16, (m, k), True)
        x_ld = out.stride(0)
    st = _lib.dlion_restore8(c.q.data_ptr(), c.q.stride(0), c.e.data_ptr(), c.e.stride(0), m, k, out.data_ptr(), x_ld, _stream(device))
    if st != OK:
        raise DlionError(st, "dlion_restore8")
    return out


def lm_loss(x: torch.Tensor, w: torch.Tensor, targets: torch.Tensor, *, ignore_index: int = -100, reduction: str = "mean",
            scale: float = 1.0, grads: bool = True, grad_dtype: torch.dtype = torch.bfloat16,
            dx: Optional[torch.Tensor] = None, dw: Optional[torch.Tensor] = None, piece: int = 0,
            workspace: Optional[torch.Tensor] = None) -> Loss:
    """Softmax cross entropy of the logits ``x wᵀ`` (``x`` [m, h], ``w`` [v, h], both bf16) against ``targets``
    (int64 [m]) and its gradient, in one call and without keeping the logits: at most ``piece`` rows of them
    (4096 where 0) exist at a time, as 16-bit codes.  ``reduction`` is "mean" (over rows whose target is not
    ``ignore_index``) or "sum"; ``scale`` multiplies the gradients only.  Rows without a target have loss and
    gradient zero."""
    device = _device(x, "x")
    m, h = _two_dim(x, "x")
    v = _two_dim(w, "w")[0]
    _matrix(x, "x", device, _ONLY_BF16, (m, h))
    _matrix(w, "w", device, _ONLY_BF16, (v, h))
    _vector(targets, "targets", device, (torch.int64,), m)
    mean = _enumerator({"sum": 0, "mean": 1}, reduction, "reduction")
    g = _grad_type(grad_dtype)
    if piece < 0:
        raise ValueError(f"piece: {piece}, expected a number of rows or 0")
    stats = torch.empty((m + 1,), dtype=torch.float32, device=device)
    loss, rows = stats[m], stats[:m]
    if grads:
        if dx is None:
            dx = x.new_empty((m, h))
        else:
            _matrix(dx, "dx", device, _ONLY_BF16, (m, h), True)
        if dw is None:
            dw = x.new_empty((v, h), dtype=grad_dtype)
        else:
            _matrix(dw, "dw", device, (grad_dtype,), (v, h), True)
    else:
        dx = dw = None
    xs, ws = x.stride(), w.stride()
    args = _Loss(m, h, v, x.data_ptr(), xs[0], xs[1], w.data_ptr(), ws[0], ws[1], targets.data_ptr(), ignore_index, mean, scale,
                 loss.data_ptr(), rows.data_ptr(), _ptr(dx), 0 if dx is None else dx.stride(0), _ptr(dw),
                 0 if dw is None else dw.stride(0), g, piece)
    _call(_LOSS, args, device, workspace)
    return Loss(loss, rows, dx, dw)


def norm_forward(x: torch.Tensor, w: Optional[torch.Tensor] = None, b: Optional[torch.Tensor] = None, *, eps: float = 1e-5,
                 out: Optional[torch.Tensor] = None, out_dtype: torch.dtype = torch.bfloat16) -> Normed:
    """Layer norm of the rows of ``x`` (bf16 or fp32 [m, n], adjacent columns): ``(x - mean) rstd w + b`` with ``w`` and
    ``b`` [n] bf16 or fp32 (1 and 0 where they are not given), and the rows' statistics, which the backward pass takes."""
    device = _device(x, "x")
    m, n = _two_dim(x, "x")
    _matrix(x, "x", device, _TYPES, (m, n), True)
    if w is not None:
        _vector(w, "w", device, _TYPES, n)
    if b is not None:
        _vector(b, "b", device, _TYPES, n)
    if out is None:
        if out_dtype not in _TYPES:
            raise ValueError(f"out_dtype: {out_dtype}, expected one of {tuple(_TYPES)}")
        out = x.new_empty(m, n, dtype=out_dtype)
    else:
        _matrix(out, "out", device, _TYPES, (m, n), True)
    stats = x.new_empty(2, m, dtype=torch.float32)
    args = _NormForward(m, n, x.data_ptr(), x.stride(0), _TYPES[x.dtype], _ptr(w), 0 if w is None else _TYPES[w.dtype], _ptr(b),
                        0 if b is None else _TYPES[b.dtype], eps, out.data_ptr(), out.stride(0), _TYPES[out.dtype], stats.data_ptr())
    st = _lib.dlion_norm_forward(ctypes.byref(args), _stream(device))
    if st != OK:
        raise DlionError(st, "dlion_norm_forward")
    return Normed(out, stats)


def norm_backward(dy: torch.Tensor, x: torch.Tensor, w: Optional[torch.Tensor], stats: torch.Tensor, *,
                  residual: Optional[torch.Tensor] = None, need_dx: bool = True, need_dw: bool = True, need_db: bool = True,
                  grad_dtype: torch.dtype = torch.bfloat16, dx: Optional[torch.Tensor] = None, dw: Optional[torch.Tensor] = None,
                  db: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """Gradients of ``norm_forward(x, w, b)``, whose ``stats`` these are: dx in ``x``'s type, ``residual`` (of that type too:
    the gradient that goes past the norm) added, and ``dw``, ``db`` ([n]) in ``grad_dtype``.  Returns (dx, dw, db), None for what
    is not needed."""
    device = _device(dy, "dy")
    m, n = _two_dim(dy, "dy")
    _matrix(dy, "dy", device, _TYPES, (m, n), True)
    _matrix(x, "x", device, _TYPES, (m, n), True)
    if w is not None:
        _vector(w, "w", device, _TYPES, n)
    _matrix(stats, "stats", device, (torch.float32,), (2, m))
    if not stats.is_contiguous():
        raise ValueError(f"stats: expected adjacent values, got strides {stats.stride()}")
    stream = (x.dtype,)
    if residual is not None:
        _matrix(residual, "residual", device, stream, (m, n), True)
    g = _grad_type(grad_dtype)
    if not need_dx:
        dx = None
    elif dx is None:
        dx = x.new_empty(m, n)
    else:
        _matrix(dx, "dx", device, stream, (m, n), True)
    if not need_dw:
        dw = None
    elif dw is None:
        dw = x.new_empty(n, dtype=grad_dtype)
    else:
        _vector(dw, "dw", device, (grad_dtype,), n)
    if not need_db:
        db = None
    elif db is None:
        db = x.new_empty(n, dtype=grad_dtype)
    else:
        _vector(db, "db", device, (grad_dtype,), n)
    args = _NormBackward(m, n, dy.data_ptr(), dy.stride(0), _TYPES[dy.dtype], x.data_ptr(), x.stride(0), _TYPES[x.dtype], _ptr(w),
                         0 if w is None else _TYPES[w.dtype], stats.data_ptr(), _ptr(residual),
                         0 if residual is None else residual.stride(0), _ptr(dx), 0 if dx is None else dx.stride(0), _ptr(dw), _ptr(db), g)
    _call(_NORM_BACKWARD, args, device, workspace)
    return dx, dw, db


def _heads(t, name: str, device: int, shape):
    """The address and the strides of rows and heads of ``t``.  Raises unless it is a bf16 tensor of ``shape`` (rows, heads, dim) that
    16-byte accesses can take: adjacent columns of a head, rows and heads that begin on the 16-byte grid and are not broadcast."""
    if not (isinstance(t, _Tensor) and t.dtype is _BF16 and t.shape == shape and t.get_device() == device):
        _refused(t, name, device, _ONLY_BF16, shape)
    rs, hs, cs = t.stride()
    p = t.data_ptr()
    if cs != 1 or p % 16 or (shape[1] > 1 and (hs % 8 or hs < shape[2])) or (shape[0] > 1 and (rs % 8 or rs < shape[2])):
        raise ValueError(f"{name}: needs adjacent columns, and rows and heads on the 16-byte grid (got strides {(rs, hs, cs)}, "
                         f"address {p % 16} beyond a multiple of 16)")
    return p, rs, hs


def _attention_sizes(q, k, v, device: int):
    """(rows, heads, kv_heads, dim), and the fields of q, k and v."""
    for t, name in ((q, "q"), (k, "k"), (v, "v")):
        if not isinstance(t, _Tensor):
            raise ValueError(f"{name}: expected a torch.Tensor, got {type(t).__name__}")
    if len(q.shape) != 3 or len(k.shape) != 3:
        raise ValueError(f"q, k: expected [rows, heads, dim], got {q.dim()} and {k.dim()} dimensions")
    rows, heads, dim = q.shape
    kv = k.shape[1]
    if kv < 1 or heads < 1 or heads % kv:
        raise ValueError(f"q: {heads} heads, not a multiple of the {kv} of k and v")
    if dim < 8 or dim > 128 or dim % 8:
        raise ValueError(f"q: heads of {dim} columns, expected a multiple of 8, at most 128")
    shared = (rows, kv, dim)
    return (rows, heads, kv, dim), (*_heads(q, "q", device, (rows, heads, dim)), *_heads(k, "k", device, shared), *_heads(v, "v", device, shared))


def _sequences(offsets, length, rows: int, device: int):
    """The fields offsets, offsets_64, sequences, length."""
    if offsets is None:
        if length is None:
            return None, 0, 0, 0
        if not isinstance(length, int) or length < 1 or rows % length:
            raise ValueError(f"length: {length!r}, expected a number that divides the {rows} rows")
        return None, 0, 0, length
    if length is not None:
        raise ValueError("offsets and length: one of them at most")
    if not isinstance(offsets, _Tensor) or offsets.dim() != 1 or offsets.shape[0] < 1:
        raise ValueError("offsets: expected a tensor of sequences + 1 values")
    _vector(offsets, "offsets", device, (torch.int32, torch.int64), offsets.shape[0])
    return offsets.data_ptr(), int(offsets.dtype == torch.int64), offsets.shape[0] - 1, 0


def _scale(scale, dim: int) -> float:
    if scale is None:
        return dim ** -0.5
    if not 0.0 < scale <= 2e38:
        raise ValueError(f"scale: {scale!r}, expected a positive number of at most 2e38")
    return scale


def attention_forward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, *, causal: bool = True, scale: Optional[float] = None,
                      offsets: Optional[torch.Tensor] = None, length: Optional[int] = None, out: Optional[torch.Tensor] = None,
                      lse: Optional[torch.Tensor] = None, zero_rest: bool = False, workspace: Optional[torch.Tensor] = None) -> Attended:
    """Attention within sequences that lie one behind the other: ``q`` [rows, heads, dim], ``k`` and ``v`` [rows, kv_heads, dim],
    bf16, each a view of any row and head strides on the 16-byte grid (of one product's output, say); heads / kv_heads query
    heads in a row share a key head.  ``offsets`` (int32 or int64 on the device, ascending, sequences + 1 of them) says where
    the sequences begin and end, ``length`` that all have so many rows; with neither all rows are one.  ``scale`` is
    1 / sqrt(dim) where it is not given.  Rows in no sequence are left as they were in ``out`` and ``lse``, unless
    ``zero_rest``; they are zero in results that are not given."""
    device = _device(q, "q")
    sizes, inputs = _attention_sizes(q, k, v, device)
    rows, heads, _, dim = sizes
    sequences = _sequences(offsets, length, rows, device)
    clear = zero_rest
    if out is None:
        out, given = q.new_empty(rows, heads, dim), False
        fields = (out.data_ptr(), heads * dim, dim)
        clear = offsets is not None
    else:
        fields, given = _heads(out, "out", device, (rows, heads, dim)), True
    if lse is None:
        lse = q.new_empty(heads, rows, dtype=torch.float32)
        ld = rows
        if given and offsets is not None and not zero_rest:
            lse.zero_()                        # a result of each kind: the given one is left as it was
    else:
        _matrix(lse, "lse", device, (torch.float32,), (heads, rows), True)
        ld = max(lse.stride(0), rows)
        if not given and clear and not zero_rest:
            out.zero_()
            clear = False
    args = _AttentionForward(*sizes, *inputs, *sequences, 1 if causal else 0, _scale(scale, dim), *fields, lse.data_ptr(), ld, 1 if clear else 0)
    _call(_ATTENTION_FORWARD, args, device, workspace)
    return Attended(out, lse)


def attention_backward(dout: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor, lse: torch.Tensor, *,
                       causal: bool = True, scale: Optional[float] = None, offsets: Optional[torch.Tensor] = None,
                       length: Optional[int] = None, dq: Optional[torch.Tensor] = None, dk: Optional[torch.Tensor] = None,
                       dv: Optional[torch.Tensor] = None, zero_rest: bool = False, workspace: Optional[torch.Tensor] = None):
    """Gradients (dq, dk, dv) of ``attention_forward`` with the same arguments, whose results ``out`` and ``lse`` are.  ``dk`` and
    ``dv`` are summed over the query heads that share them.  Views of one tensor are valid results: the gradient
    of the product that made q, k and v.  Rows in no sequence as in ``attention_forward``."""
    device = _device(dout, "dout")
    sizes, inputs = _attention_sizes(q, k, v, device)
    rows, heads, kv, dim = sizes
    sequences = _sequences(offsets, length, rows, device)
    own, shared = (rows, heads, dim), (rows, kv, dim)
    saved = (*_heads(out, "out", device, own), *_heads(dout, "dout", device, own))
    _matrix(lse, "lse", device, (torch.float32,), (heads, rows), True)
    results, fields, given = [], [], 0
    for t, name, shape in ((dq, "dq", own), (dk, "dk", shared), (dv, "dv", shared)):
        if t is None:
            t = q.new_empty(*shape)
            fields += (t.data_ptr(), shape[1] * dim, dim)
        else:
            fields += _heads(t, name, device, shape)
            given += 1
        results.append(t)
    clear = zero_rest or (offsets is not None and given == 0)
    if offsets is not None and not clear and given < 3:        # results of each kind: the given ones are left as they were
        for t, was in zip(results, (dq, dk, dv)):
            if was is None:
                t.zero_()
    args = _AttentionBackward(*sizes, *inputs, *saved, lse.data_ptr(), max(lse.stride(0), rows), *sequences, 1 if causal else 0, _scale(scale, dim),
                              *fields, 1 if clear else 0)
    _call(_ATTENTION_BACKWARD, args, device, workspace)
    return tuple(results)


def check() -> None:
    """Waits for the current stream; raises if a kernel's wait ran out since the last check."""
    st = _lib.dlion_layers_check(torch.cuda.current_stream().cuda_stream)
    if st != OK:
        raise DlionError(st, "dlion_layers_check")
