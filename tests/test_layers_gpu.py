"""The layer operators against their formulas in 64 bits.

Tolerances, element by element.  A bf16 result: half a spacing, 2^-8 of the value.  A sum of K products: the tensor
cores add 16 at a time to a binary32 accumulator and drop what does not fit, so at most (K/16 + 8) 2^-22 of the
sum of the products' sizes, whatever the order.  An operand that is itself rounded to bf16 (act(u), d): 2^-8 of the sum of the
products' sizes.  Activations: their slope is at most 1.13, their own error 2^-20."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
BF, F32, F64 = torch.bfloat16, torch.float32, torch.float64
DEV = "cuda:0"


@pytest.fixture(scope="module")
def L():
    assert torch.cuda.is_available(), "this test needs a CUDA device"
    from paper_2404_00438_b200 import build
    build.build()
    from paper_2404_00438_b200 import layers
    yield layers
    layers.check()


def normal(seed, *shape, std=1.0, dtype=BF):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return (torch.randn(*shape, generator=g, device=DEV) * std).to(dtype)


def act(z, kind):
    if kind == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if kind == "silu":
        return z * torch.special.expit(z)
    if kind == "gelu":
        return z * torch.special.expit(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))
    return z


def slope(z, kind):
    if kind == "relu":
        return (z > 0).to(z.dtype)
    if kind == "silu":
        p = torch.special.expit(z)
        return p + z * p * (1 - p)
    if kind == "gelu":
        c = 2 * math.sqrt(2 / math.pi)
        p = torch.special.expit(c * (z + 0.044715 * z ** 3))
        return p + z * p * (1 - p) * c * (1 + 0.134145 * z ** 2)
    return torch.ones_like(z)


def sum_error(k, sizes):
    return (k / 16 + 8) * 2.0 ** -22 * sizes


def close(name, got, want, tolerance):
    got = got.to(F64)
    tolerance = tolerance + (2.0 ** -8 * want.abs() if not isinstance(tolerance, float) else 0)
    bad = ~((got - want).abs() <= tolerance)
    assert not bad.any(), f"{name}: {int(bad.sum())} of {bad.numel()}, worst {float(((got - want).abs() - tolerance).max())}"


def eight(v):
    """The 8-bit form's values, from its definition."""
    m, k = v.shape
    out = torch.empty_like(v)
    for a in range(0, k, 32):
        top = v[:, a:a + 32].abs().amax(1, keepdim=True)
        e = torch.full_like(top, -126)
        while bool((127 * torch.exp2(e) < top).any()):
            e = torch.where(127 * torch.exp2(e) < top, e + 1, e)
        out[:, a:a + 32] = torch.round(v[:, a:a + 32] / torch.exp2(e)) * torch.exp2(e)
    return out


# ------------------------------------------------------------------------------------------------ forward
SHAPES = [(1, 1, 1), (1, 768, 2304), (2, 33, 31), (3, 768, 1000), (5, 129, 257), (8, 2048, 777), (17, 64, 130), (33, 100, 96), (64, 768, 768), (127, 65, 129),
          (197, 768, 768), (256, 256, 256), (300, 777, 513), (777, 768, 1001), (1000, 1, 300), (4, 4096, 64), (2048, 320, 40)]


@pytest.mark.parametrize("m,k,n", SHAPES)
@pytest.mark.parametrize("kind,transposed,f32", [("none", False, True), ("gelu", True, False), ("silu", False, False), ("relu", True, True)])
def test_forward(L, m, k, n, kind, transposed, f32):
    x = normal(1, m, k)
    w = normal(2, n, k, std=k ** -0.5).t() if transposed else normal(2, k, n, std=k ** -0.5)
    bias = normal(3, n, dtype=F32 if f32 else BF)
    residual = normal(4, m, n) if kind in ("none", "gelu") else None
    y = L.linear_forward(x, w, bias, act=kind, residual=residual, out_dtype=F32 if f32 else BF)
    z = x.to(F64) @ w.to(F64) + bias.to(F64)
    want = act(z, kind) + (0 if residual is None else residual.to(F64))
    off = 1.13 * sum_error(k, x.to(F64).abs() @ w.to(F64).abs() + bias.to(F64).abs()) + 2.0 ** -20 * (1 + z.abs() + want.abs())
    if f32:
        assert y.dtype == F32 and not ((y.to(F64) - want).abs() > off).any()
    else:
        close("y", y, want, off)


@pytest.mark.parametrize("m,k,n", [(1, 96, 33), (7, 768, 100), (197, 768, 3072 // 4), (257, 65, 2304)])
@pytest.mark.parametrize("keep", ["bf16", "8bit"])
def test_kept(L, m, k, n, keep):
    x, w, bias = normal(1, m, k), normal(2, k, n, std=k ** -0.5), normal(3, n)
    y, kept = L.linear_forward(x, w, bias, act="gelu", keep=keep)
    plain = L.linear_forward(x, w, bias, act="gelu")
    assert torch.equal(y, plain)
    z = x.to(F64) @ w.to(F64) + bias.to(F64)
    off = sum_error(k, x.to(F64).abs() @ w.to(F64).abs() + bias.to(F64).abs())
    if keep == "bf16":
        close("z", kept, z, off)
    else:       # half a step of the block, which is at most 1/127 of its largest value, and a block's doubled where it sits at the edge
        blocks = torch.nn.functional.pad(z.abs(), (0, -n % 32)).view(m, -1, 32).amax(2, keepdim=True).expand(-1, -1, 32).reshape(m, -1)[:, :n]
        got = L.restore8(kept).to(F64)
        assert not ((got - z).abs() > blocks / 63.5 + off).any()
        step = torch.exp2(kept.e.to(F64).t().repeat_interleave(32, 1)[:, :n] - 127)
        assert not ((got - z).abs() > step / 2 + off).any()


def test_forward_strides_and_alignment(L):
    """Rows off the 16-byte grid, every other column, a transposed x, broadcast rows, outputs inside a larger array."""
    m, k, n = 70, 72, 50
    big = normal(1, m + 3, 2 * k + 9)
    xs = [big[3:, 5:5 + k], big[:m, 0:2 * k:2], normal(1, k, m).t(), normal(1, 1, k).expand(m, k), big[1:m + 1, 8:8 + k], normal(1, m, 1).expand(m, k)]
    ws = [normal(2, k, n), normal(2, n, k).t(), normal(2, k + 1, n + 7)[1:, 3:3 + n], normal(2, 2 * k, n)[::2], normal(2, k, 1).expand(k, n)]
    r = normal(4, m, n + 5)[:, 1:n + 1]
    for x in xs:
        for w in ws:
            out = torch.full((m + 2, n + 6), 7.0, dtype=BF, device=DEV)
            view = out[1:m + 1, 3:3 + n]
            L.linear_forward(x, w, residual=r, out=view)
            want = x.to(F64) @ w.to(F64) + r.to(F64)
            close("y", view, want, sum_error(k, x.to(F64).abs() @ w.to(F64).abs()) + 2.0 ** -20 * want.abs())
            mask = torch.ones_like(out, dtype=torch.bool)
            mask[1:m + 1, 3:3 + n] = False
            assert bool((out[mask] == 7.0).all())


def test_residual_may_be_the_output(L):
    for m in (5, 300):
        x, w, r = normal(1, m, 256), normal(2, 256, 300), normal(3, m, 300)
        want = L.linear_forward(x, w, residual=r)
        assert torch.equal(L.linear_forward(x, w, residual=r, out=r), want)


def test_no_rows(L):
    x, w = normal(1, 0, 64), normal(2, 64, 96)
    assert L.linear_forward(x, w).shape == (0, 96)
    dx, dw, db = L.linear_backward(normal(1, 0, 96), w, x, grad_dtype=F32)
    assert dx.shape == (0, 64) and not dw.any() and not db.any()
    r = L.lm_loss(x, normal(2, 50, 64), torch.zeros(0, dtype=torch.int64, device=DEV))
    assert float(r.loss) == 0.0 and not r.dw.any()
    assert L.restore8(L.checkpoint8(x)).shape == (0, 64)


def test_not_finite(L):
    """NaN and infinity stay in their row; nothing else is touched."""
    x, w = normal(1, 40, 64), normal(2, 64, 70)
    clean = L.linear_forward(x, w, act="gelu")
    x[3, 5], x[9, 0] = float("nan"), float("inf")
    y, kept = L.linear_forward(x, w, act="gelu", keep="8bit")
    assert bool(y[3].isnan().all()) and bool((~y[9].isfinite() | (y[9] == 0)).all())
    rest = [i for i in range(40) if i not in (3, 9)]
    assert torch.equal(y[rest], clean[rest])
    assert bool(L.restore8(kept)[[3, 9]].isnan().all())
    assert bool(L.linear_forward(x, w, act="relu")[3].isnan().all())


# ------------------------------------------------------------------------------------------------ backward
@pytest.mark.parametrize("m,k,n", [(1, 33, 17), (1, 768, 2304), (9, 40, 48), (64, 768, 256), (197, 768, 768), (300, 257, 129), (777, 96, 1001), (2500, 64, 72)])
@pytest.mark.parametrize("kind,eight_bits,transposed,f32", [("none", False, False, True), ("none", True, True, False), ("gelu", True, False, False),
                                                            ("gelu", False, True, True), ("silu", True, True, False), ("relu", False, False, False)])
def test_backward(L, m, k, n, kind, eight_bits, transposed, f32):
    u, dy = normal(1, m, k), normal(2, m, n)
    w = normal(3, n, k, std=n ** -0.5).t() if transposed else normal(3, k, n, std=n ** -0.5)
    residual = normal(4, m, k) if kind != "relu" else None
    saved = L.checkpoint8(u) if eight_bits else u
    u = L.restore8(saved) if eight_bits else u
    dx, dw, db = L.linear_backward(dy, w, saved, act=kind, residual=residual, grad_dtype=F32 if f32 else BF)
    U, DY, W = u.to(F64), dy.to(F64), w.to(F64)
    s = slope(U, kind)
    want = (DY @ W.t()) * s + (0 if residual is None else residual.to(F64))
    close("dx", dx, want, 1.13 * sum_error(n, DY.abs() @ W.abs().t()) + 2.0 ** -19 * ((DY @ W.t()).abs() + want.abs()))
    a = act(U, kind)
    sizes = a.abs().t() @ DY.abs()
    off = sum_error(m, sizes) + (2.0 ** -8 * sizes if kind in ("gelu", "silu") else 0)
    want = a.t() @ DY
    assert dw.dtype == (F32 if f32 else BF) and dw.stride() == (w.stride() if k > 1 and n > 1 else dw.stride())
    if f32:
        assert not ((dw.to(F64) - want).abs() > off + 2.0 ** -24 * want.abs()).any()
    else:
        close("dw", dw, want, off)
    off = (m / 8 + 600) * 2.0 ** -24 * DY.abs().sum(0)
    if f32:
        assert not ((db.to(F64) - DY.sum(0)).abs() > off).any()
    else:
        close("db", db, DY.sum(0), off)
    # the parts asked for alone are the same
    only = L.linear_backward(dy, w, saved, act=kind, residual=residual, need_dx=False, need_db=False, grad_dtype=F32 if f32 else BF)
    assert only[0] is None and only[2] is None and torch.equal(only[1], dw)


def test_backward_against_differences(L):
    """du along a random direction against central differences of the 64-bit layer."""
    m, k, n = 24, 40, 56
    for kind in ("none", "relu", "gelu", "silu"):
        u, w, dy = normal(1, m, k), normal(2, k, n, std=k ** -0.5), normal(3, m, n)
        dx, dw, db = L.linear_backward(dy, w, u, act=kind, grad_dtype=F32)
        U, W, DY = u.to(F64), w.to(F64), dy.to(F64)
        f = lambda a, b, c: float(((act(a, kind) @ b + c) * DY).sum())      # noqa: E731
        zero = torch.zeros(n, dtype=F64, device=DEV)
        for got, at, turn in ((dx, U, lambda v: f(v, W, zero)), (dw, W, lambda v: f(U, v, zero)), (db, zero, lambda v: f(U, W, v))):
            v = normal(7, *at.shape, dtype=F64)
            h = 1e-6
            change = (turn(at + h * v) - turn(at - h * v)) / (2 * h)
            size = float((got.to(F64).abs() * v.abs()).sum())
            # roundings of the elements, 2^-8 each, add up along v at most to their sum; relu's corner: |u| < h has no bf16 here
            assert abs(float((got.to(F64) * v).sum()) - change) <= 2.0 ** -8 * size + 1e-5 * (1 + abs(change))


def test_backward_strides(L):
    m, k, n = 90, 50, 70
    base = normal(1, n, m)
    for dy in (base.t(), normal(1, m, 2 * n)[:, ::2], normal(1, 1, n).expand(m, n), normal(1, m, n + 3)[:, 1:n + 1], normal(1, m, 1).expand(m, n)):
        u, w = normal(2, m, k + 1)[:, 1:], normal(3, k, n + 1)[:, 1:]
        arena = torch.full((k * n + n + 64,), 5.0, dtype=F32, device=DEV)
        dw, db = arena[16:16 + k * n].view(k, n), arena[32 + k * n:32 + k * n + n]
        out = torch.full((m, k + 4), 5.0, dtype=BF, device=DEV)
        L.linear_backward(dy, w, u, act="silu", dx=out[:, 2:2 + k], dw=dw, db=db, grad_dtype=F32)
        U, DY, W = u.to(F64), dy.to(F64), w.to(F64)
        want = (DY @ W.t()) * slope(U, "silu")
        close("dx", out[:, 2:2 + k], want, sum_error(n, 1.13 * DY.abs() @ W.abs().t()) + 2.0 ** -19 * (DY @ W.t()).abs())
        sizes = act(U, "silu").abs().t() @ DY.abs()
        assert not ((dw.to(F64) - act(U, "silu").t() @ DY).abs() > sum_error(m, sizes) + 2.0 ** -8 * sizes).any()
        assert not ((db.to(F64) - DY.sum(0)).abs() > (m / 8 + 600) * 2.0 ** -24 * DY.abs().sum(0)).any()
        edge = torch.ones_like(arena, dtype=torch.bool)
        edge[16:16 + k * n] = False
        edge[32 + k * n:32 + k * n + n] = False
        assert bool((arena[edge] == 5.0).all()) and bool((out[:, :2] == 5.0).all()) and bool((out[:, 2 + k:] == 5.0).all())


# ------------------------------------------------------------------------------------------------ 8 bits
@pytest.mark.parametrize("m,k", [(1, 1), (1, 31), (3, 32), (5, 33), (64, 768), (100, 2048), (33, 1000)])
def test_checkpoint8(L, m, k):
    x = normal(1, m, k) * torch.exp2(torch.randint(-30, 30, (m, 1), device=DEV).float()).to(BF)
    x[0, 0] = 0
    c = L.checkpoint8(x)
    assert c.q.dtype == torch.int8 and tuple(c.e.shape) == ((k + 31) // 32, m)
    back = L.restore8(c)
    assert torch.equal(back.to(F64), eight(x.to(F64)))           # ties and all
    again = L.checkpoint8(back)
    assert torch.equal(L.restore8(again), back)                  # what it holds it holds exactly


def test_checkpoint8_special_values(L):
    x = torch.zeros(8, 96, dtype=BF, device=DEV)
    x[1, 3], x[2, 40], x[3, 95] = float("nan"), float("inf"), -float("inf")
    x[4, :32] = 3.3e38
    x[5, :32] = 1e-38
    x[6, 0], x[6, 1] = 127.0, 1.0
    x[7, 0], x[7, 1] = 127.5, 1.0
    y = L.restore8(L.checkpoint8(x))
    nan = torch.zeros_like(x, dtype=torch.bool)
    nan[1, :32], nan[2, 32:64], nan[3, 64:] = True, True, True
    assert torch.equal(y.isnan(), nan)
    assert torch.equal(y[4].to(F64), eight(x[4:5].to(F64))[0]) and bool(y[4].isfinite().all())
    assert not y[5].any() or bool((y[5, :32] > 0).all())         # steps below 2^-126 do not exist
    assert float(y[6, 0]) == 127.0 and float(y[6, 1]) == 1.0
    assert float(y[7, 1]) == 0.0 or float(y[7, 1]) == 2.0        # step 2: one is a tie, to even


def test_checkpoint8_views_and_long_offsets(L):
    x = normal(1, 50, 101)[:, 3:99]
    hold = L.Checkpoint8(torch.full((52, 100), 9, dtype=torch.int8, device=DEV)[1:51, 2:98], torch.full((3, 60), 9, dtype=torch.uint8, device=DEV)[:, 4:54])
    c = L.checkpoint8(x, out=hold)
    assert torch.equal(L.restore8(c).to(F64), eight(x.to(F64)))
    assert bool((hold.q._base[0] == 9).all()) and bool((hold.q._base[:, 98:] == 9).all()) and bool((hold.e._base[:, :4] == 9).all())
    m, k = 66000, 32800                                          # more than 2^31 values
    x = torch.empty(m, k, dtype=BF, device=DEV)
    x[-40:] = normal(2, 40, k)
    x[:-40] = 1.0
    y = L.restore8(L.checkpoint8(x))
    assert torch.equal(y[-40:].to(F64), eight(x[-40:].to(F64))) and bool((y[12345] == 1.0).all())


def test_forward_long_offsets(L):
    m, k, n = 43200, 64, 50257                                   # y has more than 2^31 values
    x, w = normal(1, m, k), normal(2, n, k).t()
    y = L.linear_forward(x, w)
    rows = torch.tensor([0, 1, 42735, 42736, m - 1], device=DEV)
    want = x[rows].to(F64) @ w.to(F64)
    close("y", y[rows], want, sum_error(k, x[rows].to(F64).abs() @ w.to(F64).abs()))


# ------------------------------------------------------------------------------------------------ loss
def loss_reference(x, w, t, ignore, mean, scale=1.0):
    X, W = x.to(F64), w.to(F64)
    keep = t != ignore
    at = t.clamp(0, len(w) - 1)
    logits = X @ W.t()
    lse = torch.logsumexp(logits, 1)
    rows = torch.where(keep, lse - logits.gather(1, at[:, None])[:, 0], torch.zeros_like(lse))
    n = int(keep.sum())
    loss = rows.sum() / (n if mean and n else 1)
    d = torch.exp(logits - lse[:, None])
    d[torch.arange(len(t), device=DEV), at] -= 1
    d = torch.where(keep[:, None], d, torch.zeros_like(d)) * (scale / (n if mean and n else 1))
    return loss, rows, d @ W, d.t() @ X, d, lse, logits


def check_loss(L, x, w, t, ignore=-100, mean=True, scale=1.0, f32=False, piece=0):
    (m, h), v = x.shape, len(w)
    r = L.lm_loss(x, w, t, ignore_index=ignore, reduction="mean" if mean else "sum", scale=scale, grad_dtype=F32 if f32 else BF, piece=piece)
    loss, rows, dx, dw, d, lse, logits = loss_reference(x, w, t, ignore, mean, scale)
    X, W = x.to(F64).abs(), w.to(F64).abs()
    # a logit's sum, and a few hundred additions and exponentials of 2^-22
    l_off = sum_error(h, (X @ W.t()).amax(1))
    off = 2 * l_off + 2.0 ** -16 * (1 + lse.abs() + logits.abs().amax(1) * 2.0 ** -4)
    assert not ((r.rows.to(F64) - rows).abs() > off).any()
    n = max(1, int((t != ignore).sum())) if mean else 1
    assert abs(float(r.loss) - float(loss)) <= float(off.sum()) / n + 2.0 ** -18 * abs(float(loss))
    alone = L.lm_loss(x, w, t, ignore_index=ignore, reduction="mean" if mean else "sum", grads=False)
    assert alone.dx is None and alone.dw is None
    assert not ((alone.rows.to(F64) - rows).abs() > off).any()
    # d: its code (2^-11 octaves), its rounding to bf16, the row's lse; at the target the part 1 is exact up to its rounding
    e = d.abs() * (2.0 ** -8 + 2.0 ** -11) + (off * 1.1)[:, None] * (d.abs() + (abs(scale) / n) * 2.0 ** -8 * (d != 0))
    e = e + (abs(scale) / n) * 1e-19
    close("dx", r.dx, dx, e @ W + sum_error(v, d.abs() @ W))
    off_w = e.t() @ X + sum_error(m, d.abs().t() @ X)
    if f32:
        assert not ((r.dw.to(F64) - dw).abs() > off_w + 2.0 ** -22 * dw.abs()).any()
    else:
        close("dw", r.dw, dw, off_w)
    return r


@pytest.mark.parametrize("m,h,v", [(1, 64, 7), (1, 768, 1000), (2, 1, 3), (33, 64, 129), (197, 768, 1000), (300, 100, 1), (257, 65, 2051), (130, 256, 50257)])
@pytest.mark.parametrize("mean,f32,piece", [(True, False, 0), (False, True, 100)])
def test_loss(L, m, h, v, mean, f32, piece):
    x, w = normal(1, m, h), normal(2, v, h, std=2 * h ** -0.5)
    t = torch.randint(0, v, (m,), device=DEV, generator=torch.Generator(device=DEV).manual_seed(3))
    if m > 2:
        t[::7] = -100
        t[1], t[2] = 0, v - 1
    check_loss(L, x, w, t, mean=mean, f32=f32, piece=piece, scale=1.0 if mean else 0.37)


@pytest.mark.parametrize("piece", [0, 1, 50, 64, 149, 150, 1000])
def test_loss_pieces(L, piece):
    x, w = normal(1, 150, 72), normal(2, 333, 72)
    t = torch.arange(150, device=DEV) * 2
    r = check_loss(L, x, w, t, piece=piece)
    assert torch.equal(r.rows, L.lm_loss(x, w, t).rows) or piece


def test_loss_sharp_and_masked(L):
    """Logits in the hundreds; words masked by the type's lowest value, a whole group of them too."""
    x, w = normal(1, 64, 96), normal(2, 700, 96, std=10.0)
    check_loss(L, x, w, torch.arange(64, device=DEV))
    w = normal(2, 700, 96, std=0.2)
    x[:, 0] = 1.0
    w[128:400, 0] = torch.finfo(BF).min
    w[650, 0] = torch.finfo(BF).min
    t = torch.arange(64, device=DEV)
    r = L.lm_loss(x, w, t, grad_dtype=F32)
    keep = torch.cat([torch.arange(128), torch.arange(400, 650), torch.arange(651, 700)]).to(DEV)
    s = check_loss(L, x, w[keep].contiguous(), t, f32=True)
    assert float((r.rows - s.rows).abs().max()) <= 1e-5
    assert bool(r.dx.isfinite().all()) and float((r.dx.float() - s.dx.float()).abs().max()) <= 2.0 ** -6 * float(s.dx.float().abs().max())
    masked = torch.ones(700, dtype=torch.bool, device=DEV)
    masked[keep] = False
    assert not r.dw[masked].any()


def test_loss_ignored_invalid_and_not_finite(L):
    x, w = normal(1, 40, 64), normal(2, 90, 64)
    t = torch.full((40,), -100, device=DEV)
    r = L.lm_loss(x, w, t)
    assert float(r.loss) == 0 and not r.rows.any() and not r.dx.any() and not r.dw.any()
    t = torch.arange(40, device=DEV)
    t[5] = 3000
    r = L.lm_loss(x, w, t, grad_dtype=F32)
    ok = [i for i in range(40) if i != 5]
    assert math.isnan(float(r.loss)) and bool(r.rows[5].isnan()) and bool(r.rows[ok].isfinite().all())
    assert bool(r.dx[5].isnan().all()) and bool(r.dx[ok].isfinite().all())
    t[5] = 5
    x[7, 0] = float("nan")
    r = L.lm_loss(x, w, t)
    ok = [i for i in range(40) if i != 7]
    assert bool(r.rows[7].isnan()) and bool(r.rows[ok].isfinite().all()) and bool(r.dx[7].isnan().all()) and bool(r.dx[ok].isfinite().all())
    t[7] = -100                                                    # ignored: its NaN goes no further than the row's own products
    r = L.lm_loss(x, w, t)
    assert math.isfinite(float(r.loss)) and float(r.rows[7]) == 0 and not r.dx[7].any()
    r = L.lm_loss(x[:7], w, t[:7], ignore_index=3)
    assert float(r.rows[3]) == 0 and not r.dx[3].any()


def test_loss_against_differences(L):
    x, w = normal(1, 20, 48), normal(2, 300, 48, std=0.3)
    t = (torch.arange(20, device=DEV) * 13) % 300
    t[4] = -100
    r = L.lm_loss(x, w, t, grad_dtype=F32)
    X, W = x.to(F64), w.to(F64)
    for got, at, f in ((r.dx, X, lambda v: loss_reference(v, W, t, -100, True)[0]), (r.dw, W, lambda v: loss_reference(X, v, t, -100, True)[0])):
        v = normal(9, *at.shape, dtype=F64)
        h = 1e-5
        change = float((f(at + h * v) - f(at - h * v)) / (2 * h))
        size = float((got.to(F64).abs() * v.abs()).sum())
        assert abs(float((got.to(F64) * v).sum()) - change) <= 2.0 ** -7 * size + 1e-6


def test_loss_strides(L):
    x, w = normal(1, 64, 100).t()[:, :50], normal(2, 130, 51)[:, 1:]
    t = torch.arange(100, device=DEV)
    check_loss(L, x, w, t)
    hold = torch.full((132, 60), 3.0, dtype=F32, device=DEV)
    L.lm_loss(x, w, t, dw=hold[1:131, 5:55], grad_dtype=F32)
    assert torch.equal(hold[1:131, 5:55], L.lm_loss(x, w, t, grad_dtype=F32).dw)
    assert bool((hold[0] == 3).all()) and bool((hold[:, 55:] == 3).all()) and bool((hold[:, :5] == 3).all())


# ------------------------------------------------------------------------------------------------ calls
def test_same_call_same_bits_and_other_streams(L):
    x, w, dy = normal(1, 300, 768), normal(2, 768, 500, std=0.05), normal(3, 300, 500)
    t = torch.arange(300, device=DEV)
    def everything():
        y, k = L.linear_forward(x, w, act="gelu", keep="8bit")
        l = L.lm_loss(x, w.t().contiguous(), t)
        return [y, *k, *L.linear_backward(dy, w, x, act="silu"), *l]
    first = everything()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        second = everything()
    side.synchronize()
    for a, b in zip(first, second):
        assert torch.equal(a, b)


def test_captured_in_a_graph(L):
    x, w, dy = normal(1, 200, 256), normal(2, 256, 384, std=0.06), normal(3, 200, 384)
    def everything():
        y, k = L.linear_forward(x, w, act="gelu", keep="8bit")
        return [y, *L.linear_backward(dy, w, x, act="gelu"), *L.lm_loss(x, w.t(), torch.zeros(200, dtype=torch.int64, device=DEV))]
    want = everything()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        everything()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = everything()
    for _ in range(2):
        g.replay()
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_binding_refusals(L):
    x, w = normal(1, 8, 64), normal(2, 64, 32)
    for bad in (lambda: L.linear_forward(x.float(), w), lambda: L.linear_forward(x, w[:32]), lambda: L.linear_forward(x, w, normal(3, 31)),
                lambda: L.linear_forward(x, w, act="tanh"), lambda: L.linear_forward(x, w, keep="4bit"), lambda: L.linear_forward(x[0], w),
                lambda: L.linear_forward(x, w, residual=normal(3, 32, 8).t()), lambda: L.linear_forward(x, w, out=torch.empty(8, 32, device=DEV).half()),
                lambda: L.linear_forward(x, w.cpu()), lambda: L.linear_forward(x, w, out=normal(3, 32, 8).t()),
                lambda: L.linear_forward(x, w, out_dtype=torch.float16),
                lambda: L.linear_backward(normal(3, 8, 32), w, None), lambda: L.linear_backward(normal(3, 8, 32), w, normal(3, 64, 8).t()),
                lambda: L.linear_backward(normal(3, 8, 32), w, x, dw=torch.empty(64, 64, dtype=BF, device=DEV)[:, ::2]),
                lambda: L.linear_backward(normal(3, 8, 32), w, x, grad_dtype=torch.float16),
                lambda: L.linear_backward(normal(3, 8, 32), w, L.Checkpoint8(torch.zeros(8, 64, dtype=torch.int8, device=DEV), torch.zeros(1, 8, dtype=torch.uint8, device=DEV))),
                lambda: L.checkpoint8(x.t()), lambda: L.checkpoint8(x.float()), lambda: L.lm_loss(x, normal(2, 9, 63), torch.zeros(8, dtype=torch.int64, device=DEV)),
                lambda: L.lm_loss(x, normal(2, 9, 64), torch.zeros(8, dtype=torch.int32, device=DEV)), lambda: L.lm_loss(x, normal(2, 9, 64), torch.zeros(7, dtype=torch.int64, device=DEV)),
                lambda: L.lm_loss(x, normal(2, 9, 64), torch.zeros(8, dtype=torch.int64, device=DEV), reduction="none"),
                lambda: L.lm_loss(x, normal(2, 9, 64), torch.zeros(8, dtype=torch.int64, device=DEV), piece=-1)):
        with pytest.raises(ValueError):
            bad()
    odd = normal(2, 64, 33)[:, :32]                                # rows off the grid: needs a workspace
    with pytest.raises(ValueError):
        L.linear_forward(x, odd, workspace=torch.empty(16, dtype=torch.uint8, device=DEV))
    big = torch.empty(1 << 20, dtype=torch.uint8, device=DEV)
    assert torch.equal(L.linear_forward(x, odd, workspace=big), L.linear_forward(x, odd))
