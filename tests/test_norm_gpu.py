"""Layer norm against its formulas in 64 bits.

Tolerances: binary32 sums of n values in a tree or in runs of at most n / 32: (n / 32 + 16) 2^-24 of the sum of the sizes;
each of the some ten roundings of an element 2^-24 of the terms' sizes; a bf16 result 2^-8 of itself.  The mean's error moves
every centred value; the variance's (twice the relative error of the centred values, and its own sum's) moves rstd by half."""
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
    return layers


def normal(seed, *shape, std=1.0, mean=0.0, dtype=BF):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return (torch.randn(*shape, generator=g, device=DEV) * std + mean).to(dtype)


def half_step(t):
    return torch.finfo(t).eps / 2


def inside(name, got, want, off):
    off = off + half_step(got.dtype) * want.abs()
    bad = ~((got.to(F64) - want).abs() <= off + 1e-37)
    assert not bad.any(), f"{name}: {int(bad.sum())} of {bad.numel()}, worst {float(((got.to(F64) - want).abs() / (off + 1e-37)).max())} of the tolerance"


def verify(x, w, b, eps, y, stats, dy=None, residual=None, grads=None):
    m, n = x.shape
    e = 2.0 ** -24
    run = (n / 32 + 16) * e
    X = x.to(F64)
    W = torch.ones(n, dtype=F64, device=DEV) if w is None else w.to(F64)
    B = torch.zeros(n, dtype=F64, device=DEV) if b is None else b.to(F64)
    mean = X.mean(1, keepdim=True)
    off_mean = run * X.abs().mean(1, keepdim=True) + e * mean.abs()
    c = X - mean
    var = (c * c).mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(var + eps)
    off_c = off_mean + 2 * e * c.abs()
    off_var = run * var + 2 * (c.abs() * off_c).mean(1, keepdim=True) + (off_c ** 2).mean(1, keepdim=True)
    rel = 0.5 * off_var / (var + eps) + 4 * e
    inside("mean", stats[0], mean[:, 0], off_mean[:, 0])
    inside("rstd", stats[1], rstd[:, 0], (rel * rstd)[:, 0])
    h = c * rstd
    off_h = off_c * rstd + h.abs() * (rel + e)
    inside("y", y, h * W + B, off_h * W.abs() + 4 * e * ((h * W).abs() + B.abs()))
    if grads is None:
        return
    dx, dw, db = grads
    D = dy.to(F64)
    u = D * W
    a, t = u.mean(1, keepdim=True), (u * h).mean(1, keepdim=True)
    off_a = run * u.abs().mean(1, keepdim=True)
    off_t = run * (u * h).abs().mean(1, keepdim=True) + (u.abs() * off_h).mean(1, keepdim=True)
    R = 0 if residual is None else residual.to(F64)
    if dx is not None:
        want = rstd * (u - a - h * t) + R
        inner = u.abs() + a.abs() + (h * t).abs()
        off = rstd * (off_a + off_h * t.abs() + h.abs() * off_t + inner * (rel + 8 * e)) + 2 * e * (want.abs() + (R.abs() if residual is not None else 0))
        inside("dx", dx, want, off)
    rows = (m / 32 + 32) * e                                      # runs over the rows: a block's, then the blocks'
    if dw is not None:
        inside("dw", dw, (D * h).sum(0), rows * (D * h).abs().sum(0) + (D.abs() * off_h).sum(0))
    if db is not None:
        inside("db", db, D.sum(0), rows * D.abs().sum(0))


WIDTHS = [1, 2, 7, 8, 31, 64, 100, 255, 256, 257, 768, 1000, 1001, 1024, 1032, 1600, 2048, 2303, 4096, 5000, 8192, 12288, 12289, 20000, 32768, 40000]


@pytest.mark.parametrize("n", WIDTHS)
@pytest.mark.parametrize("stream,branch", [(BF, BF), (F32, BF), (BF, F32), (F32, F32)])
def test_widths(L, n, stream, branch):
    m = 37 if n < 4000 else 5
    x = normal(n, m, n, std=2.0, mean=0.5, dtype=stream)
    w, b = normal(2, n, std=0.3, mean=1.0, dtype=branch), normal(3, n, dtype=stream)
    y, stats = L.norm_forward(x, w, b, out_dtype=branch)
    assert y.dtype == branch
    dy, r = normal(4, m, n, dtype=branch), normal(5, m, n, dtype=stream)
    grads = L.norm_backward(dy, x, w, stats, residual=r, grad_dtype=stream)
    assert grads[0].dtype == stream and grads[1].dtype == stream
    verify(x, w, b, 1e-5, y, stats, dy, r, grads)


@pytest.mark.parametrize("m", [1, 2, 3, 8, 197, 1000, 5001])
@pytest.mark.parametrize("n", [96, 768, 1001, 2048])
def test_rows(L, m, n):
    x, w = normal(1, m, n), normal(2, n)
    y, stats = L.norm_forward(x, w, None, eps=1e-6)
    dy = normal(4, m, n)
    verify(x, w, None, 1e-6, y, stats, dy, None, L.norm_backward(dy, x, w, stats))


@pytest.mark.parametrize("n,m", [(1001, 4801), (1536, 5003), (2047, 4750), (2056, 1300), (2303, 1250), (4096, 1201), (4450, 700), (5000, 1001), (8192, 603), (9001, 301), (16384, 300)])
@pytest.mark.parametrize("stream", [BF, F32])
def test_many_wide_rows(L, n, m, stream):
    """Blocks that stay, with several threads to a row."""
    x, w, b = normal(1, m, n, std=2.0, mean=0.5, dtype=stream), normal(2, n, std=0.3, mean=1.0), normal(3, n, dtype=F32)
    y, stats = L.norm_forward(x, w, b)
    dy = normal(4, m, n)
    verify(x, w, b, 1e-5, y, stats, dy, x, L.norm_backward(dy, x, w, stats, residual=x, grad_dtype=F32))


@pytest.mark.parametrize("n", [96, 99, 14000])
def test_what_is_not_needed(L, n):
    m = 50
    x, w, dy = normal(1, m, n), normal(2, n), normal(4, m, n)
    _, stats = L.norm_forward(x, w)
    full = L.norm_backward(dy, x, w, stats)
    for i in range(8):
        need = dict(need_dx=bool(i & 1), need_dw=bool(i & 2), need_db=bool(i & 4))
        for got, want, wanted in zip(L.norm_backward(dy, x, w, stats, **need), full, need.values()):
            assert (got is None) == (not wanted) and (got is None or torch.equal(got, want))
    y, stats = L.norm_forward(x)
    verify(x, None, None, 1e-5, y, stats, dy, None, L.norm_backward(dy, x, None, stats))


def test_layouts_and_places(L):
    """Views with rows apart, on and off the 16-byte grid; results inside larger arrays and over the inputs that may be."""
    m, n = 45, 256
    x, dy, r, w, b = normal(1, m, n), normal(2, m, n), normal(3, m, n), normal(4, n), normal(5, n)
    y, stats = L.norm_forward(x, w, b)
    want = L.norm_backward(dy, x, w, stats, residual=r, grad_dtype=F32)
    for shift in (0, 8, 1, 3):
        def place(t):
            big = torch.full((m + 2, n + 24), 9.0, dtype=t.dtype, device=DEV)
            view = big[1:m + 1, shift:shift + n]
            view.copy_(t)
            return big, view
        gy, vy = place(y)
        vy.zero_()
        got = L.norm_forward(place(x)[1], w, b, out=vy)
        assert got.out is vy
        verify(x, w, b, 1e-5, vy, got.stats)
        gdx, vdx = place(x)
        arena = torch.full((2 * n + 100,), 9.0, device=DEV)
        dw, db = arena[shift:shift + n], arena[n + 50 + shift:2 * n + 50 + shift]
        L.norm_backward(place(dy)[1], place(x)[1], w, got.stats, residual=place(r)[1], dx=vdx, dw=dw, db=db, grad_dtype=F32)
        verify(x, w, b, 1e-5, vy, got.stats, dy, r, (vdx, dw, db))
        for big in (gy, gdx):
            edge = torch.ones_like(big, dtype=torch.bool)
            edge[1:m + 1, shift:shift + n] = False
            assert bool((big[edge] == 9).all())
        assert bool((arena[shift + n:n + 50 + shift] == 9).all()) and bool((arena[2 * n + 50 + shift:] == 9).all())
    again = dy.clone()
    L.norm_backward(again, x, w, stats, residual=r, dx=again)
    assert torch.equal(again, want[0])
    again = r.clone()
    L.norm_backward(dy, x, w, stats, residual=again, dx=again)
    assert torch.equal(again, want[0])
    again = x.clone()
    L.norm_forward(again, w, b, out=again)
    assert torch.equal(again, y)


def test_values(L):
    """Constant rows (h = 0), a mean far from 0 (the squares of the centred values are summed, not the values' own), the ends of
    the types, NaN and infinities, which spoil their own row and, of the sums over rows, their columns."""
    n = 512
    x = torch.full((3, n), 7.0, dtype=BF, device=DEV)
    b = normal(1, n)
    y, stats = L.norm_forward(x, None, b)
    assert torch.equal(y, b.expand(3, n)) and bool((stats[0] == 7).all())
    x = normal(2, 40, n, std=1.0, mean=3000.0, dtype=F32)
    y, stats = L.norm_forward(x, None, None, out_dtype=F32)
    verify(x, None, None, 1e-5, y, stats)
    x = normal(3, 6, n)
    clean, _ = L.norm_forward(x)
    dy, w = normal(4, 6, n), normal(5, n)
    bad = x.clone()
    bad[2, 100], bad[4, 7] = float("nan"), float("inf")
    y, stats = L.norm_forward(bad)
    for row in range(6):
        assert bool(y[row].isnan().all()) if row in (2, 4) else torch.equal(y[row], clean[row])
    dx, dw, db = L.norm_backward(dy, bad, w, stats)
    assert bool(dx[[2, 4]].isnan().all()) and not dx[[0, 1, 3, 5]].isnan().any() and bool(dw.isnan().all()) and not db.isnan().any()
    tiny = torch.zeros(2, n, dtype=F32, device=DEV)
    tiny[:, ::2] = 1e-30
    y, stats = L.norm_forward(tiny, eps=1e-5)
    assert bool(torch.isfinite(y).all()) and bool(((stats[1] - 1e5 ** 0.5).abs() <= 2.0 ** -22 * 1e5 ** 0.5).all())
    zero = torch.zeros(2, n, device=DEV)
    assert bool(L.norm_forward(zero, eps=0.0).out.isnan().all())  # 0 times 1 / 0


def test_gradient_against_differences(L):
    m, n = 5, 60
    x, w, dy = normal(1, m, n, dtype=F32), normal(2, n, dtype=F32), normal(3, m, n, dtype=F32)
    _, stats = L.norm_forward(x, w, out_dtype=F32)
    dx, dw, db = L.norm_backward(dy, x, w, stats, grad_dtype=F32)

    def value(x, w, b):
        c = x - x.mean(1, keepdim=True)
        return ((c / torch.sqrt((c * c).mean(1, keepdim=True) + 1e-5) * w + b) * dy.to(F64)).sum()

    args = [x.to(F64), w.to(F64), torch.zeros(n, dtype=F64, device=DEV)]
    for i, g in enumerate((dx, dw, db)):
        step = normal(7 + i, *args[i].shape, dtype=F64)
        up, down = list(args), list(args)
        up[i], down[i] = args[i] + 1e-5 * step, args[i] - 1e-5 * step
        want = float(value(*up) - value(*down)) / 2e-5
        assert abs(float((g.to(F64) * step).sum()) - want) <= 1e-5 * float(g.to(F64).norm() * step.norm())


def test_no_rows(L):
    x = torch.empty(0, 64, dtype=BF, device=DEV)
    y, stats = L.norm_forward(x)
    assert y.shape == (0, 64) and stats.shape == (2, 0)
    dw = torch.full((64,), 3.0, dtype=BF, device=DEV)
    dx, dw, db = L.norm_backward(x, x, None, stats, dw=dw)
    assert dx.shape == (0, 64) and bool((dw == 0).all()) and bool((db == 0).all())


def test_same_bits_streams_and_graphs(L):
    m, n = 3000, 768
    x, w, dy = normal(1, m, n), normal(2, n), normal(3, m, n)

    def both():
        y, stats = L.norm_forward(x, w)
        return (y, stats, *L.norm_backward(dy, x, w, stats))

    want = both()
    assert all(torch.equal(a, b) for a, b in zip(both(), want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = both()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    x.copy_(normal(8, m, n))
    dy.copy_(normal(9, m, n))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, both()))


def test_more_than_2_31_elements(L):
    m, n = 1_100_000, 2048
    x = torch.zeros(m, n, dtype=BF, device=DEV)
    x[-3:] = normal(1, 3, n)
    y, stats = L.norm_forward(x)
    small, few = L.norm_forward(x[-3:].clone())
    assert torch.equal(y[-3:], small) and torch.equal(stats[:, -3:], few)
    dx, dw, _ = L.norm_backward(x, x, None, stats, need_db=False)
    sdx, sdw, _ = L.norm_backward(x[-3:].clone(), x[-3:].clone(), None, few, need_db=False)
    assert torch.equal(dx[-3:], sdx) and torch.equal(dw, sdw)


def test_refusals(L):
    x, w = normal(1, 8, 64), normal(2, 64)
    y, stats = L.norm_forward(x, w)
    for a, kw in (((x.half(),), {}), ((x[0],), {}), ((x.t(),), {}), ((x, w[:5]), {}), ((x, w.half()), {}), ((x, w, w[:3]), {}), ((x.cpu(),), {}), ((x[:, ::2],), {}),
                  ((x,), dict(out_dtype=torch.float16)), ((x,), dict(out=y[:3])), ((x,), dict(out=y.half())), (([1],), {})):
        with pytest.raises(ValueError):
            L.norm_forward(*a, **kw)
    for eps in (-1.0, float("nan"), float("inf")):
        with pytest.raises(L.DlionError):
            L.norm_forward(x, eps=eps)
    for a, kw in (((y[:3], x, w, stats), {}), ((y, x, w, stats[:1]), {}), ((y, x, w, stats.half()), {}), ((y, x, w, torch.zeros(8, 2, device=DEV).t()), {}),
                  ((y, x, w, stats), dict(residual=x.float())), ((y, x, w, stats), dict(dx=x.float())), ((y, x, w, stats), dict(dw=w.float())),
                  ((y, x, w, stats), dict(db=w[:4])), ((y, x, w, stats), dict(grad_dtype=torch.float16)), ((y, x, w, stats), dict(workspace=torch.zeros(1, device=DEV)))):
        with pytest.raises(ValueError):
            L.norm_backward(*a, **kw)
