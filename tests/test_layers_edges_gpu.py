"""The layer operators at the edges of what a call may hold: values at the ends of their types, operands and divisions that
the ordinary sizes do not meet.  Tolerances as in test_layers_gpu, where they are derived."""
import math

import pytest
import torch

from tests.test_layers_gpu import BF, DEV, F32, F64, check_loss, close, loss_reference, normal, sum_error

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def L():
    assert torch.cuda.is_available(), "this test needs a CUDA device"
    from paper_2404_00438_b200 import build
    build.build()
    from paper_2404_00438_b200 import layers
    yield layers
    layers.check()


def test_operand_of_more_adjacent_rows_than_one_turn_packs(L):
    """Column-major and off the 16-byte grid, with more rows than the packing grid's 65535 x 1024."""
    m = 65535 * 1024 + 3077
    x = normal(1, 2, m + 1, std=1.0).t()[:m]
    assert x.stride() == (1, m + 1) and m % 8 == 5
    w = normal(2, 2, 8)
    y = L.linear_forward(x, w)
    for a in (0, 65535 * 1024 - 2000, m - 5000):
        rows = slice(a, a + 5000)
        want = x[rows].to(F64) @ w.to(F64)
        close("y", y[rows], want, sum_error(2, x[rows].to(F64).abs() @ w.to(F64).abs()))
    db = L.linear_backward(x, w.t(), None, need_dx=False, need_dw=False, grad_dtype=F32)[2]
    want = x.to(F64).sum(0)
    assert not ((db.to(F64) - want).abs() > (m / 8 + 600) * 2.0 ** -24 * x.to(F64).abs().sum(0)).any()


@pytest.mark.parametrize("m,piece", [(100, 30), (100, 1), (101, 7), (101, 50), (104, 12), (96, 96)])
@pytest.mark.parametrize("f32", [False, True])
def test_loss_pieces_of_adjacent_rows(L, m, piece, f32):
    """Rows of x next to each other (column-major, on and off the 16-byte grid), pieces of any size: no piece may begin where a
    copy cannot."""
    x, w = normal(1, 64, m).t()[:, :50], normal(2, 130, 50)
    assert x.stride(0) == 1
    check_loss(L, x, w, torch.arange(m, device=DEV), f32=f32, piece=piece)


def test_loss_pieces_of_one_column(L):
    x, w = normal(1, 100, 1), normal(2, 130, 1)
    for piece in (1, 30, 99):
        check_loss(L, x, w, torch.arange(100, device=DEV), piece=piece)


@pytest.mark.parametrize("v", [90, 700, 5003])
def test_loss_of_a_row_with_one_infinite_logit(L, v):
    """An infinity in one group of words is not dropped when the groups are joined."""
    x, w = normal(1, 40, 64), normal(2, v, 64, std=0.2)
    t = torch.arange(40, device=DEV) * 2
    x[:, 0], w[:, 0] = 0, 2.0 ** -100
    w[33, 0], x[3, 0] = 2.0 ** 100, 2.0 ** 100                     # 2^200 for one word alone
    r = L.lm_loss(x, w, t)
    ok = [i for i in range(40) if i != 3]
    assert bool(r.rows[3].isnan()) and bool(r.dx[3].isnan().all()) and math.isnan(float(r.loss))
    assert bool(r.rows[ok].isfinite().all()) and bool(r.dx[ok].isfinite().all())


def masked_row(x, w, row, value):
    """Makes every logit of `row` equal to `value`, and leaves the other rows' as they are."""
    x[:, 0], w[:, 0] = 0, 1
    x[row] = 0
    x[row, 0] = value


@pytest.mark.parametrize("v", [90, 700, 5003])
def test_loss_of_a_row_at_the_lowest_value(L, v):
    """All words of one row at the type's lowest value: equal logits, so its loss is log v and its softmax 1 / v.  The
    exponentials' and the logarithm's errors are 2^-20, those of d 2^-8 (bf16) + 2^-11 (codes)."""
    x, w = normal(1, 40, 64), normal(2, v, 64, std=0.2)
    t = torch.arange(40, device=DEV) * 2
    low = torch.finfo(BF).min
    masked_row(x, w, 3, low)
    r = L.lm_loss(x, w, t, grad_dtype=F32, reduction="sum")
    assert abs(float(r.rows[3]) - math.log(v)) <= 2.0 ** -18 * (1 + math.log(v))
    assert bool(r.rows.isfinite().all()) and math.isfinite(float(r.loss))
    others = [i for i in range(40) if i != 3]
    loss, rows, dx, dw, d, lse, logits = loss_reference(x[others], w, t[others], -100, False)
    assert abs(float(r.loss) - float(loss) - math.log(v)) <= 1e-3 * float(loss)
    # dx of the row, column 0 excepted: there w is 1 and the sum of d cancels
    d3 = torch.full((v,), 1.0 / v, dtype=F64, device=DEV)
    d3[int(t[3])] -= 1
    W = w.to(F64)
    e = d3.abs() * (2.0 ** -8 + 2.0 ** -11)
    off = e @ W.abs() + sum_error(v, d3.abs() @ W.abs()) + 2.0 ** -8 * (d3 @ W).abs()
    assert not ((r.dx[3].to(F64) - d3 @ W).abs() > off)[1:].any()
    # column 0 of dw has the row's d times the lowest value, which nothing else comes near
    got = r.dw[:, 0].to(F64) / low
    assert not ((got - d3).abs() > e + 2.0 ** -20).any()


def test_loss_of_rows_beyond_the_codes(L):
    """Logits near both ends of binary32 keep their formulas; infinite ones make their row, and only it, NaN."""
    for v in (90, 700, 5003):
        t = torch.arange(40, device=DEV) * 2
        x, w = normal(1, 40, 64), normal(2, v, 64, std=0.2)
        x[:, 0], w[:, 0] = 0, 0
        w[17, 0], x[4, 0], x[9, 0] = 1.0, 3e38, 3e38
        t[9] = 17
        r = L.lm_loss(x, w, t, grad_dtype=F32, reduction="sum")
        big = float(torch.tensor(3e38).to(BF))
        assert abs(float(r.rows[4]) - big) <= 2.0 ** -20 * big and abs(float(r.rows[9])) <= 1e-6
        assert not ((r.dx[4].float() - (w[17].float() - w[8].float())).abs() > 2.0 ** -7 * (w[17].float().abs() + w[8].float().abs())).any()
        assert not r.dx[9].any()
        for value in (float("inf"), -float("inf"), float("nan")):
            x, w = normal(1, 40, 64), normal(2, v, 64, std=0.2)
            masked_row(x, w, 3, value)
            r = L.lm_loss(x, w, t)
            ok = [i for i in range(40) if i != 3]
            assert bool(r.rows[3].isnan()) and bool(r.rows[ok].isfinite().all()) and math.isnan(float(r.loss))
            assert bool(r.dx[3].isnan().all()) and bool(r.dx[ok].isfinite().all())


@pytest.mark.parametrize("m", [2, 40])
@pytest.mark.parametrize("kind", ["relu", "gelu", "silu"])
def test_slopes_at_the_ends_of_the_type(L, m, kind):
    """Far out an activation's slope is 0 or 1, up to the type's largest value, so du is 0 or the product itself."""
    ends = torch.tensor([-3.3895313892515355e38, -1e36, -1e30, -1000.0, 1000.0, 1e30, 1e36, 3.3895313892515355e38], device=DEV)
    u = ends.to(BF).repeat(m, 4).contiguous()
    dy, w = normal(1, m, 48), normal(2, 32, 48)
    plain = L.linear_backward(dy, w, u, need_dw=False, need_db=False)[0]
    got = L.linear_backward(dy, w, u, act=kind, need_dw=False, need_db=False)[0]
    want = torch.where(u > 0, plain, torch.zeros_like(plain))
    assert torch.equal(got, want)


def test_eight_bits_at_the_ends_of_the_type(L):
    """The largest value lies half a step above 127 steps of 2^121: it is held as those, not as infinity."""
    top, held = torch.finfo(BF).max, 127 * 2.0 ** 121
    x = torch.zeros(6, 70, dtype=BF, device=DEV)
    x[0, 3], x[1, 40], x[2, 69], x[3, 0], x[3, 1], x[4, :] = top, -top, top, -top, held, 2.0 ** 125
    x[5, 5], x[5, 6] = top, 2.0 ** 121
    c = L.checkpoint8(x)
    assert bool(L.restore8(c).isfinite().all())
    want = x.to(F64).clamp(-held, held)
    assert torch.equal(L.restore8(c).to(F64), want)
    assert int(c.q[0, 3]) == 127 and int(c.q[1, 40]) == -127


@pytest.mark.parametrize("m", [2, 40])
@pytest.mark.parametrize("v", [3.3895313892515355e38, 3.4028e38])
def test_eight_bits_of_sums_at_the_end_of_binary32(L, m, v):
    """z as a binary32 sum beyond the largest bf16 (its bias, 1.3e36, takes it there) in either kernel."""
    x, w = torch.zeros(m, 8, dtype=BF, device=DEV), torch.zeros(8, 64, dtype=BF, device=DEV)
    x[:, 0], w[0, 5], w[0, 40] = 1, torch.finfo(BF).max, -torch.finfo(BF).max
    bias = torch.zeros(64, device=DEV)
    bias[5], bias[40] = v - torch.finfo(BF).max, torch.finfo(BF).max - v
    y, kept = L.linear_forward(x, w, bias, keep="8bit", out_dtype=F32)
    z = L.restore8(kept).to(F64)
    want = torch.zeros(m, 64, dtype=F64, device=DEV)
    want[:, 5], want[:, 40] = 127 * 2.0 ** 121, -127 * 2.0 ** 121
    assert torch.equal(z, want) and bool(y.isfinite().all())


@pytest.mark.parametrize("m,k,n", [(9, 40, 48), (197, 768, 768), (2100, 700, 900), (2100, 2050, 2050), (520, 2050, 520), (3000, 100, 4000)])
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_gradients_have_the_same_bits_alone(L, m, k, n, transposed, dtype):
    """dx and dw are divided as beside each other when only one of them is asked for, in either type and order of dw."""
    u, dy = normal(1, m, k), normal(2, m, n)
    w = normal(3, n, k, std=n ** -0.5).t() if transposed else normal(3, k, n, std=n ** -0.5)
    args = dict(act="gelu", residual=u, grad_dtype=dtype)
    dx, dw, _ = L.linear_backward(dy, w, u, **args)
    assert torch.equal(L.linear_backward(dy, w, u, need_dw=False, need_db=False, **args)[0], dx)
    assert torch.equal(L.linear_backward(dy, w, u, need_dx=False, need_db=False, **args)[1], dw)


def test_long_sums_are_not_shifted(L):
    """2^18 positive products a sum, in a form whose tiles are whole: the tensor core drops what its accumulator does not
    hold, which unsegmented shifts every sum by 2^-10 of itself.  In segments of 1024 it is 2^-20, which turns the rounding of some
    2^-20 2^8 of the results by 2^-8: on average over 4096 of them 2^-20, with a deviation of 2^-20.  2^-18 is allowed."""
    m, k, n = 256, 1 << 18, 256 * 74
    x, w = torch.empty(m, k, dtype=BF, device=DEV), torch.empty(k, n, dtype=BF, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(1)
    x.uniform_(0.5, 1.5, generator=g)
    w.uniform_(0.5, 1.5, generator=g)
    y = L.linear_forward(x, w)[:64, :64].to(F64)
    want = x[:64].to(F64) @ w[:, :64].to(F64)
    assert abs(float(((y - want.to(BF).to(F64)) / want).mean())) <= 2.0 ** -18


def test_evaluation_in_several_pieces(L):
    """More rows than the loss without gradients takes at once: the same rows' losses, and one loss of them all."""
    m, h, v = 2 * 32768 + 1001, 40, 130
    for x in (normal(1, m, h), normal(1, h, m).t()):
        w, t = normal(2, v, h), torch.arange(m, device=DEV) % v
        t[::11] = -100
        for mean in (True, False):
            r = L.lm_loss(x, w, t, grads=False, reduction="mean" if mean else "sum")
            loss, rows = loss_reference(x, w, t, -100, mean)[:2]
            X, W = x.to(F64).abs(), w.to(F64).abs()
            off = 2 * sum_error(h, (X @ W.t()).amax(1)) + 2.0 ** -16 * (2 + rows.abs())
            assert not ((r.rows.to(F64) - rows).abs() > off).any()
            n = int((t != -100).sum()) if mean else 1
            assert abs(float(r.loss) - float(loss)) <= float(off.sum()) / n + 2.0 ** -18 * abs(float(loss))


@pytest.mark.parametrize("piece", [1, 50, 64, 149])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_loss_divided_and_whole(L, piece, dtype):
    """However the rows are divided: each row's loss and dx from the same terms in another division of the same sums, twice the
    bound of one against the formula; likewise the loss and dw."""
    x, w = normal(1, 150, 72), normal(2, 333, 72)
    t = torch.arange(150, device=DEV) * 2
    whole = L.lm_loss(x, w, t, grad_dtype=dtype)
    parts = L.lm_loss(x, w, t, grad_dtype=dtype, piece=piece)
    loss, rows, dx, dw, d, lse, logits = loss_reference(x, w, t, -100, True)
    X, W = x.to(F64).abs(), w.to(F64).abs()
    off = 2 * sum_error(72, (X @ W.t()).amax(1)) + 2.0 ** -16 * (1 + lse.abs() + logits.abs().amax(1) * 2.0 ** -4)
    assert not ((whole.rows.to(F64) - parts.rows.to(F64)).abs() > 2 * off).any()
    assert abs(float(whole.loss) - float(parts.loss)) <= 2 * (float(off.sum()) / 150 + 2.0 ** -18 * float(loss))
    e = d.abs() * (2.0 ** -8 + 2.0 ** -11) + (off * 1.1)[:, None] * (d.abs() + (1 / 150) * 2.0 ** -8 * (d != 0)) + 1e-19
    dx_off = 2 * (e @ W + sum_error(333, d.abs() @ W) + 2.0 ** -8 * dx.abs())
    assert not ((whole.dx.to(F64) - parts.dx.to(F64)).abs() > dx_off).any()
    dw_off = 2 * (e.t() @ X + sum_error(150, d.abs().t() @ X) + 2.0 ** (-8 if dtype is BF else -22) * dw.abs())
    assert not ((whole.dw.to(F64) - parts.dw.to(F64)).abs() > dw_off).any()


@pytest.mark.parametrize("m,h,v", [(1, 64, 7), (40, 200, 50257), (130, 200, 5003), (300, 100, 1), (257, 65, 2051)])
@pytest.mark.parametrize("mean", [True, False])
def test_loss_without_gradients(L, m, h, v, mean):
    """The evaluation's scalar against 64 bits, and its rows with the bits that the call with gradients has."""
    x, w = normal(1, m, h), normal(2, v, h, std=2 * h ** -0.5)
    t = (torch.arange(m, device=DEV) * 13) % v
    if m > 2:
        t[::7] = -100
    args = dict(reduction="mean" if mean else "sum")
    r = L.lm_loss(x, w, t, grads=False, **args)
    loss, rows, _, _, _, lse, logits = loss_reference(x, w, t, -100, mean)
    X, W = x.to(F64).abs(), w.to(F64).abs()
    off = 2 * sum_error(h, (X @ W.t()).amax(1)) + 2.0 ** -16 * (1 + lse.abs() + logits.abs().amax(1) * 2.0 ** -4)
    n = max(1, int((t != -100).sum())) if mean else 1
    assert abs(float(r.loss) - float(loss)) <= float(off.sum()) / n + 2.0 ** -18 * abs(float(loss))
    with_gradients = L.lm_loss(x, w, t, **args)
    assert torch.equal(r.rows, with_gradients.rows) and torch.equal(r.loss, with_gradients.loss)


def test_the_example_checks_its_kernels(L, monkeypatch):
    """A kernel that gave up a wait ends the training with an error instead of passing unnoticed."""
    from paper_2404_00438_b200 import dlion, example

    def gave_up():
        raise dlion.DlionError(5, "dlion_layers_check")
    monkeypatch.setattr(example.layers, "check", gave_up)
    with pytest.raises(dlion.DlionError):
        example.train(steps=1, workers=1, rows=32, words=50, width=32, hidden=32, blocks=1, report=lambda s: None)
