"""Attention against its formulas in 64 bits.

Tolerances, element by element, worked out beside the formulas in `oracle`.  Sums of K products on the tensor cores: (K/16 + 8)
2^-22 of the sum of the products' sizes.  p and ds are rounded to bf16 as operands, results too: 2^-8 of each.  A score that
is off by e makes its weight off by e of itself; the exponential's own error, of arguments of up to 2^7 octaves in binary32, is
2^-16 with a wide margin."""
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


def sum_error(k):
    return (k / 16 + 8) * 2.0 ** -22


def one_head(q, k, v, do, causal, scale):
    """Values and tolerances of one head of one sequence (64 bits): out, lse, dq, dk, dv."""
    n, d = q.shape
    s = (q @ k.t()) * scale
    off_s = (sum_error(d) + 2.0 ** -22) * scale * (q.abs() @ k.abs().t())
    if causal:
        hide = torch.ones(n, n, device=q.device, dtype=torch.bool).triu(1)
        s = s.masked_fill(hide, -math.inf)
        off_s = off_s.masked_fill(hide, 0.0)
    lse = torch.logsumexp(s, 1)
    p = torch.exp(s - lse[:, None])
    off_row = off_s.amax(1, keepdim=True)
    off_lse = off_row[:, 0] + 2.0 ** -16 + 2.0 ** -22 * lse.abs()
    rel = 2 * off_row + 2.0 ** -16                                # of a weight, before it is rounded
    out = p @ v
    off_out = (rel + 2.0 ** -8 + sum_error(n)) * (p @ v.abs()) + 2.0 ** -8 * out.abs()
    r = {"out": (out, off_out), "lse": (lse, off_lse)}
    if do is None:
        return r
    rel = 2 * off_row + off_lse[:, None] + 2.0 ** -16
    dv = p.t() @ do
    r["dv"] = (dv, (p * (rel + 2.0 ** -8 + sum_error(n))).t() @ do.abs(), dv.abs())
    dp = do @ v.t()
    delta = (do * out).sum(1, keepdim=True)
    ds = p * (dp - delta)
    off_dp = sum_error(d) * (do.abs() @ v.abs().t())
    off_delta = (do.abs() * off_out).sum(1, keepdim=True) + 2.0 ** -20 * (do * out).abs().sum(1, keepdim=True)
    off_ds = ds.abs() * (rel + 2.0 ** -8) + p * (off_dp + off_delta) * (1 + 2.0 ** -7)
    dq, dk = scale * (ds @ k), scale * (ds.t() @ q)
    r["dq"] = (dq, scale * ((off_ds + sum_error(n) * ds.abs()) @ k.abs()) + 2.0 ** -8 * dq.abs())
    r["dk"] = (dk, scale * ((off_ds + sum_error(n) * ds.abs()).t() @ q.abs()), dk.abs())
    return r


def compare(name, got, want, tolerance):
    got = got.to(F64)
    bad = ~((got - want).abs() <= tolerance * 1.02 + 1e-30)       # 2 %: second-order terms
    assert not bad.any(), f"{name}: {int(bad.sum())} of {bad.numel()}, worst {float(((got - want).abs() / (tolerance + 1e-30)).max())} of the tolerance"


def verify(L, q, k, v, lengths, first=0, causal=True, scale=None, do=None, results=None, **kw):
    """Runs both directions and compares every sequence's every head."""
    rows, heads, dim = q.shape
    kv = k.shape[1]
    group = heads // kv
    c = dim ** -0.5 if scale is None else scale
    out, lse = L.attention_forward(q, k, v, causal=causal, scale=scale, **kw) if results is None else results[:2]
    grads = None
    if do is not None:
        grads = L.attention_backward(do, q, k, v, out, lse, causal=causal, scale=scale, **kw) if results is None else results[2:]
    at = first
    for n in lengths:
        sl = slice(at, at + n)
        at += n
        if n == 0:
            continue
        for g in range(kv):
            dk = dv = odk = odv = 0
            for h in range(g * group, (g + 1) * group):
                w = one_head(q[sl, h].to(F64), k[sl, g].to(F64), v[sl, g].to(F64), None if do is None else do[sl, h].to(F64), causal, c)
                where = f"rows {sl.start}..{sl.stop}, head {h}: "
                compare(where + "out", out[sl, h], *w["out"])
                compare(where + "lse", lse[h, sl], *w["lse"])
                if do is None:
                    continue
                compare(where + "dq", grads[0][sl, h], *w["dq"])
                dk, odk = dk + w["dk"][0], odk + w["dk"][1]
                dv, odv = dv + w["dv"][0], odv + w["dv"][1]
            if do is not None:                 # sums over the group's heads, each with its own products, rounded once
                compare(where + "dk", grads[1][sl, g], dk, odk * (1 + group * 2.0 ** -10) + 2.0 ** -8 * dk.abs())
                compare(where + "dv", grads[2][sl, g], dv, odv * (1 + group * 2.0 ** -10) + 2.0 ** -8 * dv.abs())
    return out, lse, grads


def qkv(seed, rows, heads, kv, dim, std=1.0):
    t = normal(seed, rows, heads + 2 * kv, dim, std=std)
    return t[:, :heads], t[:, heads:heads + kv], t[:, heads + kv:]


# ------------------------------------------------------------------------------------------------ one sequence
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n,heads,kv,dim", [(1, 1, 1, 64), (2, 2, 1, 128), (7, 3, 3, 8), (16, 2, 2, 40), (17, 4, 2, 72), (64, 1, 1, 64), (127, 2, 1, 128),
                                            (128, 2, 2, 64), (129, 2, 1, 64), (197, 3, 3, 64), (255, 2, 2, 96), (256, 2, 2, 128), (257, 2, 1, 80),
                                            (384, 1, 1, 128), (385, 4, 1, 64), (513, 2, 2, 128), (1000, 2, 1, 112), (1500, 1, 1, 16)])
def test_one_sequence(L, n, heads, kv, dim, causal):
    q, k, v = qkv(n + dim, n, heads, kv, dim)
    verify(L, q, k, v, [n], causal=causal, do=normal(3, n, heads, dim))


@pytest.mark.parametrize("causal", [True, False])
def test_equal_lengths(L, causal):
    q, k, v = qkv(1, 5 * 150, 4, 2, 64)
    verify(L, q, k, v, [150] * 5, causal=causal, do=normal(3, 750, 4, 64), length=150)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n,heads,kv,dim", [(1024, 2, 1, 128), (1153, 1, 1, 96), (1300, 2, 2, 72), (1025, 3, 1, 120)])
def test_long_sequences_of_wide_heads(L, n, heads, kv, dim, causal):
    """Two tiles of queries to a block: with and without a second one at the end, its rows few and many."""
    q, k, v = qkv(n + dim, n, heads, kv, dim)
    verify(L, q, k, v, [n], causal=causal, do=normal(3, n, heads, dim))


@pytest.mark.parametrize("dim,lengths,heads,kv", [(128, [2500, 0, 129, 1], 3, 1), (64, [130] * 60 + [700, 1, 128, 129], 6, 2), (128, [300] * 30, 8, 4), (128, [1100] * 5, 16, 8)])
def test_more_pieces_than_blocks(L, dim, lengths, heads, kv):
    """Blocks that take over one piece of work after another, of all lengths, from a table and by numbers alone."""
    rows = sum(lengths)
    q, k, v = qkv(dim, rows, heads, kv, dim)
    do = normal(3, rows, heads, dim)
    for causal in (True, False):
        how = [dict(offsets=torch.tensor([0] + lengths, device=DEV).cumsum(0))] + ([dict(length=lengths[0])] if len(set(lengths)) == 1 else [])
        runs = []
        for kw in how:
            f = L.attention_forward(q, k, v, causal=causal, **kw)
            runs.append((*f, *L.attention_backward(do, q, k, v, *f, causal=causal, **kw)))
        assert all(torch.equal(a, b) for r in runs for a, b in zip(r, runs[0]))
        picked = [i for i in range(len(lengths)) if i % 7 == 0 or i == len(lengths) - 1 or lengths[i] != lengths[0]]
        ends = torch.tensor([0] + lengths).cumsum(0).tolist()
        for i in picked:
            verify(L, q, k, v, [lengths[i]], ends[i], causal, do=do, results=runs[0])


# ------------------------------------------------------------------------------------------------ packed sequences
LENGTHS = [0, 1, 0, 130, 5, 0, 256, 77, 0, 128, 3, 300, 0]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dim,offset_type", [(64, torch.int32), (128, torch.int64)])
def test_packed(L, dim, offset_type, causal):
    """Sequences of every kind with rows before and behind them; what stands in rows of no sequence, and in other sequences, does
    not matter, NaN and infinities among it; those rows are zero in results that the call allocates and stay in given ones."""
    first, behind = 9, 50
    rows = first + sum(LENGTHS) + behind
    offsets = torch.tensor([first] + LENGTHS, device=DEV).cumsum(0).to(offset_type)
    q, k, v = (t.clone() for t in qkv(1, rows, 4, 2, dim))
    do = normal(3, rows, 4, dim)
    last = rows - behind
    for t in (q, k, v, do):
        t[:first] = float("nan")
        t[last:] = float("inf")
    out, lse, (dq, dk, dv) = verify(L, q, k, v, LENGTHS, first, causal, do=do, offsets=offsets)
    for t in (out, lse.t(), dq, dk, dv):
        assert bool((t[:first] == 0).all()) and bool((t[last:] == 0).all())
    mine = [torch.full_like(t, 5.0) for t in (out, lse, dq, dk, dv)]
    L.attention_forward(q, k, v, causal=causal, offsets=offsets, out=mine[0], lse=mine[1])
    L.attention_backward(do, q, k, v, mine[0], mine[1], causal=causal, offsets=offsets, dq=mine[2], dk=mine[3], dv=mine[4])
    for t, was in zip(mine, (out, lse, dq, dk, dv)):
        t, was = (t.t(), was.t()) if t.dim() == 2 else (t, was)
        assert bool((t[:first] == 5).all()) and bool((t[last:] == 5).all()) and torch.equal(t[first:last], was[first:last])
    L.attention_forward(q, k, v, causal=causal, offsets=offsets, out=mine[0], lse=mine[1], zero_rest=True)
    L.attention_backward(do, q, k, v, mine[0], mine[1], causal=causal, offsets=offsets, dq=mine[2], dk=mine[3], dv=mine[4], zero_rest=True)
    for t, was in zip(mine, (out, lse, dq, dk, dv)):
        assert torch.equal(t, was)


@pytest.mark.parametrize("causal", [True, False])
def test_a_sequence_of_nan_stays_alone(L, causal):
    """NaN in the second of three sequences, which begin and end inside tiles: the others are as without it."""
    lengths = [70, 90, 200]
    offsets = torch.tensor([0] + lengths, device=DEV, dtype=torch.int32).cumsum(0, dtype=torch.int32)
    q, k, v = (t.clone() for t in qkv(1, 360, 2, 2, 64))
    do = normal(3, 360, 2, 64)
    clean = L.attention_forward(q, k, v, causal=causal, offsets=offsets)
    clean_grads = L.attention_backward(do, q, k, v, *clean, causal=causal, offsets=offsets)
    for t in (q, k, v, do):
        t[70:160] = float("nan")
    out, lse = L.attention_forward(q, k, v, causal=causal, offsets=offsets)
    grads = L.attention_backward(do, q, k, v, out, lse, causal=causal, offsets=offsets)
    for a, b in zip((out, lse.t(), *grads), (clean.out, clean.lse.t(), *clean_grads)):
        assert torch.equal(a[:70], b[:70]) and torch.equal(a[160:], b[160:]) and bool(a[70:160].isnan().all())


def test_no_sequences_and_no_rows(L):
    q, k, v = qkv(1, 40, 2, 1, 64)
    for offsets in (torch.zeros(1, dtype=torch.int32, device=DEV), torch.zeros(4, dtype=torch.int32, device=DEV), torch.full((3,), 40, dtype=torch.int64, device=DEV)):
        out, lse = L.attention_forward(q, k, v, offsets=offsets)
        grads = L.attention_backward(q, q, k, v, out, lse, offsets=offsets)
        assert all(bool((t == 0).all()) for t in (out, lse, *grads))
    empty = q[:0], k[:0], v[:0]
    out, lse = L.attention_forward(*empty)
    assert out.shape == (0, 2, 64) and lse.shape == (2, 0)
    assert [g.shape[0] for g in L.attention_backward(q[:0], *empty, out, lse)] == [0, 0, 0]


def test_many_short_sequences(L):
    lengths = [(7 * i) % 23 for i in range(700)]
    offsets = torch.tensor([0] + lengths, device=DEV).cumsum(0)
    rows = sum(lengths)
    q, k, v = qkv(1, rows, 1, 1, 64)
    verify(L, q, k, v, lengths, do=normal(3, rows, 1, 64), offsets=offsets)


# ------------------------------------------------------------------------------------------------ values
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("order", ["ascending", "descending", "spike"])
def test_growing_maxima(L, order, causal):
    """Scores that grow or fall along the keys by far more than a weight's range, so that the running maximum moves again and
    again, in either direction of the pass."""
    n, dim = 700, 64
    q, k, v = (t.clone() for t in qkv(1, n, 1, 1, dim))
    ramp = torch.linspace(0, 60, n, device=DEV)
    if order == "descending":
        ramp = ramp.flip(0)
    if order == "spike":
        ramp = torch.where(torch.arange(n, device=DEV) % 131 == 5, 90.0, 0.0)
    q[:, 0, 0] = 8.0
    k[:, 0, 0] = ramp.to(BF)
    verify(L, q, k, v, [n], causal=causal, do=normal(3, n, 1, dim))


@pytest.mark.parametrize("scale", [1e-3, 0.5, 3.0])
def test_scale(L, scale):
    q, k, v = qkv(1, 300, 2, 1, 80)
    verify(L, q, k, v, [300], scale=scale, do=normal(3, 300, 2, 80))


def test_one_key_takes_all(L):
    """Large scores: each row's weight sits on one key, whose value comes out as it is."""
    n = 300
    q, k, v = (t.clone() for t in qkv(1, n, 1, 1, 64))
    k[:, 0] = 0
    k[torch.arange(n), 0, torch.arange(n) % 64] = 100.0
    k[64:] = -k[64:]
    q[:, 0] = k[torch.arange(n, device=DEV) % 64, 0]
    out, _ = L.attention_forward(q, k, v, causal=False)
    assert torch.equal(out[:, 0], v[torch.arange(n, device=DEV) % 64, 0])


def test_nan_and_infinite_scores(L):
    """A row of q that is NaN, or has a score of +infinity, is NaN in out and lse, and no other row is; keys with scores of
    -infinity are as if they were not there."""
    q, k, v = (t.clone() for t in qkv(1, 200, 1, 1, 64))
    want = L.attention_forward(q, k, v, causal=False)
    q[30, 0, 3] = float("nan")
    out, lse = L.attention_forward(q, k, v, causal=False)
    rest = torch.arange(200, device=DEV) != 30
    assert bool(out[30].isnan().all()) and bool(lse[0, 30].isnan()) and torch.equal(out[rest], want.out[rest]) and torch.equal(lse[:, rest], want.lse[:, rest])
    q[30, 0, 3] = 1.0
    q[:, 0, 0] = 1.0
    k[50, 0, 0] = float("-inf")
    out, _ = L.attention_forward(q, k, v, causal=False)
    less = [t[torch.arange(200, device=DEV) != 50] for t in (k, v)]
    for row in (0, 77, 199):
        s = q[row, 0].to(F64) @ less[0][:, 0].to(F64).t() / 8
        p = torch.softmax(s, 0)
        compare("out", out[row, 0], p @ less[1][:, 0].to(F64), 2.0 ** -6 * (p @ less[1][:, 0].to(F64).abs()))
    k[50, 0, 0] = float("inf")
    out, lse = L.attention_forward(q, k, v, causal=False)
    assert bool(out.isnan().all()) and bool(lse.isnan().all())


# ------------------------------------------------------------------------------------------------ layouts
def test_layouts(L):
    """Heads before rows, rows apart, heads apart, views of one product and of its gradient, a single head of any stride."""
    rows, heads, kv, dim = 150, 4, 2, 64
    want = None
    base = [t.clone() for t in qkv(1, rows, heads, kv, dim)]
    do = normal(3, rows, heads, dim)

    def by_head(t):
        return t.transpose(0, 1).contiguous().transpose(0, 1)

    def apart(t):
        big = torch.full((t.shape[0], 2, t.shape[1], t.shape[2] + 8), float("nan"), dtype=BF, device=DEV)
        view = big[:, 1, :, 8:]
        view.copy_(t)
        return view

    for how in (lambda t: t.clone(), by_head, apart):
        q, k, v = (how(t) for t in base)
        o, dq, dk, dv = (how(torch.zeros_like(t)) for t in (base[0], *base))
        L.attention_forward(q, k, v, out=o, lse=(lse := torch.empty(heads, rows + 3, device=DEV)[:, :rows]))
        L.attention_backward(how(do), q, k, v, o, lse, dq=dq, dk=dk, dv=dv)
        got = o, lse, dq, dk, dv
        if want is None:
            want = got
            verify(L, *base, [rows], do=do, results=got)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    both = torch.full((rows, heads + 2 * kv, dim), 7.0, dtype=BF, device=DEV)
    L.attention_backward(do, *base, want[0], want[1], dq=both[:, :heads], dk=both[:, heads:heads + kv], dv=both[:, heads + kv:])
    assert torch.equal(both, torch.cat(want[2:], 1))
    one = normal(1, 2 * 33, 3, 64)[::2, 1:2]
    verify(L, one, one, one, [33], do=one)


def test_rows_beyond_32_bits(L):
    """Rows whose places pass 2^31 elements."""
    rows, stride = 300, 8 * 10 ** 6
    big = torch.empty(rows * stride + 64, dtype=BF, device=DEV)
    q = torch.as_strided(big, (rows, 1, 64), (stride, 64, 1))
    q.copy_(normal(1, rows, 1, 64))
    small = q.clone()
    want = L.attention_forward(small, small, small)
    got = L.attention_forward(q, q, q)
    assert torch.equal(got.out, want.out) and torch.equal(got.lse, want.lse)
    wide = torch.as_strided(big, (rows, 1, 64), (stride, 64, 1), 64 * 1024)
    L.attention_backward(small, q, q, q, want.out, want.lse, dq=wide, dk=torch.empty_like(small), dv=torch.empty_like(small))
    assert torch.equal(wide, L.attention_backward(small, small, small, small, want.out, want.lse)[0])


# ------------------------------------------------------------------------------------------------ use
def test_gradients_against_differences(L):
    """The derivative of sum(out * do) along a direction, by differences of the 64-bit formula, against the gradients: their
    rounding is 2^-8 of each of n d terms of either sign, some sqrt(n d) of which survive: 2 % of the norms' product over sqrt(n d)
    would be 10 times that."""
    n, dim = 90, 64
    q, k, v = (t.clone() for t in qkv(1, n, 2, 1, dim))
    do = normal(3, n, 2, dim)
    out, lse = L.attention_forward(q, k, v)
    grads = L.attention_backward(do, q, k, v, out, lse)

    def value(q, k, v):
        s = torch.einsum("ihc,jc->hij", q, k[:, 0]) / math.sqrt(dim)
        s = s.masked_fill(torch.ones(n, n, device=DEV, dtype=torch.bool).triu(1), -math.inf)
        return (torch.einsum("hij,jc->ihc", torch.softmax(s, 2), v[:, 0]) * do.to(F64)).sum()

    x = [t.to(F64) for t in (q, k, v)]
    for i in range(3):
        step = normal(10 + i, *x[i].shape, dtype=F64)
        h = 1e-5
        up, down = list(x), list(x)
        up[i], down[i] = x[i] + h * step, x[i] - h * step
        want = float(value(*up) - value(*down)) / (2 * h)
        got = float((grads[i].to(F64) * step).sum())
        assert abs(got - want) <= 0.02 * float(grads[i].to(F64).norm())


def test_same_bits_every_time_and_in_any_company(L):
    """The same call gives the same bits, and a sequence the same alone as packed with others."""
    lengths = [300, 40, 500]
    offsets = torch.tensor([0] + lengths, device=DEV).cumsum(0)
    q, k, v = qkv(1, 840, 4, 1, 128)
    do = normal(3, 840, 4, 128)
    runs = []
    for _ in range(3):
        f = L.attention_forward(q, k, v, offsets=offsets)
        runs.append((*f, *L.attention_backward(do, q, k, v, *f, offsets=offsets)))
    assert all(torch.equal(a, b) for r in runs[1:] for a, b in zip(r, runs[0]))
    alone = L.attention_forward(q[340:], k[340:], v[340:])
    assert torch.equal(alone.out, runs[0][0][340:]) and torch.equal(alone.lse, runs[0][1][:, 340:])
    grads = L.attention_backward(do[340:], q[340:], k[340:], v[340:], *alone)
    assert all(torch.equal(a, b[340:]) for a, b in zip(grads, runs[0][2:]))


@pytest.mark.parametrize("rows,length,heads,dim,causal", [(64 * 197, 197, 6, 64, False), (4000, 250, 4, 128, True), (4096, 64, 8, 64, True)])
def test_many_runs_are_alike_and_no_wait_runs_out(L, rows, length, heads, dim, causal):
    q, k, v = qkv(1, rows, heads, heads, dim)
    do = normal(3, rows, heads, dim)

    def both():
        f = L.attention_forward(q, k, v, causal=causal, length=length)
        return (*f, *L.attention_backward(do, q, k, v, *f, causal=causal, length=length))

    want = both()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    for _ in range(1500):
        graph.replay()
    L.check()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_two_streams_at_once(L):
    """Two calls that run at the same time, each with its own workspace, do not disturb each other."""
    data = [(qkv(s, 2048, 8, 2, 64), normal(s + 9, 2048, 8, 64)) for s in (1, 2)]

    def both(d):
        (q, k, v), do = d
        f = L.attention_forward(q, k, v)
        return (*f, *L.attention_backward(do, q, k, v, *f))

    want = [both(d) for d in data]
    streams = [torch.cuda.Stream() for _ in data]
    torch.cuda.synchronize()
    got = [None, None]
    for _ in range(20):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i] = both(data[i])
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert all(torch.equal(a, b) for a, b in zip(g, w))


def test_rows_with_few_keys(L):
    """A sequence's first row sees one key: its weight is 1, and neither q nor k has a gradient from it but for the
    weight's error, 2^-19, times dp (2^6 here), the other operand (4) and the scale (1/8); rows that see few keys are as exact as
    others."""
    for dim in (64, 128):
        lengths = [1, 2, 3, 17, 64, 65, 128, 129]
        rows = sum(lengths)
        offsets = torch.tensor([0] + lengths, device=DEV).cumsum(0)
        q, k, v = qkv(dim, rows, 4, 2, dim)
        do = normal(3, rows, 4, dim)
        for causal in (True, False):
            out, lse = L.attention_forward(q, k, v, causal=causal, offsets=offsets)
            dq, dk, dv = L.attention_backward(do, q, k, v, out, lse, causal=causal, offsets=offsets)
            firsts = offsets[:-1] if causal else offsets[:1]
            assert torch.equal(out[firsts], v[firsts].repeat_interleave(2, 1)) and float(dq[firsts].abs().max()) <= 2.0 ** -14
            assert float(dk[0].abs().max()) <= 2.0 ** -14
            at = 0
            for n in lengths:              # the whole gradients' errors: operands and results rounded, 2^-9 each on average: 0.0028 together
                if n >= 17:
                    w = one_head(q[at:at + n, 0].to(F64), k[at:at + n, 0].to(F64), v[at:at + n, 0].to(F64), do[at:at + n, 0].to(F64), causal, dim ** -0.5)
                    assert float((dq[at:at + n, 0].to(F64) - w["dq"][0]).norm() / w["dq"][0].norm()) <= 0.0028
                at += n


def test_streams_graphs_and_workspaces(L):
    """On another stream; captured and replayed with new inputs and new offsets; a workspace of the caller's."""
    rows = 600
    q, k, v = (t.clone() for t in qkv(1, rows, 2, 2, 64))
    do = normal(3, rows, 2, 64)
    offsets = torch.tensor([0, 200, 600], device=DEV)
    want = L.attention_forward(q, k, v, offsets=offsets)
    want_grads = L.attention_backward(do, q, k, v, *want, offsets=offsets)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = L.attention_forward(q, k, v, offsets=offsets)
        grads = L.attention_backward(do, q, k, v, *got, offsets=offsets)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((*got, *grads), (*want, *want_grads)))
    space = torch.full((1 << 20,), 255, dtype=torch.uint8, device=DEV)
    got = L.attention_forward(q, k, v, offsets=offsets, workspace=space)
    assert torch.equal(got.out, want.out)
    grads = L.attention_backward(do, q, k, v, *got, offsets=offsets, workspace=space)
    assert all(torch.equal(a, b) for a, b in zip(grads, want_grads))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = L.attention_forward(q, k, v, offsets=offsets)
        grads = L.attention_backward(do, q, k, v, *got, offsets=offsets)
    for seed, cuts in ((5, [0, 1, 600]), (6, [100, 350, 500])):
        for t, s in ((q, 0), (k, 1), (v, 2), (do, 3)):
            t.copy_(normal(seed * 10 + s, *t.shape))
        offsets.copy_(torch.tensor(cuts, device=DEV))
        graph.replay()
        torch.cuda.synchronize()
        want = L.attention_forward(q, k, v, offsets=offsets)
        want_grads = L.attention_backward(do, q, k, v, *want, offsets=offsets)
        assert all(torch.equal(a, b) for a, b in zip((*got, *grads), (*want, *want_grads)))


def test_offsets_that_are_wrong_touch_nothing_outside(L):
    """Offsets outside the rows are held to them; descending ones leave everything in bounds."""
    rows = 300
    q, k, v = qkv(1, rows, 1, 1, 64)
    guard = [torch.full((rows + 64, 1, 64), 3.0, dtype=BF, device=DEV) for _ in range(4)]
    view = [g[32:-32] for g in guard]
    lse = torch.full((1, rows), 3.0, device=DEV)
    for cuts in ([-50, 100, 1 << 40], [300, 200, 0], [0, 300, 0, 300, 0, 300], [5, 5, 400]):
        offsets = torch.tensor(cuts, device=DEV)
        L.attention_forward(q, k, v, offsets=offsets, out=view[0], lse=lse)
        L.attention_backward(q, q, k, v, view[0], lse, offsets=offsets, dq=view[1], dk=view[2], dv=view[3])
        L.check()
        for g in guard:
            assert bool((g[:32] == 3).all()) and bool((g[-32:] == 3).all())
    offsets = torch.tensor([-50, 100, 1 << 40], device=DEV)
    got, want = L.attention_forward(q, k, v, offsets=offsets), L.attention_forward(q, k, v, offsets=torch.tensor([0, 100, 300], device=DEV))
    assert torch.equal(got.out, want.out)


def test_refusals(L):
    q, k, v = qkv(1, 64, 4, 2, 64)
    out, lse = L.attention_forward(q, k, v)
    bad = [dict(q=q.float()), dict(q=q[:32]), dict(k=k[:, :, :56]), dict(q=q[:, :3]), dict(q=q[0]), dict(v=v.transpose(1, 2)), dict(scale=0.0), dict(scale=-1.0),
           dict(scale=float("nan")), dict(scale=float("inf")), dict(length=7), dict(length=0), dict(length=64, offsets=torch.zeros(2, device=DEV, dtype=torch.int32)),
           dict(offsets=torch.zeros(2, dtype=torch.int32)), dict(offsets=torch.zeros(2, device=DEV)), dict(offsets=torch.zeros(4, device=DEV, dtype=torch.int32)[::2]),
           dict(out=out.float()), dict(out=out[:32]), dict(lse=lse.half()), dict(lse=lse.t().contiguous().t()), dict(q=q.cpu()), dict(k=k.expand(64, 2, 64)[:, :1].expand(64, 2, 64)),
           dict(q=normal(1, 64, 4, 68)[:, :, 4:]), dict(q=normal(1, 64, 4, 68)[:, :, :64]), dict(workspace=torch.zeros(8, device=DEV)), dict(q=[1]),
           dict(q=normal(1, 64, 4, 136), k=normal(1, 64, 2, 136), v=normal(1, 64, 2, 136)), dict(q=normal(1, 64, 4, 12), k=normal(1, 64, 2, 12), v=normal(1, 64, 2, 12))]
    for b in bad:
        args = dict(q=q, k=k, v=v)
        args.update(b)
        if "workspace" in b:
            args["offsets"] = torch.tensor([0, 64], device=DEV)
        with pytest.raises(ValueError):
            L.attention_forward(args.pop("q"), args.pop("k"), args.pop("v"), **args)
    for kw in (dict(dq=q.float()), dict(dk=q), dict(dout=out[:10]), dict(lse=lse[:, :3]), dict(out=out.to(F32)), dict(dv=torch.empty(64, 2, 64, dtype=BF))):
        args = dict(dout=out, out=out, lse=lse)
        args.update(kw)
        with pytest.raises(ValueError):
            L.attention_backward(args.pop("dout"), q, k, v, args.pop("out"), args.pop("lse"), **args)
