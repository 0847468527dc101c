"""Every form that a layer product may take, against 64 bits and with its epilogue's parts: whole tiles of either width and
of a lone block, tiles split and joined through memory, shares of a cluster, segmented sums, two products in one launch,
few rows.  Small and odd sizes that the library divides so on a GPU of 148 SMs; which kernels ran is read off the profiler's
names, so that a size that no longer reaches its form is noticed.  Tolerances: those of test_layers_gpu."""
import re

import pytest
import torch

from tests import test_layers_gpu as base
from tests.test_layers_gpu import BF, DEV, F32, F64, normal

pytestmark = pytest.mark.gpu

WHOLE, JOINED, LONG = 0, 1, 2


@pytest.fixture(scope="module")
def L():
    assert torch.cuda.is_available(), "this test needs a CUDA device"
    from paper_2404_00438_b200 import build
    build.build()
    from paper_2404_00438_b200 import layers
    yield layers
    layers.check()


def product(cg, bn, form, two=False, epilogue="General"):
    return rf"product_kernel<{cg}, {bn}, .*{epilogue}, {form}, {'(true|1)' if two else '(false|0)'}>"


def few(along_k, tokens):
    return rf"few_rows_kernel<{'(true|1)' if along_k else '(false|0)'}, {tokens}>"


def kernels(call):
    """The kernels and memsets that `call` launches, by name; skips where the profiler sees none at all, and on a GPU whose
    number of SMs divides the work otherwise."""
    from torch.profiler import ProfilerActivity, profile
    if torch.cuda.get_device_properties(0).multi_processor_count != 148:
        pytest.skip("these sizes are for 148 SMs")
    call()
    torch.cuda.synchronize()
    with profile(activities=[ProfilerActivity.CUDA, ProfilerActivity.CPU], acc_events=True) as p:
        torch.ones(1, device=DEV)
        call()
        torch.cuda.synchronize()
    names = [e.name for e in p.events() if e.device_type == torch.autograd.DeviceType.CUDA]
    if not names:
        pytest.skip("the profiler records no kernels here")
    return names


def ran(pattern, names):
    return any(re.search(pattern, n) for n in names)


# m, k, n, binary32 result, kernel, whether tiles are split
FORWARD = [
    (40, 64, 100, False, product(1, 64, WHOLE), False),
    (40, 1500, 2304, False, product(1, 64, JOINED), False),        # two shares
    (40, 2050, 100, False, product(1, 64, JOINED), False),         # four
    (33, 1500, 101, True, product(1, 64, JOINED), False),          # eight
    (130, 200, 5003, False, product(2, 128, WHOLE), False),
    (1000, 768, 1536, True, product(2, 128, WHOLE), False),
    (300, 8192, 2000, False, product(2, 128, WHOLE), True),        # two splits of every tile
    (300, 12300, 777, False, product(2, 128, WHOLE), True),        # five
    (4100, 64, 4100, False, product(2, 256, WHOLE), False),
    (4096, 768, 8190, True, product(2, 256, WHOLE), False),
    (520, 6200, 8200, False, product(2, 256, WHOLE), True),        # one round whole, the rest in two splits
    (40, 12300, 5003, False, product(2, 256, WHOLE), True),        # three splits of every tile
    (40, 2050, 2304, True, product(2, 192, LONG), False),
    (300, 8192, 2000, True, product(2, 192, LONG), True),
    (300, 4100, 8200, True, product(2, 192, LONG), True),          # one round whole, the rest in five splits
    (40, 12300, 100, True, product(2, 192, LONG), True),
]
FEW = [(9, 768, 777, True, 2), (10, 2048, 1001, True, 2), (16, 520, 333, True, 2), (8, 2048, 777, True, 1),
       (10, 777, 520, False, 1), (16, 2048, 1001, False, 1), (11, 4100, 64, False, 1)]


def operands(m, k, n, transposed):
    w = normal(2, n, k, std=k ** -0.5).t() if transposed else normal(2, k, n, std=k ** -0.5)
    return normal(1, m, k), w


@pytest.mark.parametrize("m,k,n,f32,kernel,split", FORWARD)
def test_forward_kernel(L, m, k, n, f32, kernel, split):
    x, w = operands(m, k, n, False)
    names = kernels(lambda: L.linear_forward(x, w, out_dtype=F32 if f32 else BF))
    assert ran(kernel, names), names
    assert ran("(?i)memset", names) == split, names                # the tickets of split tiles


@pytest.mark.parametrize("kind,transposed", [("none", False), ("gelu", True), ("silu", False), ("relu", True)])
@pytest.mark.parametrize("m,k,n,f32,kernel,split", FORWARD)
def test_forward_form(L, m, k, n, f32, kernel, split, kind, transposed):
    base.test_forward(L, m, k, n, kind, transposed, f32)


@pytest.mark.parametrize("keep", ["bf16", "8bit"])
@pytest.mark.parametrize("m,k,n,f32,kernel,split", [c for c in FORWARD if not c[3]])
def test_kept_form(L, m, k, n, f32, kernel, split, keep):
    base.test_kept(L, m, k, n, keep)


@pytest.mark.parametrize("m,k,n,along_k,tokens", FEW)
def test_few_rows(L, m, k, n, along_k, tokens):
    x, w = operands(m, k, n, along_k)
    assert ran(few(along_k, tokens), kernels(lambda: L.linear_forward(x, w)))
    for kind in ("none", "gelu", "silu", "relu"):
        for f32 in (False, True):
            base.test_forward(L, m, k, n, kind, along_k, f32)
    for keep in ("bf16", "8bit"):
        base.test_kept(L, m, k, n, keep)


# m, k, n, binary32 gradients, the kernel that has both products
BACKWARD = [
    (40, 64, 100, False, product(1, 64, WHOLE, True)),
    (257, 768, 1024, False, product(1, 64, WHOLE, True)),
    (200, 2050, 257, False, product(2, 128, WHOLE, True)),
    (2100, 700, 900, False, product(2, 128, WHOLE, True)),
    (2100, 700, 900, True, product(2, 192, LONG, True)),
    (520, 2050, 520, False, product(2, 256, WHOLE, True)),
    (2100, 2050, 2050, False, product(2, 256, WHOLE, True)),       # more tiles than pairs in either product
    (2100, 2050, 2050, True, product(2, 192, LONG, True)),
    (4096, 768, 2304, False, product(2, 256, WHOLE, True)),
]


@pytest.mark.parametrize("m,k,n,f32,kernel", BACKWARD)
def test_backward_kernel(L, m, k, n, f32, kernel):
    u, dy, w = normal(1, m, k), normal(2, m, n), normal(3, k, n)
    names = kernels(lambda: L.linear_backward(dy, w, u, grad_dtype=F32 if f32 else BF))
    assert ran(kernel, names), names


@pytest.mark.parametrize("kind,eight_bits,transposed", [("none", False, False), ("gelu", True, False), ("silu", False, True), ("relu", True, True)])
@pytest.mark.parametrize("m,k,n,f32,kernel", BACKWARD)
def test_backward_form(L, m, k, n, f32, kernel, kind, eight_bits, transposed):
    base.test_backward(L, m, k, n, kind, eight_bits, transposed, f32)


@pytest.mark.parametrize("m,k,n,f32,kernel", BACKWARD)
def test_parts_alone_and_repeated(L, m, k, n, f32, kernel):
    """dx and dw have the same bits alone and together, and in a workspace whose contents are NaN."""
    u, dy, w = normal(1, m, k), normal(2, m, n), normal(3, k, n, std=n ** -0.5)
    saved = L.checkpoint8(u)
    args = dict(act="gelu", residual=u, grad_dtype=F32 if f32 else BF)
    dx, dw, db = L.linear_backward(dy, w, saved, **args)
    assert torch.equal(L.linear_backward(dy, w, saved, need_dw=False, need_db=False, **args)[0], dx)
    assert torch.equal(L.linear_backward(dy, w, saved, need_dx=False, need_db=False, **args)[1], dw)
    workspace = torch.full((1 << 28,), 255, dtype=torch.uint8, device=DEV)
    for a, b in zip(L.linear_backward(dy, w, saved, workspace=workspace, **args), (dx, dw, db)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("m,k,n,f32,kernel,split", FORWARD)
def test_forward_repeated(L, m, k, n, f32, kernel, split):
    """The same bits again, whatever the workspace held (the split sums' places and tickets are in it)."""
    x, w = operands(m, k, n, True)
    args = dict(act="silu", out_dtype=F32 if f32 else BF)
    y = L.linear_forward(x, w, **args)
    workspace = torch.full((1 << 28,), 255, dtype=torch.uint8, device=DEV)
    for _ in range(3):
        assert torch.equal(L.linear_forward(x, w, workspace=workspace, **args), y)


# m, h, v, piece, the logits' kernel, that of dx and dw where it is one
LOSS = [
    (40, 64, 100, 0, product(1, 64, WHOLE, False, "LossTile"), product(1, 64, WHOLE, True)),
    (130, 200, 5003, 0, product(2, 128, WHOLE, False, "LossTile"), None),
    (600, 64, 6001, 0, product(2, 128, WHOLE, False, "LossTile"), None),
    (40, 200, 50257, 0, product(2, 256, WHOLE, False, "LossTile"), None),
    (1100, 2050, 4099, 520, product(2, 256, WHOLE, False, "LossTile"), product(2, 128, WHOLE, True)),
    (2100, 1030, 2050, 1050, product(2, 256, WHOLE, False, "LossTile"), product(2, 256, WHOLE, True)),
]


@pytest.mark.parametrize("m,h,v,piece,kernel,both", LOSS)
def test_loss_kernel(L, m, h, v, piece, kernel, both):
    x, w = normal(1, m, h), normal(2, v, h, std=2 * h ** -0.5)
    t = (torch.arange(m, device=DEV) * 13) % v
    names = kernels(lambda: L.lm_loss(x, w, t, piece=piece))
    assert ran(kernel, names), names
    assert both is None or ran(both, names), names


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("m,h,v,piece,kernel,both", LOSS)
def test_loss_form(L, m, h, v, piece, kernel, both, f32):
    x, w = normal(1, m, h), normal(2, v, h, std=2 * h ** -0.5)
    t = (torch.arange(m, device=DEV) * 13) % v
    t[::9] = -100
    r = base.check_loss(L, x, w, t, f32=f32, piece=piece)
    workspace = torch.full((1 << 30,), 255, dtype=torch.uint8, device=DEV)
    again = L.lm_loss(x, w, t, grad_dtype=F32 if f32 else BF, piece=piece, workspace=workspace)
    for a, b in zip(r, again):
        assert torch.equal(a, b)
