"""Offsets that do not ascend: no sequence is worked on, whatever their number, and nothing is written."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
DEV = "cuda:0"


@pytest.fixture(scope="module")
def L():
    assert torch.cuda.is_available(), "this test needs a CUDA device"
    from paper_2404_00438_b200 import build
    build.build()
    from paper_2404_00438_b200 import layers
    yield layers
    layers.check()


def nothing_written(L, rows, dim, offsets, causal):
    g = torch.Generator(device=DEV)
    g.manual_seed(rows)
    q, k, v, do = (torch.randn(rows, 1, dim, generator=g, device=DEV).to(BF) for _ in range(4))
    results = [torch.full_like(q, 3.0) for _ in range(4)]
    lse = torch.full((1, rows), 3.0, device=DEV)
    need = 2 * 16 * (rows // 128 + min(offsets.shape[0] - 1, rows)) + 4 * rows + 4096
    # 77 in front of the workspace and behind it
    space = torch.full((need + (2 << 20),), 77, dtype=torch.uint8, device=DEV)
    inside = space[1 << 20:(1 << 20) + need]
    L.attention_forward(q, k, v, causal=causal, offsets=offsets, out=results[0], lse=lse, workspace=inside)
    L.attention_backward(do, q, k, v, results[0], lse, causal=causal, offsets=offsets, dq=results[1], dk=results[2], dv=results[3], workspace=inside)
    L.check()
    for t in (*results, lse):
        assert bool((t == 3).all())
    for t in (space[:1 << 20], space[(1 << 20) + need:]):
        assert bool((t == 77).all())


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("cuts", [[300, 200, 0], [0, 300, 0, 300, 0, 300], [0, 100, 99, 300], [0, 300, -5], [1 << 40, 0], [0] * 40 + [300, 299] + [300] * 40])
def test_few(L, cuts, causal):
    nothing_written(L, 300, 64, torch.tensor(cuts, device=DEV), causal)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("rows,count", [(131072, 4_200_000), (4096, 70_000), (131072, 31)])
def test_more_pieces_than_32_bits_count(L, rows, count, causal):
    """0, rows, 0, rows ...: half the sequences have all rows, with 4.2 million offsets 2^31 tiles."""
    offsets = torch.zeros(count, dtype=torch.int32, device=DEV)
    offsets[1::2] = rows
    nothing_written(L, rows, 8, offsets, causal)


def test_ascending_ones_beside_empty_ones(L):
    """Held to the rows, offsets may repeat: every sequence of them is worked on as if the empty ones were not there."""
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    q, k, v = (torch.randn(300, 2, 64, generator=g, device=DEV).to(BF) for _ in range(3))
    want = L.attention_forward(q, k, v, offsets=torch.tensor([0, 170, 300], device=DEV))
    for cuts in ([-4, 0, 0, 170, 170, 300, 1 << 35], [0] * 5000 + [170] * 5000 + [300] * 5000):
        got = L.attention_forward(q, k, v, offsets=torch.tensor(cuts, device=DEV))
        assert torch.equal(got.out, want.out) and torch.equal(got.lse, want.lse)
