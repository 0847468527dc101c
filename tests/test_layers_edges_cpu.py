"""Refusals of the layer operators, each by itself, in a process that sees no GPU."""
import ctypes
import glob
import os
import re

import pytest

from paper_2404_00438_b200 import build as dl_build
from tests import conftest

P = 1 << 20      # an aligned address that is no memory
EINVAL, EALIGN = 1, 2


@pytest.fixture(scope="module")
def lib():
    dl_build.build()
    from paper_2404_00438_b200 import layers
    return layers._lib


class Run:
    """What conftest asks of pytest's configuration."""
    def __init__(self, markexpr):
        self.markexpr = markexpr

    def addinivalue_line(self, name, line):
        pass

    def getoption(self, name, default=None):
        return self.markexpr if name == "markexpr" else default


def test_host_only_runs_see_no_gpu(monkeypatch):
    for markexpr, seen in (("not gpu", ""), ("gpu", "0"), ("", "0")):
        monkeypatch.setenv("CUDA_VISIBLE_DEVICES", "0")
        conftest.pytest_configure(Run(markexpr))
        assert os.environ["CUDA_VISIBLE_DEVICES"] == seen


@pytest.mark.parametrize("kw,status", [
    (dict(x_ld=39), EINVAL), (dict(q_ld=39), EINVAL), (dict(e_ld=3), EINVAL), (dict(k=0), EINVAL), (dict(m=-1), EINVAL),
    (dict(m=(1 << 30) + 1), EINVAL), (dict(k=65535 * 256 + 1, x_ld=1 << 25, q_ld=1 << 25), EINVAL), (dict(x_ld=-40), EINVAL),
    (dict(x=None), EINVAL), (dict(q=None), EINVAL), (dict(e=None), EINVAL), (dict(x=P + 1), EALIGN),
])
def test_checkpoint_and_restore_refuse(lib, kw, status):
    a = dict(x=P, x_ld=40, m=4, k=40, q=P, q_ld=40, e=P, e_ld=4)       # two blocks of exponents: rows of 4
    a.update(kw)
    assert lib.dlion_checkpoint8(a["x"], a["x_ld"], a["m"], a["k"], a["q"], a["q_ld"], a["e"], a["e_ld"], None) == status
    assert lib.dlion_restore8(a["q"], a["q_ld"], a["e"], a["e_ld"], a["m"], a["k"], a["x"], a["x_ld"], None) == status


def test_kernels_that_start_early_use_plain_loads():
    """A kernel that starts beside its predecessor lives while that one writes, which the read-only path rules out."""
    early = set()
    for path in glob.glob(os.path.join(dl_build.CSRC, "*.cu*")):
        source = open(path).read()
        if "wait_for_previous()" in source:
            early.add(os.path.basename(path))
            assert not re.search(r"__ldg\b|\.nc\b|ld_nc|__restrict__", source), path
    assert {"product.cu", "product.cuh", "few_rows.cu", "layers_linear.cu", "layers_loss.cu"} <= early


def test_evaluation_workspace_is_bounded(lib):
    """The loss without gradients holds 8 bytes a row and group of 32768 rows at most, at 50257 words not a GB."""
    from paper_2404_00438_b200 import layers
    a = dict(h=768, v=50257, x=P, x_rs=768, x_cs=1, w=P, w_rs=768, w_cs=1, targets=P, ignore_index=-100, mean=1, scale=1.0, loss=P, rows=P)
    sizes = [lib.dlion_lm_loss_workspace(ctypes.byref(layers._Loss(m=m, **a))) for m in (1 << 10, 1 << 15, 1 << 20, 1 << 30)]
    assert sizes[0] < sizes[1] == sizes[2] == sizes[3] < 1 << 29
