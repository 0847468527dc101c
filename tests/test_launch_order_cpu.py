"""The order in which a kernel takes tensor memory and lets its successor start, read from the sources.

A block of the successor waits for the whole of the kernel before it; if it can have taken an SM's tensor memory before a block of
that kernel has its own, the two wait for each other without end.  So the successor may start once every block of the kernel has its
tensor memory, or where a block of it leaves no shared memory on its SM for another."""
import glob
import os
import re

import pytest

from paper_2404_00438_b200 import build as dl_build


def kernels():
    """(file, name, body) of every __global__ function."""
    for path in sorted(glob.glob(os.path.join(dl_build.CSRC, "*.cu*"))):
        text = re.sub(r"//[^\n]*", "", open(path).read())
        for m in re.finditer(r"__global__\s+void\s+(?:__launch_bounds__\((?:[^()]|\([^()]*\))*\)\s*)?(\w+)\s*\(", text):
            at = text.index("{", m.end())
            depth, end = 0, at
            while True:
                depth += {"{": 1, "}": -1}.get(text[end], 0)
                end += 1
                if depth == 0:
                    break
            yield os.path.basename(path), m.group(1), text[at:end]


TAKING = [k for k in kernels() if "tmem_alloc" in k[2]]


def test_kernels_are_found():
    assert {name for _, name, _ in TAKING} == {"attend_kernel", "query_gradient_kernel", "key_gradient_kernel", "product_kernel"}


@pytest.mark.parametrize("file,name,body", TAKING, ids=[k[1] for k in TAKING])
def test_successors_start_behind_the_allocation(file, name, body):
    if name == "product_kernel":               # alone on its SM: 227 KB is all that blocks get of one
        header = open(os.path.join(dl_build.CSRC, file)).read()
        number = {n: int(v) for n, v in re.findall(r"constexpr int (\w+) = (\d+);", header)}
        assert re.search(r"constexpr int kSmem = kRingBytes \+ kEpilogueWarps \* kStaging \+ 1024 \+ 256;", header)
        assert 227 * 1024 - (number["kRingBytes"] + number["kEpilogueWarps"] * number["kStaging"] + 1280) < 4096
        return
    starts = [m.start() for m in re.finditer("let_next_start", body)]
    taken = body.index("tmem_alloc")
    assert len(starts) == 1
    assert "__syncthreads" in body[taken:starts[0]], "the successor may start before the block has its tensor memory"
    assert starts[0] < body.index("wait_for_previous")
