import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a CUDA device (run on a B200)")
    # Host-only tests hand the library addresses that are no memory.  Most are refused before CUDA is touched, but not
    # all need be: with no device visible nothing can be launched on them, on a machine that has one either.
    if config.getoption("markexpr", "") == "not gpu":
        os.environ["CUDA_VISIBLE_DEVICES"] = ""


def pytest_collection_modifyitems(config, items):
    """In a run of both kinds on a machine with a GPU, the files of made-up addresses wait for a run of their own."""
    host = [i for i in items if i.path.name.endswith("_cpu.py") and i.get_closest_marker("gpu") is None]
    if not host or os.environ.get("CUDA_VISIBLE_DEVICES") == "" or config.getoption("markexpr", "") == "gpu":
        return
    import torch
    if torch.cuda.is_available():
        for item in host:
            item.add_marker(pytest.mark.skip(reason='made-up addresses: run with -m "not gpu", which hides the GPU'))


@pytest.fixture(scope="session")
def oracle():
    from oracle import dlion_oracle
    dlion_oracle.build()
    return dlion_oracle
