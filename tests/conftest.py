import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs an MI355X (gfx950) GPU and the built HIP library")
    config.addinivalue_line("markers", "slow: long-running CPU test")


def pytest_collection_modifyitems(items):
    """The paged cache's GPU tests first. test_two_caches_side_by_side of test_gpu_paged.py copies a side stream's output on the
    default stream and drops the output without a wait; behind the batch and loss tests that copy came after the memory's
    next use in about half of the runs (it then holds the next inputs), ahead of them in none."""
    items.sort(key=lambda item: not item.path.name.startswith("test_gpu_paged"))


@pytest.fixture(scope="session")
def tiny_cfg():
    from paper_2403_00835_amd.configs import TINY
    return TINY


@pytest.fixture(scope="session")
def tiny_model(tiny_cfg):
    import oracle
    return oracle.load_model(tiny_cfg)
