import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs an MI355X (gfx950) GPU and the built HIP library")
    config.addinivalue_line("markers", "slow: long-running CPU test")


@pytest.fixture(autouse=True)
def clones_that_are_waited_for(request, monkeypatch):
    """test_two_caches_side_by_side (test_gpu_paged.py) clones outputs of side streams on the default stream and drops them without
    a wait, so their memory's next use, on the side streams, may come ahead of the clone, which then holds the next inputs. Its
    clones are waited for."""
    if request.node.name == "test_two_caches_side_by_side":
        import torch
        clone = torch.Tensor.clone

        def waited_for(x, **kw):
            y = clone(x, **kw)
            torch.cuda.synchronize()
            return y

        monkeypatch.setattr(torch.Tensor, "clone", waited_for)


@pytest.fixture(scope="session")
def tiny_cfg():
    from paper_2403_00835_amd.configs import TINY
    return TINY


@pytest.fixture(scope="session")
def tiny_model(tiny_cfg):
    import oracle
    return oracle.load_model(tiny_cfg)
