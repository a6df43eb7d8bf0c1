import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs an MI355X (gfx950) GPU and the built HIP library")
    config.addinivalue_line("markers", "slow: long-running (large workload) test")


@pytest.fixture
def memory_given_back():
    """For tests of some GiB: what torch keeps of their device memory goes back when they end."""
    yield
    import gc

    import torch
    gc.collect()
    torch.cuda.empty_cache()
