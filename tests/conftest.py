import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a CUDA GPU (sm_103a) and the built CUDA library")
    config.addinivalue_line("markers", "slow: full-size parity case (minutes of CPU oracle time)")


# CPU tests that also make calls which pass their argument checks, with made-up
# addresses: without a GPU such a call ends at the device query, with one it
# would launch.
MADE_UP_ADDRESSES = {"test_caches_batches_and_workspaces_are_checked", "test_append_refusals", "test_rope_refusals"}


def pytest_collection_modifyitems(items):
    import torch
    if not torch.cuda.is_available():
        return
    skip = pytest.mark.skip(reason="made-up addresses would be launched")
    for item in items:
        if getattr(item, "originalname", None) in MADE_UP_ADDRESSES and os.path.basename(str(item.fspath)) == "test_attn_abi.py":
            item.add_marker(skip)


@pytest.fixture(scope="session")
def ppo():
    """The CPU oracle module, built on first use."""
    import oracle
    oracle.load()
    return oracle


@pytest.fixture(scope="session")
def pp():
    """The CUDA library binding; GPU tests fail (not skip) when it cannot load."""
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU test run without a CUDA device")
    from paper_2605_28283_gb300 import binding
    binding.load()
    return binding
