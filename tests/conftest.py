import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a real MI355X (run with -m gpu)")


def skip_made_up_addresses(items, gpus):
    """The *_abi.py files' tests without the gpu mark call the library with addresses that are none. Some of their helpers make two or
    three calls of which a change spoils only one: the others are complete, and where there is a GPU they would be launched on it."""
    for item in items:
        if gpus and item.path.name.endswith("_abi.py") and item.get_closest_marker("gpu") is None:
            item.add_marker(pytest.mark.skip(reason="calls with made-up addresses: for machines without a GPU"))


def pytest_collection_modifyitems(items):
    import torch
    skip_made_up_addresses(items, torch.cuda.device_count())


@pytest.fixture(scope="session")
def tw():
    """The ctypes binding of libtw (HIP library). Fails loudly if it is not built."""
    import paper_2505_11329_amd as pkg
    return pkg
