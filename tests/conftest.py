import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a real MI355X (run through the C-ABI library)")


@pytest.fixture(scope="session")
def golden_dir():
    return os.path.join(ROOT, "tests", "golden")


MADE_UP = 0x7F0000001000  # the address that host tests give to calls which they expect to be refused


def pytest_collection_modifyitems(items):
    """Host tests hand made-up addresses to calls beside each other, of which only some are refused; without a GPU the others end as errors of the launch.  Where there
    is a GPU they would run on it and fault it, so these tests are for machines without one."""
    import torch
    host = [i for i in items if getattr(i.module, "P", None) == MADE_UP and i.get_closest_marker("gpu") is None]
    if host and torch.cuda.device_count() > 0:
        for i in host:
            i.add_marker(pytest.mark.skip(reason="made-up addresses: only where there is no GPU"))
