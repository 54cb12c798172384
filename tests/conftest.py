import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs an MI355X (HIP device) to run")


@pytest.fixture(scope="session")
def golden_dir():
    return os.path.join(ROOT, "tests", "golden")


def pytest_collection_modifyitems(items):
    """test_gpu_wfbp.py first, however the files are named or given: its overlap
    tests need a hardware queue for each of three streams, and which of the
    process's four queues a stream gets depends on the streams made before it."""
    items.sort(key=lambda item: item.path.name != "test_gpu_wfbp.py")
