import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a real MI355X (run with -m gpu)")


def _has_gpu():
    try:
        import torch
        return torch.cuda.is_available()
    except Exception:
        return False


# Tests of one file behind those of another.  The replay that is timed against the model of two copy streams comes before the tests that
# take streams of torch's pool: which hardware queues its own streams share goes by how many were made before.  What counts
# allocations comes last.
ORDER = (("test_gpu_vs_oracle_", 1), ("test_zz_", 2))


def _place(item):
    return next((at for start, at in ORDER if os.path.basename(str(item.fspath)).startswith(start)), 0)


def pytest_collection_modifyitems(config, items):
    items.sort(key=_place)   # (stable)
    if _has_gpu():
        return
    skip = pytest.mark.skip(reason="no GPU in this process")
    for item in items:
        if "gpu" in item.keywords:
            item.add_marker(skip)
