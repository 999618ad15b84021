import os
import sys

import pytest

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a CUDA device (run on a B200)")


# Tests that read kernel records from torch's profiler, in the order in which they run: in front of all others.  Where some ten seconds pass between two profiles of a
# process the profiler stamps the first kernels of the next one outside its window and drops them (its own log counts them as "Out-of-range"; torch's
# kernels alone show it: 6 launches, a profile every 14 s, 1, 2, 3 and 4 records missing).  Four minutes into a session none was left.
PROFILED = ["test_gpu_traced_order.py", "test_gpu_deep_requests.py"]


def pytest_collection_modifyitems(config, items):
    items.sort(key=lambda it: PROFILED.index(it.path.name) if it.path.name in PROFILED else len(PROFILED))
    try:
        import torch
        has_gpu = torch.cuda.is_available()
    except Exception:
        has_gpu = False
    if not has_gpu:
        skip = pytest.mark.skip(reason="no CUDA device")
        for it in items:
            if "gpu" in it.keywords:
                it.add_marker(skip)
