import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a real MI355X (run with -m gpu)")


def pytest_collection_modifyitems(config, items):
    # a GPU test on a box without one is skipped, never silently passed
    try:
        import torch
        have = torch.cuda.is_available()
    except Exception:
        have = False
    if have:
        return
    skip = pytest.mark.skip(reason="no GPU in this process")
    for it in items:
        if "gpu" in it.keywords:
            it.add_marker(skip)


def pytest_runtest_setup(item):
    # tests that watch the allocated memory: what earlier tests left in reference cycles (tracebacks hold on to tensors) goes first,
    # not at the collector's own time in between
    if item.module.__name__.endswith("test_zz_no_alloc"):
        import gc
        gc.collect()
