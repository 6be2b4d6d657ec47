import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs an MI355X (gfx950) GPU")
    config.addinivalue_line("markers", "slow: long-running CPU test")


def pytest_collection_modifyitems(items):
    for item in items:
        if item.nodeid.endswith("test_gpu_pages.py::test_update[19]"):
            # its pool has too few pages, and it holds the outcome in which row 92 (1 token) goes on in
            # place in a page that row 248 (113 tokens, no page left for its copy) still holds; the right
            # one: test_gpu_pages_short.py::test_short_updates[19]
            item.add_marker(pytest.mark.xfail(reason="holds an outcome that loses a row's token", strict=True))
