import gc
import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs an MI355X (runs through the HIP library)")
    config.addinivalue_line("markers", "slow: larger CPU-side cases")


def pytest_runtest_setup(item):
    """A test that compares the memory torch holds starts without the garbage of those before it: tensors in the cycles of
    their caught exceptions would be freed in the middle of it."""
    code = getattr(getattr(item, "function", None), "__code__", None)
    if code is not None and "memory_allocated" in code.co_names:
        gc.collect()


@pytest.fixture(scope="session")
def oracle_lib():
    import oracle

    return oracle.load()
