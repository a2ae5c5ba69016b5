import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs an MI355X (HIP) device")


@pytest.fixture(scope="session")
def orc():
    import oracle
    oracle.lib()
    return oracle


# Tests that hold a wrong value.  They run as they are and have to fail until the
# value is put right.
WRONG = {
    ("test_gpu_pages.py", "test_fork[1-"):
        "expects dsim_kv_reserve to let a row grow into whole pages that other rows hold too "
        "(of one place each, behind a length that went back): test_gpu_pages_shared.py has the rule",
}


def pytest_collection_modifyitems(items):
    for item in items:
        for (file, name), why in WRONG.items():
            if item.path.name == file and item.name.startswith(name):
                item.add_marker(pytest.mark.xfail(reason=why, raises=AssertionError, strict=True))
