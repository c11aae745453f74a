import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs an MI355X (gfx950) GPU and the built HIP library")
    config.addinivalue_line("markers", "slow: full-size workload (minutes of host work)")


# Tests whose expected value is wrong, by the test that holds the right one.
WRONG_VALUE = {
    "test_gpu_kv_cache.py::test_a_copy_that_finds_no_page_changes_nothing":
        "wants status 0 for a request whose page another sequence still holds; the right values are in "
        "test_cache_grants.py::test_a_refused_sharer_that_leaves_frees_the_page_for_the_other",
}


def pytest_collection_modifyitems(items):
    for item in items:
        reason = WRONG_VALUE.get(item.nodeid.split("/")[-1])
        if reason:
            item.add_marker(pytest.mark.xfail(reason=reason, strict=True))
