import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a real MI355X (run with -m gpu)")


# Cases of a test that hold a wrong value: they are run as they stand, and have to differ.
_FORK = ("the model gives the continuation of a row whose last page is missing a page that nothing is copied to, so it would attend to what that page's last "
         "owner left there; test_forks_of_rows_with_missing_pages has the same calls with the entry missing in the continuation too")
WRONG = {"test_gpu_kv_pages.py::test_against_the_model[%s]" % case: _FORK
         for case in ("3-60-2-16-128-dtype1-9-12-token", "2-400-3-32-64-dtype2-40-30-head", "1-9001-1-16-64-dtype3-300-80-token")}


def pytest_collection_modifyitems(items):
    for item in items:
        reason = WRONG.get(item.nodeid.split("/")[-1])
        if reason:
            item.add_marker(pytest.mark.xfail(reason=reason, strict=True, raises=AssertionError))


@pytest.fixture(scope="session")
def oracle():
    from oracle import attn_ref
    attn_ref.build()
    return attn_ref
