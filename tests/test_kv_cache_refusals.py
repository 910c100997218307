"""Calls around the paged cache that are refused before any HIP call, beyond those of test_kv_cache_abi.py."""
import pytest
import torch

from paper_2510_14719_amd import kv_cache as kv
from tests.test_kv_cache_abi import ALIAS, I, K, L, O, OVERFLOW, Q, V, W, batch, pages, rows  # noqa: F401


@pytest.fixture(scope="module")
def lib():
    return kv._load()


def book(**kw):
    return kv._Book(**{"ref": I, "table": I + (1 << 20), "kv_len": I + (1 << 24), "pages": 100, "rows": 9, "table_width": 20, "table_stride": 20, "page_size": 16, **kw})


def test_a_reserve_whose_pages_cannot_be_counted(lib):
    """8192 rows of 2^18 entries: with lengths that the device does not check, 2^31 pages would be wanted, and their sum is an int."""
    wide = book(rows=8192, table_width=1 << 18, table_stride=1 << 18, kv_len=I + (1 << 34))
    assert lib.kv_reserve(wide, L, L + (1 << 16), 8192, W, None) == OVERFLOW
