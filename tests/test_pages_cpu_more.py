"""More of what the calls for pages refuse before anything is launched (see test_pages_cpu_binding.py)."""
import ctypes as C

import pytest

from tests.test_pages_cpu_binding import INVALID, SOME, books, war  # noqa: F401


@pytest.mark.parametrize("missing", [7, 8])
def test_a_fork_of_no_requests_still_says_what_it_did(war, missing):
    a = [C.byref(books(war, B=0, d_refs=None, d_free=None, d_page_table=None, d_held=None)), None, 8, None, None, None, None, SOME, SOME, None]
    a[missing] = None
    assert war._lib.war_pages_fork(*a) == INVALID
