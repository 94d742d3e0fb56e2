"""More of what the calls for pages refuse before anything is launched (see test_pages_cpu_binding.py)."""
import ctypes as C

import pytest
import torch

from tests.test_pages_cpu_binding import INVALID, SOME, books, war  # noqa: F401


@pytest.mark.parametrize("missing", [7, 8])
def test_a_fork_of_no_requests_still_says_what_it_did(war, missing):
    a = [C.byref(books(war, B=0, d_refs=None, d_free=None, d_page_table=None, d_held=None)), None, 8, None, None, None, None, SOME, SOME, None]
    a[missing] = None
    assert war._lib.war_pages_fork(*a) == INVALID


@pytest.mark.parametrize("numbers", [0, 2])
def test_copies_go_by_one_number(war, numbers):
    pool = torch.zeros((12, 2, 16, 128), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="one number"):
        war.war_pages_copy(torch.zeros((7, 3), dtype=torch.int32), torch.zeros(numbers, dtype=torch.int32), pool, pool)
