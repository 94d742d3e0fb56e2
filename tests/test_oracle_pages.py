"""Pins of the oracle for pages: hand-worked cases, and identities that any books keep."""
import numpy as np
import pytest

from oracle import pages_oracle as O
from tests import pages_util as U


def small():
    #          request 0: prompt pages 5, 2 and a partly filled 7; request 1: the same prompt, its own page 0; request 2: empty
    return O.Books(9, 6, [[5, 2, 7], [5, 2, 0], []], [10, 9, 0], [[1], [2], [3]], [1, 1, -1])


def test_refs_and_free():
    b = small()
    assert b.refs() == [1, 0, 2, 0, 0, 2, 0, 1, 0] and b.free() == [1, 3, 4, 6, 8]


def test_grow_takes_the_lowest_pages_in_order():
    b = small()
    assert O.grow(b, 4, 4) == [1, 1, 0]                  # 14 and 13 positions: one more page each; the third is not running
    assert b.rows == [[5, 2, 7, 1], [5, 2, 0, 3], []]
    b = small()
    assert O.grow(b, 13, 4) == [1, 0, 0]                 # 23 -> six pages; then 22 -> six pages, two are left
    assert b.rows[0] == [5, 2, 7, 1, 3, 4] and b.rows[1] == [5, 2, 0]


def test_fork_shares_full_pages_and_copies_the_last():
    b = small()
    assert O.fork(b, [-1, 1, 0], 4) == (True, [(7, 1, 2)])
    assert b.rows == [[5, 2, 7], [5, 2, 0], [5, 2, 1]] and b.prefix == [10, 9, 10] and b.tail[2] == [1] and b.tail_len == [1, 1, 1]


def test_swap_needs_no_copy():
    b = small()
    assert O.fork(b, [1, 0, -1], 4) == (True, [])
    assert b.rows == [[5, 2, 0], [5, 2, 7], []] and b.prefix == [9, 10, 0]


def test_both_take_one():
    b = small()
    b.tail_len[2], b.rows[2], b.prefix[2] = 1, [8], 3
    assert O.fork(b, [2, 2, 0], 4) == (True, [(8, 1, 3)])               # 0 gets page 8 itself, 1 a copy, 2 page 7 itself
    assert b.rows == [[8], [1], [5, 2, 7]]


def test_compact():
    b = small()
    copies, top = O.compact(b, 100, 4)
    assert copies == [(7, 1, 4), (5, 3, 4)] and top == 4
    assert b.rows == [[3, 2, 1], [3, 2, 0], []]
    b = small()
    assert O.compact(b, 1, 4) == ([(7, 1, 4)], 6)


def test_groups_by_hand():
    rows = [[5, 2, 7], [5, 2, 0], [5, 9], [4, 2, 1]]
    assert O.groups(rows, [12, 9, 8, 12], [True] * 4, 4, 1) == ([0, 0, 0, 3], [4, 4, 4, 0])
    assert O.groups(rows, [12, 9, 8, 12], [True] * 4, 4, 5) == ([0, 1, 2, 3], [0, 0, 0, 0])       # (3 has page 2 there too, but not page 5)
    assert O.groups(rows[:3], [12, 9, 8], [True] * 3, 4, 5) == ([0, 0, 2], [8, 8, 0])


@pytest.mark.parametrize("seed", range(20))
def test_identities(seed):
    rng = np.random.default_rng(seed)
    page = int(rng.choice([1, 4, 16]))
    b = U.random_books(rng, int(rng.integers(1, 12)), page, 40, int(rng.integers(0, 30)), room=5)
    held = lambda x: {p for r in x.rows for p in r}
    before = U.books_copy(b)
    O.compact(b, 10 ** 6, page)
    assert held(b) == set(range(len(held(before))))                     # dense, nothing lost
    assert sorted(b.refs())[::-1][:len(held(b))] == sorted(x for x in before.refs() if x)[::-1]
    B = len(b.rows)
    before = U.books_copy(b)
    ok, copies = O.fork(b, rng.integers(-1, B, B).tolist(), page)
    if ok:
        assert not {c[1] for c in copies} & held(before) and len({c[1] for c in copies}) == len(copies)
        for i, r in enumerate(b.rows):
            if b.tail_len[i] >= 0 and b.prefix[i] % page and b.prefix[i] // page < len(r):
                mine = r[b.prefix[i] // page]                           # the page that is written next belongs to one request
                assert sum(mine in x for x in b.rows) == 1
    O.release(b, [1] * B)
    assert b.refs() == [0] * b.num_pages
