"""Books that contradict themselves: a held page that refs does not count and the free map offers, pages outside the pool, and calls
for no requests.  Such books are reported, no other request's entries or pages change for them, and what the call leaves has a bit
set iff refs is 0."""
import numpy as np
import pytest
import torch

from oracle import pages_oracle as O
from tests import pages_util as U
from tests.test_gpu_pages import DEV, fork, t

pytestmark = pytest.mark.gpu
BAD_PAGE = 8


@pytest.fixture(scope="module")
def war():
    from paper_2607_17299_b200 import binding
    return binding


def uncount(d, page):
    """One entry that holds the page is not counted any more."""
    d.pages.refs[page] -= 1
    d.pages.free.copy_(torch.from_numpy(U.words(d.pages.refs.tolist())))


def agree(d):
    refs = d.pages.refs.tolist()
    assert min(refs) >= 0 and d.pages.free.tolist() == U.words(refs).tolist()
    return refs


def compact(war, d, ws, most=8, page=4):
    lines = torch.zeros((most, 3), dtype=torch.int32, device=DEV)
    war.war_pages_compact(d.pages, page, ws, lines, d.n, d.word)
    torch.cuda.synchronize()
    return [tuple(x[:2]) for x in lines[:int(d.n)].tolist()]


@pytest.mark.parametrize("left", [0, 1, 2, 3, -1, 0x7FFFFFFF])
def test_compaction_of_a_page_that_is_marked_free(war, left):
    """Whatever the workspace held before, the entry stays as it is."""
    d = U.Device(war, O.Books(4, 3, [[0], [3]], [4, 4], [[1], [2]], [1, 1]))
    uncount(d, 3)
    ws = war.new_compact_workspace(d.pages)
    ws.view(torch.int32).fill_(left)
    assert compact(war, d, ws) == [] and int(d.word) == 1
    assert war.war_device_status() == BAD_PAGE
    assert d.pages.page_table.tolist() == [[0, -1, -1], [3, -1, -1]] and agree(d) == [1, 0, 0, 0]


def test_compaction_after_another_one_with_the_same_workspace(war):
    d = U.Device(war, O.Books(6, 2, [[0], [5], [3]], [4, 4, 4], [[1], [2], [3]], [1, 1, 1]))
    ws = war.new_compact_workspace(d.pages)
    assert compact(war, d, ws) == [(5, 1), (3, 2)] and war.war_device_status() == 0
    d = U.Device(war, O.Books(6, 2, [[0], [5], [3]], [4, 4, 4], [[1], [2], [3]], [1, 1, 1]))
    uncount(d, 5)
    assert compact(war, d, ws) == [(3, 1)] and war.war_device_status() == BAD_PAGE
    assert d.pages.page_table[:, 0].tolist() == [0, 5, 1] and agree(d) == [1, 1, 0, 0, 0, 0]


@pytest.mark.parametrize("left", [0, 1, -1])
@pytest.mark.parametrize("most", [0, 1, 8])
def test_compaction_onto_a_page_that_is_held(war, left, most):
    """Below the pages in use, the free map gives the page away; its holder is reported, moved or not."""
    d = U.Device(war, O.Books(6, 2, [[0], [5], [3]], [4, 4, 4], [[1], [2], [3]], [1, 1, 1]))
    uncount(d, 0)
    ws = war.new_compact_workspace(d.pages)
    ws.view(torch.int32).fill_(left)
    assert compact(war, d, ws, most) == [(5, 0), (3, 1)][:most] and war.war_device_status() == BAD_PAGE
    assert d.pages.page_table[:, 0].tolist() == [0, 5 if most < 1 else 0, 3 if most < 2 else 1]
    agree(d)


@pytest.mark.parametrize("left", [0, -1])
def test_compaction_of_many_pages_with_a_few_uncounted(war, left):
    """Both sides of the pages in use, words of all blocks, against the counted entries alone."""
    n = 3000
    place = torch.randperm(n, generator=torch.Generator().manual_seed(3)).tolist()
    rows = [place[40 * i:40 * i + 40] for i in range(45)]
    lost = [(3, 7), (11, 0), (44, 39), (20, 20), (29, 1)]
    d = U.Device(war, O.Books(n, 50, rows, [160] * 45, [[0]] * 45, [1] * 45))
    for i, j in lost:
        uncount(d, rows[i][j])
    ws = war.new_compact_workspace(d.pages)
    ws.view(torch.int32).fill_(left)
    counted = O.Books(n, 50, [[p for j, p in enumerate(r) if (i, j) not in lost] for i, r in enumerate(rows)], [160] * 45, [[0]] * 45, [1] * 45)
    copies, top = O.compact(counted, 700, 4)
    assert compact(war, d, ws, 700) == [c[:2] for c in copies] and int(d.word) == top
    assert war.war_device_status() == BAD_PAGE and agree(d) == counted.refs()
    for i, r in enumerate(d.pages.page_table.tolist()):
        assert [p for j, p in enumerate(r[:40]) if (i, j) not in lost] == counted.rows[i], i
        assert all(r[j] == rows[i][j] for k, j in lost if k == i), i


def books():
    return O.Books(40, 6, [[3, 4, 5], [3, 4, 9], [20, 21], []], [10, 11, 8, 0], [[1], [2], [3], [4]], [1, 1, 1, -1])


def test_fork_of_a_page_that_is_not_counted(war):
    """The copies count, and the page is not given out any more."""
    d = U.Device(war, books())
    uncount(d, 20)
    fork(war, d, [-1, -1, -1, 2], 4)
    assert war.war_device_status() == BAD_PAGE and int(d.word) == 1 and int(d.n) == 0
    assert d.pages.page_table[3].tolist() == [20, 21, -1, -1, -1, -1]
    refs = agree(d)
    assert refs[20] == 1 and refs[21] == 2
    war.war_pages_grow(d.pages, 16, 4, d.prefix, d.tail_len, d.granted)
    table = d.pages.page_table.tolist()
    assert d.granted.tolist() == [0, 0, 1, 1] and [r.count(20) for r in table] == [0, 0, 1, 1]      # (26 and 27 positions: too many for a row)
    assert war.war_device_status() == BAD_PAGE


def test_fork_in_place_of_a_page_that_is_not_counted(war):
    d = U.Device(war, books())
    uncount(d, 20)
    fork(war, d, [-1, -1, 0, -1], 4)
    assert war.war_device_status() == BAD_PAGE and int(d.word) == 1 and d.listed() == [(5, 0, 2)]
    assert d.pages.page_table[2].tolist() == [3, 4, 0, -1, -1, -1]
    refs = agree(d)
    assert [refs[x] for x in (0, 3, 4, 20, 21)] == [1, 3, 3, 0, 0]


def test_fork_in_place_of_two_entries_of_which_one_is_counted(war):
    d = U.Device(war, books())
    uncount(d, 3)
    fork(war, d, [2, 2, -1, -1], 4)
    assert war.war_device_status() == BAD_PAGE
    refs = agree(d)
    assert [refs[x] for x in (3, 4, 5, 9, 20, 21)] == [0, 0, 0, 0, 3, 3]


def test_fork_that_gives_out_a_page_of_its_source(war):
    """The lowest free page is one that the source holds: it counts for both."""
    d = U.Device(war, O.Books(8, 4, [[0, 1], []], [6, 0], [[1], [2]], [1, -1]))
    uncount(d, 0)
    fork(war, d, [-1, 0], 4)
    assert war.war_device_status() == BAD_PAGE and d.listed() == [(1, 0, 2)]
    assert d.pages.page_table[1].tolist() == [0, 0, -1, -1]
    assert agree(d) == [2, 1, 0, 0, 0, 0, 0, 0]


def test_fork_that_gives_out_a_page_of_what_is_replaced(war):
    d = U.Device(war, O.Books(8, 4, [[0], [2, 3]], [4, 6], [[1], [2]], [1, 1]))
    uncount(d, 0)
    fork(war, d, [1, -1], 4)
    assert war.war_device_status() == BAD_PAGE and d.listed() == [(3, 0, 2)]
    assert d.pages.page_table.tolist() == [[2, 0, -1, -1], [2, 3, -1, -1]] and agree(d) == [1, 0, 2, 1, 0, 0, 0, 0]


@pytest.mark.parametrize("seed", range(6))
def test_forks_of_books_that_count_too_little(war, seed):
    """refs goes by the changes alone, whatever the order of the blocks: entries afterwards minus those that were not counted, or 0."""
    rng = np.random.default_rng(seed)
    B, page = int(rng.choice([5, 40, 300])), 4
    b = U.random_books(rng, B, page, 60, 3 * B, room=6)
    live = [i for i in range(B) if b.tail_len[i] >= 0]
    src = [int(rng.choice(live)) if rng.random() < 0.6 else -1 for _ in range(B)]
    d = U.Device(war, b)
    free, lost = b.free(), {}
    for i in rng.permutation(live)[:4].tolist():
        full = b.rows[i][:b.prefix[i] // page]
        full = [p for p in full if p > free[B]]                                   # (what is given out is below)
        if full:
            p = int(rng.choice(full))
            for _ in range(int(rng.integers(1, b.refs()[p] + 1)) if p not in lost else 0):
                uncount(d, p)
                lost[p] = lost.get(p, 0) + 1
    zero = [p for p in lost if int(d.pages.refs[p]) == 0]
    touched = {p for i in range(B) for p in b.rows[i] if (src[i] >= 0 and src[i] != i) or i in [s for k, s in enumerate(src) if s != k]}
    before = b.refs()
    ok, copies = O.fork(b, src, page)
    fork(war, d, src, page)
    assert ok and int(d.word) == 1 and d.listed() == copies
    after = b.refs()
    assert agree(d) == [max(0, n - lost.get(p, 0)) for p, n in enumerate(after)]
    status = war.war_device_status()
    assert status in (0, BAD_PAGE)
    if any(p in touched and before[p] != after[p] for p in zero):
        assert status == BAD_PAGE


@pytest.mark.parametrize("page", [40, -3, 0x7FFFFFFF, -2147483648])
@pytest.mark.parametrize("replaced", [False, True])
def test_fork_of_a_partly_filled_page_outside_the_pool(war, page, replaced):
    """No copy of another page's rows, and no fresh page for it: the entry is none."""
    d = U.Device(war, books())
    d.pages.page_table[0, 2] = page
    d.pages.refs[5] = 0
    d.pages.free.copy_(torch.from_numpy(U.words(d.pages.refs.tolist())))
    fork(war, d, [2 if replaced else -1, -1, 0, 0], 4)
    assert war.war_device_status() == BAD_PAGE and int(d.word) == 1 and d.listed() == []
    first = [20, 21, -1] if replaced else [3, 4, page]
    assert [r[:3] for r in d.pages.page_table.tolist()] == [first, [3, 4, 9], [3, 4, -1], [3, 4, -1]]
    assert d.pages.held.tolist() == [2 if replaced else 3, 3, 3, 3] and d.prefix.tolist() == [8 if replaced else 10, 11, 10, 10]
    refs = agree(d)
    assert [refs[x] for x in (0, 3, 4, 9, 20, 21)] == ([0, 3, 3, 1, 1, 1] if replaced else [0, 4, 4, 1, 0, 0])


@pytest.mark.parametrize("page", [40, -3])
@pytest.mark.parametrize("src", [[-1, -1, -1, 0], [2, -1, -1, 0], [2, -1, 0, -1]])
def test_fork_of_a_full_page_outside_the_pool(war, page, src):
    """The entry is copied as it is and reported, and counts nowhere."""
    d = U.Device(war, books())
    d.pages.page_table[0, 1] = page
    uncount(d, 4)
    fork(war, d, src, 4)
    assert war.war_device_status() == BAD_PAGE and int(d.word) == 1
    taker = src.index(0)
    assert d.pages.page_table[taker, :2].tolist() == [3, page] and agree(d)[4] == 1


def test_a_fork_and_its_copies_leave_the_first_page_alone(war):
    d = U.Device(war, books())
    d.pages.page_table[0, 2] = 99
    k, v = (torch.randn((40, 2, 4, 128), device=DEV).to(torch.bfloat16) for _ in range(2))
    want = k.clone(), v.clone()
    fork(war, d, [-1, -1, 1, 0], 4)                                              # (request 2: a sound one behind it)
    war.war_pages_copy(d.copies, d.n, k, v)
    assert war.war_device_status() == BAD_PAGE and d.listed() == [(9, 0, 3)]
    for x, y in zip((k, v), want):
        y[0, :, :3] = y[9, :, :3]
        assert torch.equal(x, y)


def test_a_fork_of_no_requests_leaves_no_copies(war):
    """What follows does not apply an earlier list again."""
    pages = war.new_pages(40, 0, 5, DEV)
    none, copies, n, ok = t([]), t([[1, 2, 4], [3, 4, 4]]), t([2]), t([-7])
    war.war_pages_fork(pages, none, 4, none, torch.zeros((0, 8), dtype=torch.int32, device=DEV), none, copies, n, ok)
    assert int(n) == 0 and int(ok) == 1
    k, v = (torch.randn((40, 2, 4, 128), device=DEV).to(torch.bfloat16) for _ in range(2))
    want = k.clone(), v.clone()
    war.war_pages_copy(copies, n, k, v)
    assert torch.equal(k, want[0]) and torch.equal(v, want[1]) and war.war_device_status() == 0
