"""The books of a pool where they could go wrong: the largest batch, books that contradict themselves, requests that cannot be served."""
import numpy as np
import pytest
import torch

from oracle import pages_oracle as O
from tests import pages_util as U
from tests.test_gpu_pages import DEV, fork, t

pytestmark = pytest.mark.gpu
INVALID, BAD_PAGE = 1, 8


@pytest.fixture(scope="module")
def war():
    from paper_2607_17299_b200 import binding
    return binding


def grow(war, d, N, page):
    war.war_pages_grow(d.pages, N, page, d.prefix, d.tail_len, d.granted)
    torch.cuda.synchronize()


def test_the_largest_batch(war):
    rng = np.random.default_rng(7)
    B, page = 4096, 4
    b = U.random_books(rng, B, page, 8, 9000, room=2)
    b.width += 4
    d = U.Device(war, b)
    grow(war, d, 6, page)
    assert d.granted.tolist() == O.grow(b, 6, page)
    d.check(b)
    live = [i for i in range(B) if b.tail_len[i] >= 0]
    src = [int(rng.choice(live)) if rng.random() < 0.4 else -1 for _ in range(B)]
    fork(war, d, src, page)
    ok, copies = O.fork(b, src, page)
    assert int(d.word) == ok and d.listed() == copies and ok
    d.check(b)
    leader, shared = (torch.full((B,), -7, dtype=torch.int32, device=DEV) for _ in range(2))
    war.war_prefix_groups(d.pages.page_table, d.prefix, d.tail_len, page, 1, leader, shared)
    want = O.groups(b.rows, b.prefix, [x >= 0 for x in b.tail_len], page, 1)
    assert leader.tolist() == want[0] and shared.tolist() == want[1]
    done = (rng.random(B) < 0.5).astype(int).tolist()
    O.release(b, done)
    war.war_pages_free(d.pages, t(done), d.tail_len)
    torch.cuda.synchronize()
    d.check(b)
    lines = torch.zeros((50, 3), dtype=torch.int32, device=DEV)
    war.war_pages_compact(d.pages, page, war.new_compact_workspace(d.pages), lines, d.n, d.word)
    torch.cuda.synchronize()
    copies, top = O.compact(b, 50, page)
    assert [tuple(x) for x in lines[:int(d.n)].tolist()] == copies and int(d.word) == top
    d.check(b)
    assert war.war_device_status() == 0


def books():
    return O.Books(40, 6, [[3, 4, 5], [3, 4, 9], [20, 21], []], [10, 11, 8, 0], [[1], [2], [3], [4]], [1, 1, 1, -1])


def test_entries_outside_the_pool(war):
    b = books()
    d = U.Device(war, b)
    d.pages.page_table[2, 0], d.pages.page_table[1, 2] = 40, -9
    war.war_pages_free(d.pages, t([0, 1, 1, 0]), d.tail_len)
    torch.cuda.synchronize()
    assert war.war_device_status() == BAD_PAGE
    refs = d.pages.refs.tolist()
    assert [refs[x] for x in (3, 4, 5, 9, 20, 21)] == [1, 1, 1, 1, 1, 0]        # (9 and 20 had been lost before)
    assert d.pages.held.tolist() == [3, 0, 0, 0] and (d.pages.page_table[1:3] == -1).all() and d.tail_len.tolist() == [1, -1, -1, -1]


def test_more_entries_than_counted(war):
    b = books()
    d = U.Device(war, b)
    d.pages.refs[20] = 0
    war.war_pages_free(d.pages, t([0, 0, 1, 0]), d.tail_len)
    torch.cuda.synchronize()
    assert war.war_device_status() == BAD_PAGE and int(d.pages.refs[20]) == 0
    d = U.Device(war, books())
    d.pages.refs[20] = 0
    fork(war, d, [-1, -1, 0, -1], 4)
    assert war.war_device_status() == BAD_PAGE


@pytest.mark.parametrize("held", [-1, 7])
def test_held_outside_the_row(war, held):
    d = U.Device(war, books())
    d.pages.held[1] = held
    before = d.pages.page_table[1].clone()
    war.war_pages_free(d.pages, t([0, 1, 0, 0]), d.tail_len)
    torch.cuda.synchronize()
    assert war.war_device_status() == BAD_PAGE and int(d.pages.held[1]) == held and torch.equal(d.pages.page_table[1], before)
    grow(war, d, 8, 4)
    assert war.war_device_status() == BAD_PAGE and d.granted.tolist() == [1, 0, 1, 0]
    war.war_pages_compact(d.pages, 4, war.new_compact_workspace(d.pages), d.copies, d.n, d.word)
    torch.cuda.synchronize()
    assert war.war_device_status() == BAD_PAGE and torch.equal(d.pages.page_table[1], before)
    fork(war, d, [-1, -1, -1, 1], 4)                                             # as a source
    assert war.war_device_status() == INVALID and int(d.n) == 0
    fork(war, d, [-1, 0, -1, -1], 4)                                             # as what is replaced
    assert war.war_device_status() == INVALID and int(d.n) == 0


def test_bits_behind_the_last_page(war):
    """40 pages, two words: the rest of the second one is never given out."""
    for what in ("grow", "fork"):
        b = books()
        d = U.Device(war, b)
        d.pages.free[1] = -1
        guard = d.pages.refs.clone()
        if what == "grow":
            b.width = 6
            d.prefix[3], d.tail_len[3] = 0, 0
            wide = war.Pages(d.pages.refs, d.pages.free, torch.full((4, 60), -1, dtype=torch.int32, device=DEV), d.pages.held)
            wide.page_table[:, :6] = d.pages.page_table
            war.war_pages_grow(wide, 33 * 4, 4, d.prefix, d.tail_len, d.granted)     # requests 0 and 1 want 33 each: there are 34
            torch.cuda.synchronize()
            free = [x for x in range(40) if int(guard[x]) == 0]
            assert d.granted.tolist() == [1, 0, 0, 0] and wide.page_table[0, 3:36].tolist() == free[:33] and int((wide.refs > 0).sum()) == 39
        else:
            d.pages.free[0] = 0
            d.pages.free[1] = ~0xff
            fork(war, d, [-1, -1, -1, 0], 4)                                     # one copy, no page
            assert int(d.word) == 0 and int(d.n) == 0 and torch.equal(d.pages.refs, guard)
    assert war.war_device_status() == 0


def test_sources_that_are_none(war):
    for src, why in (([-1, -1, -1, 4], "no request"), ([3, -1, -1, -1], "not running"), ([-1, -1, -1, 2], "fewer pages than its prefix")):
        b = books()
        d = U.Device(war, b)
        if why.startswith("fewer"):
            d.prefix[2] = b.prefix[2] = 9
        fork(war, d, src, 4)
        assert war.war_device_status() == INVALID and int(d.word) == 1 and int(d.n) == 0, why
        d.check(b)


def test_the_same_source_for_everybody(war):
    """One of them keeps the source's partly filled page only where the source goes away itself."""
    for src in ([-1, 0, 0, 0], [2, 0, 0, 0]):
        b = books()
        d = U.Device(war, b)
        fork(war, d, src, 4)
        ok, copies = O.fork(b, src, 4)
        assert ok and d.listed() == copies
        d.check(b)
    assert war.war_device_status() == 0


def test_a_row_that_is_too_short(war):
    b = books()
    d = U.Device(war, b)
    want = O.grow(b, 14, 4)                                                      # request 1: 25 positions, 7 pages
    grow(war, d, 14, 4)
    assert war.war_device_status() == BAD_PAGE and d.granted.tolist() == want == [1, 0, 1, 0]
    d.check(b)
    d.prefix[0] = -1
    grow(war, d, 1, 4)
    assert war.war_device_status() == BAD_PAGE and d.granted.tolist() == [0, 1, 1, 0]


def test_copies_of_pages_that_are_none(war):
    k = torch.randn((8, 2, 16, 128), device=DEV).to(torch.bfloat16)
    v = torch.randn((8, 2, 16, 128), device=DEV).to(torch.bfloat16)
    want = k.clone(), v.clone()
    for x in want:
        x[5, :, :16], x[6, :, :3] = x[1], x[2, :, :3]
    war.war_pages_copy(t([[1, 5, 99], [-1, 3, 16], [1, 8, 16], [8, 4, 16], [2, 6, 3], [2, 7, 0], [2, 0, -4]]), t([7]), k, v)
    torch.cuda.synchronize()
    assert war.war_device_status() == BAD_PAGE and torch.equal(k, want[0]) and torch.equal(v, want[1])


def test_an_empty_pool_and_a_full_one(war):
    p = war.new_pages(33, 2, 40, DEV)
    prefix, granted, n, top = t([0, 0]), t([-7, -7]), t([-7]), t([-7])
    war.war_pages_compact(p, 1, war.new_compact_workspace(p), t([[0, 0, 0]]), n, top)
    assert int(n) == 0 and int(top) == 0
    war.war_pages_grow(p, 33, 1, prefix, None, granted)                          # the first takes everything
    assert granted.tolist() == [1, 0] and p.page_table[0, :33].tolist() == list(range(33)) and not p.free.any()
    war.war_pages_compact(p, 1, war.new_compact_workspace(p), t([[0, 0, 0]]), n, top)
    assert int(n) == 0 and int(top) == 33
    war.war_pages_free(p, t([1, 0]))
    assert [int(x) & 0xffffffff for x in p.free.tolist()] == [0xffffffff, 1] and not p.refs.any()
    assert war.war_device_status() == 0


def test_captured_behind_other_work(war):
    """Calls whose predecessor in a graph is a fill, a copy, a kernel of another stream or one of the set: each waits for what it is
    behind, and what follows waits for it."""
    b = books()
    b.width = 12
    d = U.Device(war, b)
    state = [x.clone() for x in (*d.pages, d.prefix, d.tail, d.tail_len)]
    back = list(zip((*d.pages, d.prefix, d.tail, d.tail_len), state))
    src, done, x, y = t([-1, -1, -1, 0]), t([0, 1, 0, 0]), torch.zeros(1 << 24, device=DEV), torch.zeros(1 << 24, device=DEV)
    leader, shared, seen = t([-7] * 4), t([-7] * 4), t([-7] * 4)
    fork(war, d, [-1] * 4, 4)                                                    # (one-time set-up of the device)
    other = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=torch.cuda.Stream()):
        main = torch.cuda.current_stream()
        for a, c in back:
            a.copy_(c)
        d.granted.zero_()
        war.war_pages_fork(d.pages, src, 4, d.prefix, d.tail, d.tail_len, d.copies, d.n, d.word)
        other.wait_stream(main)
        with torch.cuda.stream(other):
            x.add_(1)
            y.copy_(x)
            d.prefix.add_(1)                                                     # seen by the calls behind the meeting
        main.wait_stream(other)
        war.war_pages_free(d.pages, done, d.tail_len)
        war.war_pages_grow(d.pages, 3, 4, d.prefix, d.tail_len, d.granted)
        war.war_prefix_groups(d.pages.page_table, d.prefix, d.tail_len, 4, 4, leader, shared)
        seen.copy_(leader)
    ok, copies = O.fork(b, src.tolist(), 4)
    b.prefix = [v + 1 for v in b.prefix]
    O.release(b, done.tolist())
    want = O.grow(b, 3, 4)
    groups = O.groups(b.rows, b.prefix, [v >= 0 for v in b.tail_len], 4, 4)
    for _ in range(20):
        g.replay()
    torch.cuda.synchronize()
    assert ok and d.listed() == copies and d.granted.tolist() == want
    d.check(b)
    assert seen.tolist() == groups[0] and shared.tolist() == groups[1] and float(y[-1]) == 20
    assert war.war_device_status() == 0


def test_behind_an_event_of_another_stream(war):
    """Not captured: the calls wait for what their stream waits for, not only for the kernel that they are behind."""
    b = books()
    b.width = 12
    d = U.Device(war, b)
    prefix, leader, shared = d.prefix.clone(), t([-7] * 4), t([-7] * 4)
    other, x = torch.cuda.Stream(), torch.zeros(1 << 20, device=DEV)
    for k in range(1, 21):
        main = torch.cuda.current_stream()
        other.wait_stream(main)
        with torch.cuda.stream(other):
            torch.cuda._sleep(300_000)
            prefix.copy_(d.prefix + k)
        x.add_(1)
        main.wait_stream(other)
        war.war_prefix_groups(d.pages.page_table, prefix, d.tail_len, 4, 4, leader, shared)
        torch.cuda.synchronize()
        want = O.groups(b.rows, [min(v + k, 4 * len(r)) for v, r in zip(b.prefix, b.rows)], [v >= 0 for v in b.tail_len], 4, 4)
        assert (leader.tolist(), shared.tolist()) == want, k
        leader.fill_(-7)
    assert war.war_device_status() == 0
