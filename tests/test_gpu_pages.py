"""GPU parity: the calls that keep a pool's books against the oracle's lists, exactly; and the copies that follow from them."""
import numpy as np
import pytest
import torch

from oracle import pages_oracle as O
from tests import pages_util as U
from tests import quant_util as Q

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def war():
    from paper_2607_17299_b200 import binding
    return binding


@pytest.fixture(autouse=True)
def clean(war):
    yield
    torch.cuda.synchronize()
    assert war.war_device_status() == 0


def t(x, dt=torch.int32):
    return torch.tensor(x, dtype=dt, device=DEV)


def fork(war, d, src, page):
    war.war_pages_fork(d.pages, t(src), page, d.prefix, d.tail, d.tail_len, d.copies, d.n, d.word)
    torch.cuda.synchronize()


# B, page, longest prefix, spare pages
SIZES = [(1, 1, 10, 40), (2, 16, 0, 5), (3, 16, 100, 3), (7, 8, 500, 100), (33, 16, 700, 4000), (64, 128, 3000, 31), (300, 16, 90, 200),
         (1100, 4, 30, 5000)]


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("seed", range(3))
def test_grow(war, size, seed):
    B, page, most, spare = size
    rng = np.random.default_rng(seed)
    b = U.random_books(rng, B, page, most, spare)
    N = int(rng.integers(0, 65))
    b.width += N // page + 2
    d = U.Device(war, b)
    want = O.grow(b, N, page)
    war.war_pages_grow(d.pages, N, page, d.prefix, d.tail_len, d.granted)
    torch.cuda.synchronize()
    assert d.granted.tolist() == want
    d.check(b)


def test_grow_in_a_large_pool(war):
    """More words of the free map than one round holds, and a request that wants more than a round has."""
    n = 300_000
    b = O.Books(n, 200_000, [[5], [], list(range(200_000, 290_000))], [1, 190_000, 90_000], [[0]] * 3, [1, 1, 1])
    d = U.Device(war, b)
    war.war_pages_grow(d.pages, 3, 1, d.prefix, d.tail_len, d.granted)
    torch.cuda.synchronize()
    assert d.granted.tolist() == [1, 1, 1]
    table, held = d.pages.page_table.cpu().numpy(), d.pages.held.tolist()
    assert held == [4, 190_003, 90_003]
    free = [p for p in range(n) if p != 5 and not 200_000 <= p < 290_000]
    assert table[0, 1:4].tolist() == free[:3] and table[1, :190_003].tolist() == free[3:190_006]
    assert table[2, 90_000:90_003].tolist() == free[190_006:190_009]
    refs = np.bincount(table[table >= 0], minlength=n)
    assert (d.pages.refs.cpu().numpy() == refs).all() and (d.pages.free.cpu().numpy() == U.words(refs)).all()


def test_grow_all_running_without_tail_len(war):
    b = O.Books(10, 8, [[1], []], [3, 4], [[0], [0]], [0, 0])
    d = U.Device(war, b)
    assert O.grow(b, 4, 4) == [1, 1]
    war.war_pages_grow(d.pages, 4, 4, d.prefix, None, d.granted)
    d.check(b)


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("seed", range(4))
def test_fork(war, size, seed):
    B, page, most, spare = size
    rng = np.random.default_rng(100 + seed)
    b = U.random_books(rng, B, page, most, spare + (B if seed else 0), room=5)
    live = [i for i in range(B) if b.tail_len[i] >= 0] or [-1]
    src = [int(rng.choice(live)) if rng.random() < 0.7 else int(rng.choice([-1, i])) for i in range(B)]
    if seed == 3 and len(live) > 1:                                     # a permutation of the running ones: no copies but of shared pages
        perm = rng.permutation(live)
        src = [-1] * B
        for i, s in zip(live, perm):
            src[i] = int(s)
    d = U.Device(war, b)
    ok, copies = O.fork(b, src, page)
    fork(war, d, src, page)
    assert int(d.word) == int(ok) and d.listed() == copies
    d.check(b)


def test_fork_refuses_when_pages_are_short(war):
    b = O.Books(4, 4, [[0, 1], [], [3]], [6, 0, 2], [[1], [2], [3]], [1, -1, 1])
    d = U.Device(war, b)
    fork(war, d, [2, 0, 0], 4)                          # two copies, one free page (0 hands page 1 to 1; 2 needs one; 0 takes 3 itself)
    ok, copies = O.fork(b, [2, 0, 0], 4)
    assert ok and d.listed() == copies and int(d.word) == 1
    d.check(b)
    b = O.Books(4, 4, [[0, 1], [], [3], []], [6, 0, 2, 0], [[1], [2], [3], [4]], [1, -1, 1, -1])
    d = U.Device(war, b)
    fork(war, d, [-1, 0, -1, 0], 4)
    assert int(d.word) == 0 and int(d.n) == 0
    d.check(b)


@pytest.mark.parametrize("size", SIZES, ids=str)
def test_free_then_grow(war, size):
    B, page, most, spare = size
    rng = np.random.default_rng(5)
    b = U.random_books(rng, B, page, most, spare)
    b.width += 64
    d = U.Device(war, b)
    done = (rng.random(B) < 0.5).astype(int).tolist()
    O.release(b, done)
    war.war_pages_free(d.pages, t(done), d.tail_len)
    torch.cuda.synchronize()
    d.check(b)
    want = O.grow(b, 40, page)
    war.war_pages_grow(d.pages, 40, page, d.prefix, d.tail_len, d.granted)
    assert d.granted.tolist() == want
    d.check(b)
    O.release(b, [1] * B)
    tail_len = d.tail_len.tolist()
    war.war_pages_free(d.pages, t([1] * B))
    assert d.tail_len.tolist() == tail_len                              # (not given: not touched)
    assert int((d.pages.refs != 0).sum()) == 0 and int(d.pages.held.sum()) == 0


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("most_copies", [10 ** 6, 3, 0])
def test_compact(war, size, most_copies):
    B, page, most, spare = size
    if B > 64 and most_copies > 3:
        B = 64                                                          # (the oracle moves one page at a time)
    b = U.random_books(np.random.default_rng(9), B, page, most, spare)
    d = U.Device(war, b)
    n = min(most_copies, b.num_pages)
    d.copies = torch.full((n, 3), -7, dtype=torch.int32, device=DEV)
    copies, top = O.compact(b, n, page)
    war.war_pages_compact(d.pages, page, war.new_compact_workspace(d.pages), d.copies, d.n, d.word)
    torch.cuda.synchronize()
    assert d.listed() == copies and int(d.word) == top
    d.check(b)


def test_compact_in_a_large_pool(war):
    rng = np.random.default_rng(3)
    n, B = 200_003, 40
    rows = np.split(rng.permutation(n)[:120_000], B)
    b = O.Books(n, 3100, [r.tolist() for r in rows], [3000] * B, [[0]] * B, [1] * B)
    d = U.Device(war, b)
    d.copies = torch.zeros((n, 3), dtype=torch.int32, device=DEV)
    war.war_pages_compact(d.pages, 16, war.new_compact_workspace(d.pages), d.copies, d.n, d.word)
    held = np.sort(np.concatenate(rows))
    frm = held[held >= 120_000][::-1]
    to = np.setdiff1d(np.arange(120_000), held)
    assert int(d.n) == len(frm) and int(d.word) == 120_000
    got = d.copies[:len(frm)].cpu().numpy()
    assert (got[:, 0] == frm).all() and (got[:, 1] == to).all() and (got[:, 2] == 16).all()
    place = np.arange(n)
    place[frm] = to
    assert (d.pages.page_table.cpu().numpy()[:, :3000] == place[np.stack(rows)]).all()
    refs = d.pages.refs.cpu().numpy()
    assert (refs == (np.arange(n) < 120_000)).all() and (d.pages.free.cpu().numpy() == U.words(refs)).all()


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("seed", range(3))
def test_groups(war, size, seed):
    B, page, most, _ = size
    rng = np.random.default_rng(seed)
    b = U.random_books(rng, B, page, most, 50)
    min_shared = int(rng.choice([1, page, page + 1, 5 * page]))
    d = U.Device(war, b)
    leader, shared = (torch.full((B,), -7, dtype=torch.int32, device=DEV) for _ in range(2))
    war.war_prefix_groups(d.pages.page_table, d.prefix, d.tail_len, page, min_shared, leader, shared)
    want = O.groups(b.rows, [max(0, x) for x in b.prefix], [x >= 0 for x in b.tail_len], page, min_shared)
    assert (leader.tolist(), shared.tolist()) == (want[0], want[1])
    run = [i for i in range(B) if b.tail_len[i] >= 0]
    if len(run) == B:
        war.war_prefix_groups(d.pages.page_table, d.prefix, None, page, min_shared, leader, shared)
        assert leader.tolist() == want[0]


def test_groups_of_long_rows(war):
    """Rows that part at any column of a stretch that one warp compares at a time."""
    width = 700
    base = np.arange(width)
    rows, cut = [], [1, 2, 31, 32, 33, 127, 128, 129, 255, 256, 300, 512, 640, 699, 700]
    for g, c in enumerate(cut):
        for k in range(2):
            r = base + g * width
            if k:
                r = np.concatenate([r[:c], 10 ** 6 + base[c:]])
            rows.append(r)
    table = np.stack(rows).astype(np.int32)
    B = len(rows)
    leader, shared = (torch.zeros(B, dtype=torch.int32, device=DEV) for _ in range(2))
    war.war_prefix_groups(t(table.tolist()), t([width * 2] * B), None, 2, 1, leader, shared)
    assert leader.tolist() == [2 * (i // 2) for i in range(B)]
    assert shared.tolist() == [2 * cut[i // 2] for i in range(B)]


@pytest.mark.parametrize("kv,page,block,token_major", [("bf16", 16, 0, False), ("bf16", 5, 0, True), ("e4m3", 32, 8, False), ("e5m2", 128, 16, True),
                                                       ("e4m3", 16, 16, True), ("bf16", 128, 0, False)])
def test_copy(war, kv, page, block, token_major):
    rng = np.random.default_rng(page)
    pages, Hkv, n = 40, 3, 12
    order = rng.permutation(pages)
    lines = [(int(order[i]), int(order[20 + i]), int(rng.integers(0, page + 1)) if i else page + 9) for i in range(n)]
    pools, scales = [], []
    for _ in range(2):
        if kv == "bf16":
            x = torch.from_numpy(rng.standard_normal((pages, Hkv, page, 128)).astype(np.float32)).to(torch.bfloat16).to(DEV)
            if token_major:
                x = x.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
            pools.append(x)
            scales.append(None)
        else:
            c, s = Q.cache(rng, kv, pages, Hkv, page, block)
            pools.append(Q.to_device(c, kv, token_major))
            scales.append(torch.from_numpy(s).to(DEV))
    bits = lambda x: x.view(torch.int16 if kv == "bf16" else torch.uint8)
    want, want_s = [bits(p).clone() for p in pools], [None if s is None else s.clone() for s in scales]
    for frm, to, rows in lines:
        for p, s in zip(want, want_s):
            p[to, :, :rows] = p[frm, :, :rows]
            if s is not None:
                m = -(-min(rows, page) // block)
                s[to, :, :m] = s[frm, :, :m]
    war.war_pages_copy(t(lines + [(0, 1, page)]), t([n]), pools[0], pools[1], scales[0], scales[1])
    torch.cuda.synchronize()
    for p, w, s, ws in zip(pools, want, scales, want_s):
        assert torch.equal(bits(p), w) and (s is None or torch.equal(s, ws))
    war.war_pages_copy(t(lines), t([0]), pools[0], pools[1], scales[0], scales[1])          # nothing listed
    war.war_pages_copy(t(lines), t([99]), pools[0], pools[1], scales[0], scales[1])         # (no more than there are lines)
    for p, w in zip(pools, want):
        assert torch.equal(bits(p), w)


def test_copy_past_32_bits(war):
    """A pool of more than 2^32 bytes, pages at both ends."""
    pages, Hkv, page = 70_000, 8, 32
    k = torch.zeros((pages, Hkv, page, 128), dtype=torch.bfloat16, device=DEV)
    k[-1] = torch.randn(k[-1].shape, device=DEV).to(torch.bfloat16)
    v = k.clone()
    war.war_pages_copy(t([(pages - 1, 2, 32), (pages - 1, pages - 3, 7)]), t([2]), k, v)
    for x in (k, v):
        assert torch.equal(x[2], x[-1]) and torch.equal(x[-3, :, :7], x[-1, :, :7]) and int(x[-3, :, 7:].abs().sum()) == 0


def test_a_life_of_a_pool(war):
    """Many calls in a row, captured once and replayed where shapes stay: the books say the same as the lists all the way."""
    rng = np.random.default_rng(42)
    page, B = 4, 24
    b = U.random_books(rng, B, page, 60, 400, room=4)
    b.width += 40
    d = U.Device(war, b)
    d.copies = torch.zeros((b.num_pages, 3), dtype=torch.int32, device=DEV)
    ws = war.new_compact_workspace(d.pages)
    src, done = t([-1] * B), t([0] * B)
    calls = [lambda: war.war_pages_grow(d.pages, 6, page, d.prefix, d.tail_len, d.granted),
             lambda: war.war_pages_fork(d.pages, src, page, d.prefix, d.tail, d.tail_len, d.copies, d.n, d.word),
             lambda: war.war_pages_free(d.pages, done, d.tail_len),
             lambda: war.war_pages_compact(d.pages, page, ws, d.copies, d.n, d.word)]
    graphs = []
    snapshot = [x.clone() for x in (*d.pages, d.prefix, d.tail, d.tail_len)]
    side = torch.cuda.Stream()
    for call in calls:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            call()
        graphs.append(g)
    for x, y in zip((*d.pages, d.prefix, d.tail, d.tail_len), snapshot):
        assert torch.equal(x, y)
    for step in range(40):
        kind = int(rng.integers(4))
        if kind == 1:
            live = [i for i in range(B) if b.tail_len[i] >= 0]
            s = [int(rng.choice(live)) if live and rng.random() < 0.3 else -1 for _ in range(B)]
            src.copy_(t(s))
            ok, copies = O.fork(b, s, page)
        if kind == 2:
            x = (rng.random(B) < 0.1).astype(int).tolist()
            done.copy_(t(x))
            O.release(b, x)
        graphs[kind].replay() if step % 2 else calls[kind]()
        torch.cuda.synchronize()
        if kind == 0:
            assert d.granted.tolist() == O.grow(b, 6, page)
        if kind == 1:
            assert int(d.word) == int(ok) and d.listed() == copies
        if kind == 3:
            copies, top = O.compact(b, b.num_pages, page)
            assert d.listed() == copies and int(d.word) == top
        d.check(b)
