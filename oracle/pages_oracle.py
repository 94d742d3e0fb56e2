"""The books of a paged cache in plain Python (test infrastructure): requests as lists of page numbers, one request after the other.

The paper rolls every prompt out several times (Section 5.3: four and eight rollouts); it does not describe the cache's pages.  Rules:

    grow      a request wants pages until its prefix + N positions have some; the lowest free page comes first, requests in order; the
              first request whose pages are not all there ends it for all behind it that want any
    fork      requests become copies of others as they were before: full pages shared, the partly filled page copied, or handed
              over to the lowest request that takes a request which is itself replaced
    free      a page is free once nobody holds it
    compact   the highest used page moves to the lowest free one, while that lies below it
    groups    running requests with the same page at one place of their prefixes, and what their tables have in common from the front
"""
from __future__ import annotations

from collections import Counter
from dataclasses import dataclass, field
from typing import List


@dataclass
class Books:
    num_pages: int
    width: int                                   # entries of a page table's row
    rows: List[List[int]]                        # pages that each request holds
    prefix: List[int]
    tail: List[List[int]]
    tail_len: List[int]
    entries: List[List[int]] = field(default_factory=list)

    def refs(self) -> List[int]:
        c = Counter(p for row in self.rows for p in row)
        return [c.get(p, 0) for p in range(self.num_pages)]

    def free(self) -> List[int]:
        held = {p for row in self.rows for p in row}
        return [p for p in range(self.num_pages) if p not in held]


def grow(b: Books, N: int, page: int) -> List[int]:
    granted, full = [], False
    for i, row in enumerate(b.rows):
        want = -(-(b.prefix[i] + N) // page) - len(row)
        if b.tail_len[i] < 0 or want + len(row) > b.width:
            granted.append(0)
            continue
        if want <= 0:
            granted.append(1)
            continue
        free = b.free()
        if full or want > len(free):
            full = True
            granted.append(0)
            continue
        row.extend(free[:want])
        granted.append(1)
    return granted


def fork(b: Books, src: List[int], page: int):
    """(ok, copies): copies are (from, to, rows) in the order of the requests; nothing is changed when ok is False."""
    B = len(b.rows)
    moves = {i: s for i, s in enumerate(src) if s >= 0 and s != i and s < B and b.tail_len[s] >= 0 and len(b.rows[s]) * page >= b.prefix[s]}
    refs, free = b.refs(), b.free()
    new, copies, handed = {}, [], set()
    for i, s in sorted(moves.items()):
        full, rest = divmod(b.prefix[s], page)
        row = b.rows[s][:full]
        if rest:
            last = b.rows[s][full]
            if s in moves and s not in handed and refs[last] == 1 and min(k for k, v in moves.items() if v == s) == i:
                handed.add(s)
                row = row + [last]
            else:
                if not free:
                    return False, []
                to = free.pop(0)
                copies.append((last, to, rest))
                row = row + [to]
        new[i] = (row, b.prefix[s], list(b.tail[s]), b.tail_len[s])
    for i, (row, prefix, tail, tail_len) in new.items():
        b.rows[i], b.prefix[i], b.tail[i], b.tail_len[i] = row, prefix, tail, tail_len
    return True, copies


def release(b: Books, done) -> None:
    for i, d in enumerate(done):
        if d:
            b.rows[i] = []
            b.tail_len[i] = -1


def compact(b: Books, most: int, page: int):
    """(copies, top)."""
    copies = []
    while len(copies) < most:
        used = sorted({p for row in b.rows for p in row})
        free = b.free()
        if not used or not free or used[-1] < free[0]:
            break
        a, c = used[-1], free[0]
        b.rows = [[c if p == a else p for p in row] for row in b.rows]
        copies.append((a, c, page))
    used = {p for row in b.rows for p in row}
    return copies, max(used) + 1 if used else 0


def groups(rows, prefix, running, page: int, min_shared: int):
    """(leader, shared_len); rows: page tables, of which the first prefix // page entries count."""
    at = (min_shared - 1) // page
    full = [r[: p // page] if run else [] for r, p, run in zip(rows, prefix, running)]
    leader, shared = list(range(len(rows))), [0] * len(rows)
    for i in range(len(rows)):
        if len(full[i]) <= at:
            continue
        members = [j for j in range(len(rows)) if len(full[j]) > at and full[j][at] == full[i][at]]
        common = 0
        while all(len(full[j]) > common and full[j][common] == full[members[0]][common] for j in members):
            common += 1
        if len(members) > 1 and common > at:
            leader[i], shared[i] = members[0], common * page
    return leader, shared
