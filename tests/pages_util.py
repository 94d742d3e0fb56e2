"""Books of a pool for the tests: the oracle's lists and the library's arrays of the same state."""
import copy

import numpy as np
import torch

from oracle import pages_oracle as O


def random_books(rng, B, page, most_prefix, spare, prompts=3, P=8, running=0.8, room=0, width=None):
    """Groups that share full pages, some requests not running and without pages, pages shuffled over the pool."""
    at, rows, prefix, tail_len = 0, [], [], []
    common = []
    for _ in range(prompts):
        n = int(rng.integers(0, most_prefix // page + 1))
        common.append(list(range(at, at + n)))
        at += n
    for _ in range(B):
        shared = common[int(rng.integers(prompts))]
        if rng.random() >= running:
            rows.append([])
            prefix.append(int(rng.integers(-3, most_prefix)))
            tail_len.append(-1)
            continue
        pl = len(shared) * page + int(rng.integers(0, most_prefix + 1))
        own = -(-(pl + int(rng.integers(0, room + 1))) // page) - len(shared)
        rows.append(shared + list(range(at, at + own)))
        at += own
        prefix.append(pl)
        tail_len.append(int(rng.integers(0, P + 1)))
    num_pages = at + spare
    place = rng.permutation(num_pages)
    rows = [[int(place[x]) for x in r] for r in rows]
    width = max([len(r) for r in rows] + [0]) + 4 if width is None else width
    tail = rng.integers(0, 32000, (B, P)).tolist()
    return O.Books(max(1, num_pages), width, rows, prefix, tail, tail_len)


def books_copy(b):
    return copy.deepcopy(b)


class Device:
    """The arrays of a state on the device, entries behind the held ones -1."""

    def __init__(self, war, b, dev="cuda:0"):
        B = len(b.rows)
        table = np.full((B, b.width), -1, np.int32)
        for i, r in enumerate(b.rows):
            table[i, :len(r)] = r
        refs = np.array(b.refs(), np.int32)
        t = lambda x, dt=np.int32: torch.from_numpy(np.ascontiguousarray(np.asarray(x, dt))).to(dev)
        self.pages = war.Pages(t(refs), t(words(refs)), t(table), t([len(r) for r in b.rows]))
        self.prefix, self.tail, self.tail_len = t(b.prefix), t(b.tail).view(B, -1), t(b.tail_len)
        self.B = B
        self.copies = torch.full((max(1, B), 3), -7, dtype=torch.int32, device=dev)
        self.n, self.word = (torch.full((1,), -7, dtype=torch.int32, device=dev) for _ in range(2))
        self.granted = torch.full((B,), -7, dtype=torch.int32, device=dev)

    def check(self, b):
        """The arrays say what the lists say."""
        refs, free, table, held = (x.cpu().numpy() for x in self.pages)
        assert held.tolist() == [len(r) for r in b.rows]
        assert refs.tolist() == b.refs()
        assert (free == words(refs)).all()
        for i, r in enumerate(b.rows):
            assert table[i, :len(r)].tolist() == r, i
            assert (table[i, len(r):] == -1).all(), i
        assert self.prefix.tolist() == b.prefix and self.tail.tolist() == b.tail and self.tail_len.tolist() == b.tail_len

    def listed(self):
        return [tuple(x) for x in self.copies[:int(self.n)].tolist()]


def words(refs):
    bits = np.zeros(-(-len(refs) // 32) * 32, np.uint8)
    bits[:len(refs)] = np.asarray(refs) == 0
    return np.packbits(bits, bitorder="little").view(np.int32)
