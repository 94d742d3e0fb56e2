"""The ring of war_verify_attn_shared_sm100.cu as a model on the CPU, run in random orders (see test_ring_protocol.py).

Loads K0 K1 V0 K2 V1 ... V(T-1) go into five slots in this order; two producers bring half of each.  Load n has barriers number
n % 8 for "landed" and "free".  Two MMA issuers either take the tiles in turn or both use every tile.  The model has the kernel's order and waits; it checks that nobody uses a slot before its load is in
it or after it was given up, that no barrier gets an arrival that its phase does not expect, and that nobody waits for ever."""
import random

import pytest

from tests.test_ring_protocol import Broken

SLOTS, BARS = 5, 8


class Barrier:
    def __init__(self, count):
        self.count, self.phase, self.pending, self.tx = count, 0, count, 0

    def arrive(self, tx=0):
        if self.pending == 0:
            raise Broken("one arrival too many")
        self.pending -= 1
        self.tx += tx
        self.settle()

    def land(self):
        self.tx -= 1
        self.settle()

    def settle(self):
        if self.pending == 0 and self.tx == 0:
            self.phase, self.pending = self.phase + 1, self.count

    def passed(self, parity):                                    # mbarrier.try_wait.parity
        return (self.phase & 1) != parity


def seq_k(t):
    return 0 if t == 0 else 2 * t - 1


def seq_v(t, T):
    return 2 * T - 1 if t == T - 1 else 2 * t + 2


class Model:
    def __init__(self, units, rng, stragglers, bars=BARS, early=False):
        """units: (tiles, both issuers use every tile); early: a slot is given up as soon as one of the two users is through"""
        self.units, self.rng, self.stragglers, self.bars, self.early = units, rng, stragglers, bars, early
        self.full, self.empty = [Barrier(2) for _ in range(bars)], [Barrier(1 if early else 2) for _ in range(bars)]
        self.content, self.halves, self.flying, self.now = [None] * SLOTS, [0] * SLOTS, [], 0
        self.s, self.p, self.pv = set(), set(), set()
        actors = [self.producer(), self.producer(), self.issuer(0), self.issuer(1), self.softmax(0), self.softmax(1)]
        waits = [next(a, None) for a in actors]
        while any(w is not None for w in waits):
            self.now += 1
            for x in [x for x in self.flying if x[0] <= self.now]:
                self.flying.remove(x)
                i = x[1] % SLOTS
                self.content[i] = None if self.content[i] not in (x[1], None) else self.content[i]
                self.halves[i] += 1
                if self.halves[i] == 2:
                    self.content[i], self.halves[i] = x[1], 0
                self.full[x[1] % bars].land()
            ready = [i for i, w in enumerate(waits) if w is not None and w()]
            if ready:
                i = rng.choice(ready)
                waits[i] = next(actors[i], None)
            elif not self.flying:
                raise Broken("nobody can go on")

    def at(self, bars, ld):
        return lambda: bars[ld % self.bars].passed((ld // self.bars) & 1)

    def producer(self):
        for ld in range(2 * sum(T for T, _ in self.units)):
            if ld >= SLOTS:
                yield self.at(self.empty, ld - SLOTS)
            self.full[ld % self.bars].arrive(tx=1)
            late = self.rng.random() < self.stragglers
            self.flying.append((self.now + self.rng.randint(1, 400 if late else 12), ld))

    def use(self, ld):
        if self.content[ld % SLOTS] != ld:
            raise Broken("a slot is used before its load is there, or after it was given up")

    def mine(self, T, pair, g):
        return range(T) if pair else range(g, T, 2)

    def through(self, u):
        T, pair = self.units[u]
        return all((u, t, g) in self.pv for g in range(2) for t in self.mine(T, pair, g))

    def issuer(self, g):
        ld0 = 0
        for u, (T, pair) in enumerate(self.units):
            def release(ld):
                if self.early:
                    if g == 0 or not pair:
                        self.empty[ld % self.bars].arrive()
                    return
                for _ in range(1 if pair else 2):
                    self.empty[ld % self.bars].arrive()
            yield lambda: u == 0 or self.through(u - 1)              # q_ready: both groups' epilogues of the unit before
            tiles = self.mine(T, pair, g)
            for t in tiles[:1]:
                yield self.at(self.full, ld0 + seq_k(t))
                self.use(ld0 + seq_k(t))
                release(ld0 + seq_k(t))
                self.s.add((u, t, g))
            for t in tiles:
                nxt = t + tiles.step
                yield self.at(self.full, ld0 + seq_v(t, T))
                if nxt < T:
                    yield self.at(self.full, ld0 + seq_k(nxt))
                for half in range(2):                                # P V of a half, the next S of that half
                    yield lambda: (u, t, g, half) in self.p
                    self.use(ld0 + seq_v(t, T))
                    if nxt < T:
                        self.use(ld0 + seq_k(nxt))
                release(ld0 + seq_v(t, T))
                self.pv.add((u, t, g))
                if nxt < T:
                    release(ld0 + seq_k(nxt))
                    self.s.add((u, nxt, g))
            ld0 += 2 * T

    def softmax(self, g):
        ld0 = 0
        for u, (T, pair) in enumerate(self.units):
            for t in self.mine(T, pair, g):
                yield lambda: (u, t, g) in self.s
                for half in range(2):
                    for _ in range(self.rng.randint(0, 3)):
                        yield lambda: True
                    if t == T - 1 and half == 0:                     # rows past the part's end are zeroed in V's slot
                        yield self.at(self.full, ld0 + seq_v(t, T))
                        self.use(ld0 + seq_v(t, T))
                    self.p.add((u, t, g, half))
            ld0 += 2 * T


def units(rng):
    return [(rng.choice([1, 1, 2, 3, 4, 5, 7, 12, 40]), rng.random() < 0.5) for _ in range(rng.randint(1, 8))]


def test_loads_are_used_when_they_are_there():
    rng = random.Random(1)
    for _ in range(300):
        Model(units(rng), rng, stragglers=rng.choice([0.0, 0.02, 0.2]))


def test_two_barriers_would_not_tell_the_loads_apart():
    rng = random.Random(2)
    with pytest.raises(Broken):
        for _ in range(300):
            Model(units(rng), rng, stragglers=0.02, bars=2)


def test_a_slot_is_free_only_when_both_users_are_through():
    rng = random.Random(3)
    with pytest.raises(Broken):
        for _ in range(300):
            Model(units(rng), rng, stragglers=0.02, early=True)


class WideningModel(Model):
    """war_verify_attn_shared_quant_sm100.cu: the producers' loads go into two slots of codes, load n with barriers n % 4; four wideners, a
    quarter of each load apiece, wait for the codes and for the ring's slot (four of them) and bring the load into it."""

    SLOTS, STAGES, STAGE_BARS = 4, 2, 4

    def __init__(self, units, rng, stragglers, bars=BARS, stage_bars=STAGE_BARS):
        self.units, self.rng, self.stragglers, self.bars, self.early, self.stage_bars = units, rng, stragglers, bars, False, stage_bars
        self.full, self.empty = [Barrier(4) for _ in range(bars)], [Barrier(2) for _ in range(bars)]
        self.codes_full, self.codes_empty = [Barrier(2) for _ in range(stage_bars)], [Barrier(4) for _ in range(stage_bars)]
        self.codes = [[None] * self.STAGES for _ in range(2)]            # each producer's half of a slot
        self.quarters = [[None] * self.SLOTS for _ in range(4)]          # each widener's quarter of a slot
        self.flying, self.now, self.s, self.p, self.pv = [], 0, set(), set(), set()
        actors = [self.producer(0), self.producer(1), *(self.widener(w) for w in range(4)), self.issuer(0), self.issuer(1), self.softmax(0), self.softmax(1)]
        waits = [next(a, None) for a in actors]
        while any(w is not None for w in waits):
            self.now += 1
            for x in [x for x in self.flying if x[0] <= self.now]:
                self.flying.remove(x)
                self.codes[x[2]][x[1] % self.STAGES] = x[1]
                self.codes_full[x[1] % stage_bars].land()
            ready = [i for i, w in enumerate(waits) if w is not None and w()]
            if ready:
                i = rng.choice(ready)
                waits[i] = next(actors[i], None)
            elif not self.flying:
                raise Broken("nobody can go on")

    def at_stage(self, bars, ld):
        return lambda: bars[ld % self.stage_bars].passed((ld // self.stage_bars) & 1)

    def producer(self, half):
        for ld in range(2 * sum(T for T, _ in self.units)):
            if ld >= self.STAGES:
                yield self.at_stage(self.codes_empty, ld - self.STAGES)
            self.codes_full[ld % self.stage_bars].arrive(tx=1)
            late = self.rng.random() < self.stragglers
            self.flying.append((self.now + self.rng.randint(1, 400 if late else 12), ld, half))

    def widener(self, w):
        for ld in range(2 * sum(T for T, _ in self.units)):
            yield self.at_stage(self.codes_full, ld)
            if ld >= self.SLOTS:
                yield self.at(self.empty, ld - self.SLOTS)
            for _ in range(self.rng.randint(0, 2)):
                yield lambda: True
            if any(c[ld % self.STAGES] != ld for c in self.codes):
                raise Broken("codes are widened before they are there, or after the slot was given up")
            self.quarters[w][ld % self.SLOTS] = ld
            self.codes_empty[ld % self.stage_bars].arrive()
            self.full[ld % self.bars].arrive()

    def use(self, ld):
        if any(q[ld % self.SLOTS] != ld for q in self.quarters):
            raise Broken("a slot is used before its load is there, or after it was given up")


def test_widened_loads_are_used_when_they_are_there():
    rng = random.Random(4)
    for _ in range(200):
        WideningModel(units(rng), rng, stragglers=rng.choice([0.0, 0.02, 0.2]))


def test_one_barrier_would_not_tell_the_codes_apart():
    rng = random.Random(5)
    with pytest.raises(Broken):
        for _ in range(300):
            WideningModel(units(rng), rng, stragglers=0.05, stage_bars=1)
