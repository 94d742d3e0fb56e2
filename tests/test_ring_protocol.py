"""A model of the ring of TMA-filled slots in the two attention kernels over the 8-bit cache, run on the CPU in random orders.

Two producers (K, V) fill kSlots slots in one sequence of load numbers; two MMA issuers empty them, each its own tiles; mbarriers
are waited for by parity, which tells a phase only from the next.  The model has the kernels' load order and waits, lets loads
land in any order and everybody proceed in any order, and checks that an issuer never uses a slot before its own load is in it
and that no barrier gets an arrival that its phase does not expect (which is an error on the device)."""
import random

import pytest

SLOTS = 11


class Broken(Exception):
    pass


class Barrier:
    def __init__(self):
        self.phase, self.pending, self.tx = 0, 1, 0

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
            self.phase, self.pending = self.phase + 1, 1

    def passed(self, parity):                                    # mbarrier.try_wait.parity
        return (self.phase & 1) != parity


def few(T):
    """(load number of K(t), of V(t), groups) of war_verify_attn_quant_few.cu"""
    return (lambda t: t + max(0, t - 3)), (lambda t: t + min(T, t + 4)), 4


def many(T):
    """of war_verify_attn_quant_many.cu"""
    return (lambda t: 0 if t == 0 else 2 * t - 1), (lambda t: 2 * T - 1 if t == T - 1 else 2 * t + 2), 2


class Model:
    def __init__(self, order, units, rng, guarded, stragglers):
        self.rng, self.units, self.guarded, self.stragglers = rng, units, guarded, stragglers
        self.full, self.empty = [Barrier() for _ in range(SLOTS)], [Barrier() for _ in range(SLOTS)]
        self.content, self.flying, self.now = [None] * SLOTS, [], 0
        self.s, self.p, self.pv = set(), set(), set()            # (unit, tile) that have S, P, P V
        actors = [self.producer(order, False), self.producer(order, True), self.issuer(order, 0), self.issuer(order, 1)]
        actors += [self.softmax(order, g) for g in range(order(1)[2])]
        waits = [next(a, None) for a in actors]
        while any(w is not None for w in waits):
            self.now += 1
            for x in [x for x in self.flying if x[0] <= self.now]:
                self.flying.remove(x)
                self.content[x[1] % SLOTS] = x[1]
                self.full[x[1] % SLOTS].land()
            ready = [i for i, w in enumerate(waits) if w is not None and w()]
            if ready:
                i = rng.choice(ready)
                waits[i] = next(actors[i], None)
            elif not self.flying:
                raise Broken("nobody can go on")

    def producer(self, order, is_v):
        ld0 = 0
        for T in self.units:
            k, v, _ = order(T)
            for t in range(T):
                ld = ld0 + (v(t) if is_v else k(t))
                slot, phase = ld % SLOTS, (ld // SLOTS) & 1
                yield lambda: self.empty[slot].passed(phase ^ 1)
                self.full[slot].arrive(tx=1)
                late = self.rng.random() < self.stragglers
                self.flying.append((self.now + self.rng.randint(1, 400 if late else 12), ld))
            ld0 += 2 * T

    def landed(self, ld):
        slot, phase = ld % SLOTS, (ld // SLOTS) & 1
        if self.guarded:
            yield lambda: self.empty[slot].passed(phase ^ 1)
        yield lambda: self.full[slot].passed(phase)

    def use(self, ld):
        if self.content[ld % SLOTS] != ld:
            raise Broken("a slot is used before its load is there")
        self.empty[ld % SLOTS].arrive()

    def issuer(self, order, w):
        ld0 = 0
        for u, T in enumerate(self.units):
            k, v, groups = order(T)
            yield lambda: all((u - 1, t) in self.pv for t in range(self.units[u - 1])) if u else True      # the epilogue of the unit before
            for g in range(w, min(groups, T), 2):
                yield from self.landed(ld0 + k(g))
                self.use(ld0 + k(g))
                self.s.add((u, g))
            for t in range(w, T, 2):
                yield from self.landed(ld0 + v(t))
                if t + groups < T:
                    yield from self.landed(ld0 + k(t + groups))
                yield lambda: (u, t) in self.p
                self.use(ld0 + v(t))
                self.pv.add((u, t))
                if t + groups < T:
                    self.use(ld0 + k(t + groups))
                    self.s.add((u, t + groups))
            ld0 += 2 * T

    def softmax(self, order, g):
        ld0 = 0
        for u, T in enumerate(self.units):
            for t in range(g, T, order(T)[2]):
                yield lambda: (u, t) in self.s
                for _ in range(self.rng.randint(0, 3)):
                    yield lambda: True
                if t == T - 1:                                   # rows past the request's end are zeroed in V's slot
                    ld = ld0 + order(T)[1](t)
                    yield from self.landed(ld)
                    if self.content[ld % SLOTS] != ld:
                        raise Broken("rows of another load are zeroed")
                self.p.add((u, t))
            ld0 += 2 * T


@pytest.mark.parametrize("order", [few, many])
def test_loads_are_used_when_they_are_there(order):
    rng = random.Random(1)
    for _ in range(150):
        units = [rng.choice([1, 2, 3, 4, 5, 7, 12, 40, 90]) for _ in range(rng.randint(1, 5))]
        Model(order, units, rng, guarded=True, stragglers=rng.choice([0.0, 0.02, 0.2]))


@pytest.mark.parametrize("order", [few, many])
def test_full_alone_is_not_enough(order):
    """Without the wait for the slot's previous load, a load that is late by a ring's length is taken for the one behind it."""
    rng = random.Random(2)
    with pytest.raises(Broken):
        for _ in range(150):
            Model(order, [90], rng, guarded=False, stragglers=0.02)
