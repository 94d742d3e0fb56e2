"""The rings of war_verify_attn_shared_quant_sm100.cu as a model on the CPU, with its own order of waits and its scales (see
test_ring_protocol_shared.py, whose issuers wait for V(t) and K(t + 1) together).

An issuer waits for V(t) before the first half of a tile and for K(t + 1) between that half's P V and its next S.  The first producer writes the
scales of a tile into a ring of six, tile t + 1 behind its load of K(t + 1) and a unit's first tile in front of its first load, without a wait
for the ring: that its readers are through with the tile six back has to follow from the loads' own waits."""
import random

import pytest

from tests.test_ring_protocol import Broken
from tests.test_ring_protocol_shared import Barrier, WideningModel, seq_k, seq_v, units


class Model(WideningModel):
    def __init__(self, units, rng, stragglers, scale_tiles=6):
        self.scales, self.scale_bars = [None] * scale_tiles, [Barrier(1) for _ in range(scale_tiles)]
        super().__init__(units, rng, stragglers)

    def write_scales(self, tile):
        at = tile % len(self.scales)
        self.scales[at] = tile
        self.scale_bars[at].arrive()

    def producer(self, half):
        ld = tile0 = 0
        for T, _ in self.units:
            loads = {seq_k(t): t for t in range(T)}                  # which of the unit's loads are K's
            if half == 0:
                self.write_scales(tile0)
            for n in range(2 * T):
                if ld >= self.STAGES:
                    yield self.at_stage(self.codes_empty, ld - self.STAGES)
                self.codes_full[ld % self.stage_bars].arrive(tx=1)
                late = self.rng.random() < self.stragglers
                self.flying.append((self.now + self.rng.randint(1, 400 if late else 12), ld, half))
                ld += 1
                if half == 0 and loads.get(n, 0) > 0:
                    self.write_scales(tile0 + loads[n])
            tile0 += T

    def issuer(self, g):
        ld0 = 0
        for u, (T, pair) in enumerate(self.units):
            def release(ld):
                for _ in range(1 if pair else 2):
                    self.empty[ld % self.bars].arrive()
            yield lambda: u == 0 or self.through(u - 1)
            tiles = self.mine(T, pair, g)
            for t in tiles[:1]:
                yield self.at(self.full, ld0 + seq_k(t))
                self.use(ld0 + seq_k(t))
                self.s.update(((u, t, g, 0), (u, t, g, 1)))
                release(ld0 + seq_k(t))
            for t in tiles:
                nxt = t + tiles.step
                yield self.at(self.full, ld0 + seq_v(t, T))
                for half in range(2):
                    yield lambda: (u, t, g, half) in self.p
                    self.use(ld0 + seq_v(t, T))
                    if half:
                        release(ld0 + seq_v(t, T))
                    if nxt < T:
                        if half == 0:
                            yield self.at(self.full, ld0 + seq_k(nxt))
                        self.use(ld0 + seq_k(nxt))
                        self.s.add((u, nxt, g, half))
                        if half:
                            release(ld0 + seq_k(nxt))
                self.pv.add((u, t, g))
            ld0 += 2 * T

    def softmax(self, g):
        tile0 = 0
        for u, (T, pair) in enumerate(self.units):
            for t in self.mine(T, pair, g):
                tile = tile0 + t
                at = tile % len(self.scales)
                for half in range(2):
                    yield lambda: (u, t, g, half) in self.s
                    if half == 0:
                        yield lambda: self.scale_bars[at].passed((tile // len(self.scales)) & 1)
                    for _ in range(self.rng.randint(0, 3)):
                        if self.scales[at] != tile:
                            raise Broken("a tile's scales are read before they are there, or after the next ones were written over them")
                        yield lambda: True
                    if self.scales[at] != tile:
                        raise Broken("a tile's scales are read before they are there, or after the next ones were written over them")
                    self.p.add((u, t, g, half))
            tile0 += T


def test_loads_and_scales_are_used_when_they_are_there():
    rng = random.Random(6)
    for _ in range(200):
        Model(units(rng), rng, stragglers=rng.choice([0.0, 0.02, 0.2]))


def test_units_of_one_tile():
    rng = random.Random(7)
    for _ in range(100):
        Model([(1, rng.random() < 0.5) for _ in range(30)], rng, stragglers=rng.choice([0.0, 0.1]))


def test_three_tiles_of_scales_would_not_do():
    rng = random.Random(8)
    with pytest.raises(Broken):
        for _ in range(300):
            Model(units(rng), rng, stragglers=0.05, scale_tiles=3)
