"""Rollouts as they would be run: a few prompts, several requests each, on one pool.  Every step gives requests that have ended their
pages back, starts new ones as copies of running ones, makes room, stores a tree's keys and values, finds the groups, computes the
attention over their shared prefixes, picks the target's tokens, accepts and commits; now and then the pool is compacted.

Checked at every step: the books against plain lists; what every request's cache holds, through its own table, bit for bit across
forks, copies and compaction; attention against the fp64 oracle on that (bounds of test_gpu_attention_shared.py); acceptance."""
import numpy as np
import pytest
import torch

from oracle import accept_oracle as ACC
from oracle import attention_oracle as A
from oracle import cache_oracle as C
from oracle import pages_oracle as O
from tests import pages_util as U
from tests import quant_util as Q

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def war():
    from paper_2607_17299_b200 import binding
    return binding


def t(x, dt=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(x))).to(dt).to(DEV)


class Cache:
    def __init__(self, war, kv, pages, Hkv, page, block):
        self.war, self.kv, self.page, self.block = war, kv, page, block
        if kv == "bf16":
            self.pools = [torch.full((pages, Hkv, page, 128), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in "kv"]
            self.scales = [None, None]
        else:
            self.pools = [torch.full((pages, Hkv, page, 128), 0x7F, dtype=torch.uint8, device=DEV).view(Q.KV_DTYPE[kv]) for _ in "kv"]
            self.scales = [torch.full((pages, Hkv, page // block), float("nan"), device=DEV) for _ in "kv"]

    def all(self):
        return (*self.pools, *self.scales) if self.kv != "bf16" else tuple(self.pools)

    def rows(self, table, n):
        """K and V of the first n positions, float64 [n, Hkv, 128]."""
        pos = np.arange(n)
        pg, r = np.asarray(table, np.int64)[pos // self.page], pos % self.page
        if self.kv == "bf16":
            return [x.cpu()[pg, :, r].double().numpy() for x in self.pools]
        return [C.decode(Q.codes_of(x)[pg, :, r], self.kv) * s.cpu().numpy()[pg, :, r // self.block][..., None] for x, s in zip(self.pools, self.scales)]


@pytest.mark.parametrize("kv,page,block,seed", [("bf16", 16, 0, 1), ("bf16", 64, 0, 2), ("e4m3", 16, 16, 3), ("e5m2", 32, 8, 4), ("e4m3", 64, 16, 5)])
def test_rollouts(war, kv, page, block, seed):
    rng = np.random.default_rng(seed)
    B, N, Hq, Hkv, V, P, pages, width = 9, 12, 12 if page == 64 else 8, 2, 6, 8, 150, 40
    cache = Cache(war, kv, pages, Hkv, page, block)
    b = O.Books(pages, width, [[] for _ in range(B)], [0] * B, [[0] * P for _ in range(B)], [-1] * B)
    d = U.Device(war, b)
    d.copies = torch.zeros((pages, 3), dtype=torch.int32, device=DEV)
    compact_ws = war.new_compact_workspace(d.pages)
    inv = t((10000.0 ** (-np.arange(64) / 64)), torch.float32)
    leader, shared = (torch.zeros(B, dtype=torch.int32, device=DEV) for _ in range(2))
    scale = 1.0 / np.sqrt(128)
    held_rows = {}                                                   # request: its context's rows as last seen

    def store(nn, parent, n_slots):
        qkv = torch.randn((B, n_slots, Hq + 2 * Hkv, 128), generator=gen).to(torch.bfloat16).to(DEV)
        q, k, v = qkv.split([Hq, Hkv, Hkv], dim=2)
        q_out = torch.zeros((B, n_slots, Hq, 128), dtype=torch.bfloat16, device=DEV)
        war.war_rope_store(q, k, v, inv, d.pages.page_table, d.prefix, t(nn), t(parent), *cache.pools, *cache.scales, q_out)
        return q_out

    def unchanged():
        for i in range(B):
            if b.tail_len[i] >= 0:
                for x, y in zip(cache.rows(b.rows[i], b.prefix[i]), held_rows[i]):
                    assert np.array_equal(x, y), i

    def remember():
        for i in range(B):
            if b.tail_len[i] >= 0:
                held_rows[i] = cache.rows(b.rows[i], b.prefix[i])

    gen = torch.Generator().manual_seed(seed)
    # two prompts, a chain of tokens each, written as trees without branches
    for i, n in ((0, 61), (5, 200)):
        for first in range(0, n, 50):
            m = min(50, n - first)
            b.prefix[i], b.tail_len[i] = first, 0
            d.prefix[i], d.tail_len[i] = first, 0
            want = O.grow(b, m, page)
            war.war_pages_grow(d.pages, m, page, d.prefix, d.tail_len, d.granted)
            assert d.granted.tolist() == want
            chain = np.tile(np.arange(-1, 49), (B, 1))
            nn = np.zeros(B, np.int64)
            nn[i] = m
            store(nn, chain, 50)
        b.prefix[i] = n
        d.prefix[i] = n
    d.check(b)
    remember()
    accepted, biggest = 0, 0
    for step in range(12):
        # ---- requests that have ended, and new ones as copies of running ones ----
        live = [i for i in range(B) if b.tail_len[i] >= 0]
        if step >= 3 and len(live) > 3:
            done = [int(i in live[1:] and rng.random() < 0.25) for i in range(B)]
            O.release(b, done)
            war.war_pages_free(d.pages, t(done), d.tail_len)
            d.check(b)
            live = [i for i in live if not done[i]]
        src = [-1] * B
        for i in range(B):
            if b.tail_len[i] < 0 and rng.random() < 0.7:
                src[i] = int(rng.choice(live))
        if step == 6:
            src[live[0]], src[live[-1]] = live[-1], live[0]          # two change places
        before = dict(held_rows)
        ok, copies = O.fork(b, src, page)
        war.war_pages_fork(d.pages, t(src), page, d.prefix, d.tail, d.tail_len, d.copies, d.n, d.word)
        war.war_pages_copy(d.copies, d.n, *cache.pools, *cache.scales)
        assert ok and int(d.word) == 1 and d.listed() == copies
        d.check(b)
        for i, s in enumerate(src):
            if s >= 0:
                held_rows[i] = before[s]
        unchanged()
        if step % 4 == 2:
            most = d.copies.shape[0]
            copies, top = O.compact(b, most, page)
            war.war_pages_compact(d.pages, page, compact_ws, d.copies, d.n, d.word)
            war.war_pages_copy(d.copies, d.n, *cache.pools, *cache.scales)
            assert d.listed() == copies and int(d.word) == top
            for x in cache.pools:                                    # nothing is read above the top
                x[top:] = float("nan") if kv == "bf16" else x[top:]
            d.check(b)
            unchanged()
        # ---- room for the trees, their keys and values, the attention ----
        want = O.grow(b, N, page)
        war.war_pages_grow(d.pages, N, page, d.prefix, d.tail_len, d.granted)
        assert d.granted.tolist() == want
        d.check(b)
        nn, parent = Q.trees(rng, B, N)
        nn[[i for i in range(B) if b.tail_len[i] < 0]] = 0
        ids = rng.integers(0, V, (B, N))
        q = store(nn, parent, N)
        war.war_prefix_groups(d.pages.page_table, d.prefix, d.tail_len, page, page, leader, shared)
        want = O.groups(b.rows, b.prefix, [x >= 0 for x in b.tail_len], page, page)
        assert leader.tolist() == want[0] and shared.tolist() == want[1]
        biggest = max(biggest, max(want[0].count(l) for l in want[0]))
        quant = kv != "bf16"
        p = (war.attn_quant_params if quant else war.attn_params)(q, *cache.all(), d.pages.page_table, scale)
        ws = (war.new_shared_quant_workspace if quant else war.new_shared_workspace)(p, DEV)
        out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:3], 7.0, device=DEV)
        (war.war_verify_attn_shared_quant if quant else war.war_verify_attn_shared)(
            q, *cache.all(), d.pages.page_table, d.prefix, t(nn), t(parent), leader, shared, p, ws, out, lse)
        torch.cuda.synchronize()
        assert war.war_device_status() == 0
        for i in range(B):
            n = int(nn[i])
            assert (out[i, n:] == 7.0).all() and (lse[i, n:] == 7.0).all()
            if n == 0:
                continue
            K, Vv = cache.rows(b.rows[i], b.prefix[i] + n)
            x = q[i].double().cpu().numpy()
            ref, ref_lse = A.verify_attention_request(x, K, Vv, b.prefix[i], parent[i], n, scale)
            mass, _ = A.verify_attention_request(x, K, np.abs(Vv), b.prefix[i], parent[i], n, scale)
            bound = 2.0 ** -8 * np.abs(ref) + 1.05 * 2.0 ** -8 * mass
            if quant:
                bound += 1.05 * len(K) * 2.0 ** -17 / 14 * np.repeat(np.abs(Vv).max(axis=(0, 2)), Hq // Hkv)[None, :, None]
            assert (np.abs(out[i, :n].double().cpu().numpy() - ref) <= bound).all(), (step, i)
            np.testing.assert_allclose(lse[i, :n].cpu().numpy(), ref_lse, atol=1e-4, rtol=1e-5)
        # ---- the target's tokens, acceptance, commit ----
        logits = torch.randn((B, N, V), generator=gen).to(DEV)
        target, alen, bonus = (torch.zeros(s, dtype=torch.int32, device=DEV) for s in ((B, N), (B,), (B,)))
        path = torch.zeros((B, N), dtype=torch.int32, device=DEV)
        war.war_target(logits, t(nn), t(ids), t(parent), target)
        war.war_accept(t(ids), t(parent), t(nn), target, 0, alen, path, bonus)
        picks = logits.argmax(-1).cpu().numpy()
        for i in range(B):
            assert (target.cpu().numpy()[i, :nn[i]] == picks[i, :nn[i]]).all()
        want = ACC.accept_batch(ids.astype(np.int32), parent, nn, target.cpu().numpy(), 0)
        for x, y in zip((alen, path, bonus), want):
            assert (x.cpu().numpy()[nn > 0] == y[nn > 0]).all()
        if not quant:                                                # the accepted rows, in order, behind the context and the root
            for i in np.nonzero(nn)[0]:
                K, Vv = cache.rows(b.rows[i], b.prefix[i] + int(nn[i]))
                keep = [*range(b.prefix[i] + 1), *(b.prefix[i] + path[i, :int(alen[i])].cpu().numpy())]
                held_rows[i] = [K[keep], Vv[keep]]
        (war.war_commit_quant if quant else war.war_commit)(t(ids), alen, path, bonus, *cache.all(), d.pages.page_table, d.prefix, d.tail, d.tail_len)
        torch.cuda.synchronize()
        for i in range(B):
            if nn[i]:
                accepted += int(alen[i])
                b.prefix[i] += int(alen[i]) + 1
        assert d.prefix.tolist() == b.prefix
        b.tail, b.tail_len = d.tail.tolist(), d.tail_len.tolist()
        d.check(b)
        if quant:
            remember()
        else:
            unchanged()
        assert war.war_device_status() == 0
    assert accepted > 10 and biggest >= 4
