"""GPU parity: attention over shared prefixes against the fp64 oracle, which looks at every request by itself.

Tolerances.  bf16 cache: the weights are rounded to bf16 once (2^-8 of themselves), their sum is not, and the output once more, so
per element  |error| <= 2^-8 |out| + 1.05 * 2^-8 * sum w |v|  (w: the exact weights; 5 % for 32-bit sums, the fast exp2 and products of roundings); the log-sum-exp sees 32-bit
arithmetic.  8-bit cache: the bound of tests/test_gpu_attention_quant.py (weights in two 8-bit parts)."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as A
from oracle import cache_oracle as O
from tests import quant_util as Q

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def war():
    from paper_2607_17299_b200 import binding
    return binding


class Case:
    """groups: (shared tokens, [own tokens of each member]); requests are shuffled, unused table entries are out of range."""

    def __init__(self, seed, kv, groups, N, Hq, Hkv, page, block=0, token_major=False, full=False, stopped=()):
        rng = np.random.default_rng(seed)
        self.kv, self.N, self.Hq, self.Hkv, self.page, self.block = kv, N, Hq, Hkv, page, block
        B = sum(len(own) for _, own in groups)
        order = rng.permutation(B).tolist()
        self.nn, self.parent = Q.trees(rng, B, N, full)
        self.nn[list(stopped)] = 0
        self.prefix, self.leader, self.shared = np.zeros(B, np.int32), np.arange(B, dtype=np.int32), np.full(B, 12345, np.int32)
        rows, at = [None] * B, 0
        for shared, own in groups:
            idx = [order.pop() for _ in own]
            common = np.arange(at, at + shared // page)
            at += len(common)
            for i, mine in zip(idx, own):
                self.prefix[i] = shared + mine
                need = -(-(int(self.prefix[i]) + N) // page) - len(common)
                rows[i] = np.concatenate([common, np.arange(at, at + need)])
                at += need
            if len(idx) > 1:
                self.leader[idx] = min(idx) if seed % 2 else idx[0]
                self.shared[idx] = shared
        total = at + 3
        place = rng.permutation(total)
        self.pt = np.full((B, max(len(r) for r in rows) + 1), 1 << 30, np.int32)
        for i, r in enumerate(rows):
            self.pt[i, :len(r)] = place[r]
        if kv == "bf16":
            self.k, self.v = (torch.from_numpy(rng.standard_normal((total, Hkv, page, 128)).astype(np.float32)).to(torch.bfloat16) for _ in "kv")
        else:
            (self.k, self.sk), (self.v, self.sv) = (Q.cache(rng, kv, total, Hkv, page, block) for _ in "kv")
        live = np.zeros((total, page), bool)                             # rows that nobody uses hold NaN
        for i in range(B):
            pos = np.arange(int(self.prefix[i] + self.nn[i]))
            live[self.pt[i, pos // page], pos % page] = True
        if kv == "bf16":
            for x in (self.k, self.v):
                x.permute(0, 2, 1, 3)[torch.from_numpy(~live)] = float("nan")
            put = lambda x: (x.to(DEV).permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) if token_major else x.to(DEV))
            self.cache = (put(self.k), put(self.v))
        else:
            for c in (self.k, self.v):
                c[np.broadcast_to(~live[:, None, :], c.shape[:3])] = 0x7F
            dead = ~live.reshape(total, page // block, block).any(-1)
            for s in (self.sk, self.sv):
                s[np.broadcast_to(dead[:, None, :], s.shape)] = np.nan
            t = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(DEV)
            self.cache = (Q.to_device(self.k, kv, token_major), Q.to_device(self.v, kv, token_major), t(self.sk), t(self.sv))
        self.q = torch.randn((B, N, Hq, 128), generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16)
        self.scale = 1.0 / np.sqrt(128)
        t = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(DEV)
        self.d_q = self.q.to(DEV)
        self.ints = [t(x) for x in (self.pt, self.prefix, self.nn, self.parent, self.leader, self.shared)]

    def args(self, war):
        quant = self.kv != "bf16"
        p = (war.attn_quant_params if quant else war.attn_params)(self.d_q, *self.cache, self.ints[0], self.scale)
        ws = (war.new_shared_quant_workspace if quant else war.new_shared_workspace)(p, DEV)
        ws.fill_(0xA5)
        out = torch.full(self.d_q.shape, 7.0, dtype=torch.bfloat16, device=DEV)
        lse = torch.full(self.d_q.shape[:3], 7.0, device=DEV)
        return (self.d_q, *self.cache, *self.ints, p, ws, out, lse)

    def call(self, war, a):
        (war.war_verify_attn_shared_quant if self.kv != "bf16" else war.war_verify_attn_shared)(*a)

    def run(self, war):
        a = self.args(war)
        self.call(war, a)
        torch.cuda.synchronize()
        return a[-2], a[-1]

    def values(self, i):
        L = int(self.prefix[i] + self.nn[i])
        pos = np.arange(L)
        pg, r = self.pt[i, pos // self.page], pos % self.page
        if self.kv == "bf16":
            return [x[pg, :, r].double().numpy() for x in (self.k, self.v)]
        return [O.decode(c[pg, :, r], self.kv) * s[pg, :, r // self.block][..., None] for c, s in ((self.k, self.sk), (self.v, self.sv))]

    def check(self, out, lse, requests=None, untouched=()):
        got, got_lse = out.float().cpu().numpy().astype(np.float64), lse.cpu().numpy()
        for i in range(len(self.prefix)) if requests is None else requests:
            n = 0 if i in untouched else int(self.nn[i])
            assert (got[i, n:] == 7.0).all() and (got_lse[i, n:] == 7.0).all(), i
            if n == 0:
                continue
            K, V = self.values(i)
            q = self.q[i].double().numpy()
            want, want_lse = A.verify_attention_request(q, K, V, int(self.prefix[i]), self.parent[i], n, self.scale)
            mass, _ = A.verify_attention_request(q, K, np.abs(V), int(self.prefix[i]), self.parent[i], n, self.scale)
            bound = 2.0 ** -8 * np.abs(want) + 1.05 * 2.0 ** -8 * mass
            if self.kv != "bf16":
                top = np.repeat(np.abs(V).max(axis=(0, 2)), self.Hq // self.Hkv)[None, :, None]
                bound += 1.05 * len(K) * 2.0 ** -17 / 14 * top
            err = np.abs(got[i, :n] - want)
            assert (err <= bound).all(), (i, float((err / bound).max()))
            np.testing.assert_allclose(got_lse[i, :n], want_lse, atol=1e-4, rtol=1e-5)


CASES = [
    # seed, kv, groups, N, Hq, Hkv, page, block, token_major
    (1, "bf16", [(256, [0, 1, 100, 7])], 1, 8, 2, 16),                                              # the first token behind a shared prefix
    (2, "bf16", [(16, [0, 0]), (1024, [5, 300, 129]), (0, [77])], 8, 8, 2, 16),
    (3, "bf16", [(400, [40] * 9)], 16, 16, 2, 16, 0, True),                                         # 1152 rows: nine row blocks, requests across their borders
    (4, "bf16", [(8, [1, 2]), (4000, [10, 20]), (128, [0, 128])], 64, 8, 1, 8),                      # 512 rows a request
    (5, "bf16", [(640, [3, 500, 64])], 5, 15, 3, 128),                                              # five query heads a group
    (6, "bf16", [(96, [1])] * 5, 3, 4, 4, 32, 0, True),                                             # nobody shares
    (7, "bf16", [(7984, [3, 4, 5, 6, 7, 8, 9, 10])], 7, 8, 1, 16),                                  # long: many chunks
    (8, "bf16", [(48, [0, 9])] * 40, 2, 4, 1, 16),                                                  # 80 requests: the chunk length is not searched
    (11, "e4m3", [(256, [0, 1, 100, 7])], 1, 8, 2, 16, 16),
    (12, "e4m3", [(16, [0, 0]), (1024, [5, 300, 129]), (0, [77])], 8, 8, 2, 16, 8),
    (13, "e5m2", [(400, [40] * 9)], 16, 16, 2, 16, 16, True),
    (14, "e4m3", [(8, [1, 2]), (4000, [10, 20]), (128, [0, 128])], 64, 8, 1, 8, 8, True),
    (15, "e5m2", [(640, [3, 500, 64])], 5, 15, 3, 128, 32),
    (16, "e4m3", [(7984, [3, 4, 5, 6, 7, 8, 9, 10])], 7, 8, 1, 16, 16),
    (17, "e5m2", [(48, [0, 9])] * 40, 2, 4, 1, 16, 8),
]


@pytest.mark.parametrize("case", CASES, ids=[str(c[0]) for c in CASES])
def test_matches_oracle(war, case):
    c = Case(*case)
    c.check(*c.run(war))
    assert war.war_device_status() == 0


@pytest.mark.parametrize("seed", range(10))
def test_random_shapes(war, seed):
    rng = np.random.default_rng(300 + seed)
    kv = ["bf16", "e4m3", "e5m2"][seed % 3]
    page = int(rng.choice([8, 16, 32, 64, 128]))
    block = int(rng.choice([b for b in (8, 16, 32, 64, 128) if b <= page]))
    Hkv, G = int(rng.integers(1, 4)), int(rng.choice([1, 2, 3, 7, 8]))
    N = int(rng.integers(1, min(64, 512 // G) + 1))
    groups = [(int(rng.integers(0, 1200 // page)) * page, rng.integers(0, 400, int(rng.integers(1, 6))).tolist()) for _ in range(int(rng.integers(1, 5)))]
    B = sum(len(o) for _, o in groups)
    c = Case(seed, kv, groups, N, Hkv * G, Hkv, page, block, bool(rng.integers(2)), stopped=[i for i in range(B) if rng.random() < 0.2])
    c.check(*c.run(war))
    assert war.war_device_status() == 0
