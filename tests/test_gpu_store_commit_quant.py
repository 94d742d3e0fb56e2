"""GPU parity: war_rope_store and war_commit_quant against the plain checker, and a run of whole steps on the 8-bit cache.

Tolerances.  V rows and moved rows are compared code for code.  A rotated value y carries the 32-bit errors of the sine and
cosine (half an ulp each) and of two products and a sum: |error| <= 2^-21 (|a| + |b|).  It
may therefore round to a neighbouring code or bf16 value, so keys are compared by value: half a step of the type at that
magnitude plus the error above (bf16: 2^-8 relative; codes: half the gap around them)."""
import numpy as np
import pytest
import torch

from oracle import accept_oracle as ACC
from oracle import attention_oracle as A
from oracle import cache_oracle as O
from tests import quant_util as Q

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def war():
    from paper_2607_17299_b200 import binding
    return binding


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV)


class Store:
    def __init__(self, seed, kv, prefix, N, Hq, Hkv, page, block, rot, interleaved=False, token_major=False, pow2=True, zero=False,
                 magnitude=1.0, full=False):
        rng = np.random.default_rng(seed)
        B = len(prefix)
        self.kv, self.block, self.interleaved, self.rot = kv, block, interleaved, rot
        self.prefix = np.asarray(prefix, np.int32)
        self.nn, self.parent = Q.trees(rng, B, N, full)
        # leading pages are shared by everybody: only the last ones are written
        first = np.maximum(self.prefix // page - 1, 0)
        width = max(int(p) + N for p in prefix) // page + 2
        per = (N - 1) // page + 3
        self.pt = np.tile(np.arange(width) % 4, (B, 1)).astype(np.int32)
        perm = rng.permutation(B * per) + 4
        for i in range(B):
            c = min(per, width - first[i])
            self.pt[i, first[i]:first[i] + c] = perm[i * per:i * per + c]
        total = 4 + B * per
        if kv == "bf16":
            g = torch.Generator().manual_seed(seed)
            self.ck, self.cv = (torch.randn((total, Hkv, page, 128), generator=g).to(torch.bfloat16) for _ in range(2))
            self.sk = self.sv = None
            lay = lambda t: (t.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) if token_major else t.contiguous()).to(DEV)
            if token_major:
                lay = lambda t: t.to(DEV).permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
            self.k_pool, self.v_pool = lay(self.ck), lay(self.cv)
        else:
            self.ck, self.sk = Q.cache(rng, kv, total, Hkv, page, block, pow2=pow2)
            self.cv, self.sv = Q.cache(rng, kv, total, Hkv, page, block, pow2=pow2)
            self.k_pool, self.v_pool = Q.to_device(self.ck, kv, token_major), Q.to_device(self.cv, kv, token_major)
        self.dsk, self.dsv = (None, None) if self.sk is None else (dev(self.sk), dev(self.sv))
        g = torch.Generator().manual_seed(seed + 1)
        qkv = torch.randn((B, N, (Hq + 2 * Hkv) * 128), generator=g) * torch.exp(torch.randn((B, N, 1), generator=g)) * magnitude
        if zero:
            qkv = qkv * 0
        self.qkv = qkv.to(torch.bfloat16)
        d = self.qkv.to(DEV)
        self.dq, self.dk, self.dv = (x.unflatten(2, (-1, 128)) for x in d.split([Hq * 128, Hkv * 128, Hkv * 128], dim=2))
        self.inv_freq = (10000.0 ** (-np.arange(rot // 2) / max(1, rot // 2))).astype(np.float32)

    def run(self, war, factor=1.0):
        self.q_out = torch.full(self.dq.shape, 7.0, dtype=torch.bfloat16, device=DEV)
        war.war_rope_store(self.dq, self.dk, self.dv, dev(self.inv_freq), dev(self.pt), dev(self.prefix), dev(self.nn), dev(self.parent),
                           self.k_pool, self.v_pool, self.dsk, self.dsv, self.q_out, interleaved=self.interleaved, factor=factor)
        torch.cuda.synchronize()

    def check(self, factor=1.0, skip=()):
        x = [t.double().cpu().numpy() for t in (self.dq, self.dk, self.dv)]
        q_out = self.q_out.double().cpu().numpy()
        page = self.ck.shape[2]
        if self.kv == "bf16":
            got_k, got_v = self.k_pool.cpu(), self.v_pool.cpu()
            want_k, want_v = self.ck.clone(), self.cv.clone()
        else:
            got_k, got_v = Q.codes_of(self.k_pool), Q.codes_of(self.v_pool)
            got_sk, got_sv = self.dsk.cpu().numpy(), self.dsv.cpu().numpy()
            want_k, want_sk, want_v, want_sv = self.ck.copy(), self.sk.copy(), self.cv.copy(), self.sv.copy()
            steps = np.diff(O.values(self.kv)[: (0x7F if self.kv == "e4m3" else 0x7C)])
        near = []                                              # key rows compared by value
        for b in range(len(self.prefix)):
            if b in skip:
                assert (q_out[b] == 7).all()
                continue
            n, p = int(self.nn[b]), int(self.prefix[b])
            assert (q_out[b, n:] == 7).all()
            keys = np.zeros((n,) + x[1].shape[2:])
            for j in range(n):
                at = p + O.depth_of(self.parent[b], j)
                want = O.rotate(x[0][b, j], at, self.inv_freq, self.interleaved, factor)
                size = np.abs(x[0][b, j]) + np.abs(x[0][b, j]).max(-1, keepdims=True)
                assert (np.abs(q_out[b, j] - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -21 * factor * size).all(), (b, j)
                keys[j] = O.rotate(x[1][b, j], at, self.inv_freq, self.interleaved, factor)
            err = 2.0 ** -21 * factor * 2 * np.abs(x[1][b, :n]).max(-1, keepdims=True)
            if self.kv == "bf16":
                for j in range(n):
                    pg, r = self.pt[b, (p + j) // page], (p + j) % page
                    d = np.abs(got_k[pg, :, r].double().numpy() - keys[j])
                    assert (d <= 2.0 ** -8 * np.abs(keys[j]) + err[j]).all(), (b, j)
                    want_k[pg, :, r] = got_k[pg, :, r]
                    want_v[pg, :, r] = self.dv[b, j].cpu()
                continue
            O.store_rows(want_v, want_sv, self.kv, self.block, self.pt[b], p, x[2][b, :n])
            for pg, h, r, j in O.store_rows(want_k, want_sk, self.kv, self.block, self.pt[b], p, keys):
                near.append((pg, h, r))
                s = float(got_sk[pg, h, r // self.block])
                assert s == want_sk[pg, h, r // self.block]
                code = got_k[pg, h, r]
                gap = steps[np.minimum(code & 0x7F, len(steps) - 1)]
                assert (np.abs(O.decode(code, self.kv) * s - keys[j, h]) <= 0.5 * gap * s + err[j, h]).all(), (b, j, h)
        if self.kv == "bf16":
            assert torch.equal(got_k, want_k) and torch.equal(got_v, want_v)
            return
        np.testing.assert_array_equal(got_v, want_v)
        np.testing.assert_array_equal(got_sv, want_sv)
        np.testing.assert_array_equal(got_sk, want_sk)
        for place in near:
            want_k[place] = got_k[place]
        np.testing.assert_array_equal(got_k, want_k)             # older rows re-encoded, all others untouched


CASES = [
    # seed, kv, prefixes, N, Hq, Hkv, page, block, rot, interleaved, token_major
    (1, "e4m3", [0, 5, 15, 16, 17, 4000], 1, 8, 2, 16, 16, 128, False, False),
    (2, "e4m3", [0, 3, 77, 1000], 8, 8, 2, 16, 8, 128, True, False),
    (3, "e5m2", [9, 100, 31], 64, 4, 1, 32, 32, 64, False, True),
    (4, "e5m2", [250, 0], 33, 5, 5, 128, 64, 98, False, False),      # 49 pairs: no lane boundary between partners
    (5, "e4m3", [130, 8], 20, 2, 1, 8, 8, 32, True, True),
    (6, "bf16", [0, 15, 300], 16, 8, 2, 16, 16, 128, False, False),
    (7, "bf16", [7, 90], 64, 3, 3, 24, 24, 2, False, True),          # a page size of 24, one pair
    (8, "bf16", [1], 1, 1, 1, 1, 1, 0, False, False),                # nothing rotated, pages of one token
    (9, "e4m3", [100], 12, 0, 2, 16, 16, 16, False, False),          # no queries
]


@pytest.mark.parametrize("case", CASES, ids=[str(c[0]) for c in CASES])
def test_store_matches_checker(war, case):
    s = Store(*case)
    if case[4] == 0:
        war.war_rope_store(None, s.dk, s.dv, dev(s.inv_freq), dev(s.pt), dev(s.prefix), dev(s.nn), dev(s.parent), s.k_pool, s.v_pool,
                           s.dsk, s.dsv, None, interleaved=s.interleaved)
        s.q_out = torch.full(s.dq.shape, 7.0, dtype=torch.bfloat16, device=DEV)
    else:
        s.run(war)
    s.check()
    assert war.war_device_status() == 0


@pytest.mark.parametrize("kv,rot,interleaved", [("e4m3", 126, False), ("bf16", 126, True), ("e5m2", 100, True), ("e4m3", 48, False),
                                                ("e4m3", 112, True), ("bf16", 16, False), ("e5m2", 16, True), ("bf16", 34, False)])
def test_store_rotations(war, kv, rot, interleaved):
    """Every layout of a lane's pairs, the largest table (64 slots) where the rotation ends inside a lane; blocks of more rows
    than stay in registers."""
    s = Store(27, kv, [33, 900], 64, 9, 2, 32, 32, rot, interleaved, full=True)
    s.run(war)
    s.check()
    assert war.war_device_status() == 0


def test_store_many_requests_and_none(war):
    """More requests than thread blocks fit the GPU, some without a slot."""
    s = Store(29, "e5m2", [k % 50 for k in range(400)], 2, 3, 1, 16, 16, 32)
    s.nn[::7] = 0
    s.run(war)
    s.check(skip=range(0, 400, 7))
    assert war.war_device_status() == 0


@pytest.mark.parametrize("kw", [dict(pow2=False), dict(zero=True), dict(magnitude=1e-30), dict(magnitude=1e30), dict(magnitude=300.0)])
def test_store_scales(war, kw):
    """Old scales that are no powers of two, rows of zeros, rows far smaller and far larger than what the block holds."""
    for kv in ("e4m3", "e5m2"):
        s = Store(21, kv, [5, 33, 64], 6, 2, 2, 16, 16, 0, **kw)
        s.run(war)
        s.check()


def test_store_far_positions_and_factor(war):
    s = Store(22, "e4m3", [900_001, 131_071, 65_535], 8, 4, 1, 16, 16, 128)
    s.run(war, factor=1.25)
    s.check(factor=1.25)


def test_store_twice_is_the_same_and_in_place(war):
    s = Store(23, "e4m3", [12, 40], 16, 4, 2, 16, 16, 128, full=True)
    s.run(war)
    k, sc = Q.codes_of(s.k_pool), s.dsk.clone()
    q = s.dq.contiguous()
    want = s.q_out.clone()
    war.war_rope_store(q, s.dk, s.dv, dev(s.inv_freq), dev(s.pt), dev(s.prefix), dev(s.nn), dev(s.parent), s.k_pool, s.v_pool,
                       s.dsk, s.dsv, q)
    torch.cuda.synchronize()
    assert torch.equal(q, want) and (Q.codes_of(s.k_pool) == k).all() and torch.equal(s.dsk, sc)


def test_store_nan_and_infinity(war):
    s = Store(24, "e4m3", [16], 4, 1, 1, 16, 16, 0, full=True)
    s.dv[0, 1, 0, 3], s.dv[0, 2, 0, 4] = float("nan"), float("-inf")
    s.run(war)
    pg, scale = s.pt[0, 1], float(s.dsv[int(s.pt[0, 1]), 0, 0])
    rows = O.decode(Q.codes_of(s.v_pool)[pg, 0, :4], "e4m3")
    assert np.isnan(rows[1, 3]) and rows[2, 4] == -448 and np.isfinite(scale) and np.isfinite(np.delete(rows.ravel(), 128 + 3)).all()


def test_store_leaves_bad_requests(war):
    s = Store(25, "e4m3", [20, 30, 40, 50], 8, 4, 2, 16, 16, 128, full=True)
    s.parent[1, 2] = 5
    s.prefix[2] = 1 << 20
    s.run(war)
    s.check(skip=(1, 2))
    assert war.war_device_status() in (7, 8)
    s = Store(26, "e4m3", [20, 30], 4, 4, 2, 16, 16, 128, full=True)
    before = Q.codes_of(s.k_pool)
    s.pt[0, 1] = -5
    s.run(war)
    assert war.war_device_status() == 8
    s.pt[0, 1] = 0
    after = Q.codes_of(s.k_pool)
    assert (after[s.pt[1, 1]] != before[s.pt[1, 1]]).any()
    others = [p for p in range(len(after)) if p not in set(s.pt[1].tolist())]
    assert (after[others] == before[others]).all()


def _paths(rng, nn, parent, N):
    alen, path = np.zeros(len(nn), np.int32), np.full((len(nn), N), -1, np.int32)
    for b in range(len(nn)):
        j = int(rng.integers(0, nn[b]))
        up = []
        while j > 0:
            up.append(j)
            j = int(parent[b, j])
        alen[b] = len(up)
        path[b, :len(up)] = up[::-1]
    return alen, path


@pytest.mark.parametrize("kv,N,Hkv,page,block,token_major,pow2", [
    ("e4m3", 8, 2, 16, 16, False, True), ("e4m3", 16, 3, 16, 8, True, False), ("e5m2", 64, 1, 32, 32, False, False),
    ("e5m2", 24, 8, 8, 8, True, True), ("e4m3", 64, 2, 128, 128, False, False), ("e4m3", 1, 2, 16, 16, False, True),
    ("e5m2", 40, 9, 64, 16, True, False)])
def test_commit_matches_checker(war, kv, N, Hkv, page, block, token_major, pow2):
    rng = np.random.default_rng(N + page + Hkv)
    B, P = 23, 32
    prefix = rng.integers(0, 300, B).astype(np.int32)
    prefix[:5] = [0, block - 1, block, page - 1, 2 * page]
    nn, parent = Q.trees(rng, B, N)
    alen, path = _paths(rng, nn, parent, N)
    pt, total = Q.pages(rng, prefix + N, page)
    ck, sk = Q.cache(rng, kv, total, Hkv, page, block, spread=1.0, pow2=pow2)
    cv, sv = Q.cache(rng, kv, total, Hkv, page, block, spread=1.0, pow2=pow2)
    ids = rng.integers(0, 1000, (B, N)).astype(np.int32)
    bonus = np.where(rng.random(B) < 0.3, -1, rng.integers(0, 1000, B)).astype(np.int32)
    tail_len = rng.integers(0, P + 1, B).astype(np.int32)
    tail = rng.integers(0, 1000, (B, P)).astype(np.int32)
    tail_len[7] = -1                                            # not running
    alen[8] = 2                                                 # malformed: slots that do not increase, or more than the tree has
    path[8, :2] = [3, 1][:N]
    k_pool, v_pool = Q.to_device(ck, kv, token_major), Q.to_device(cv, kv, token_major)
    dsk, dsv, dpl, dt, dtl = dev(sk), dev(sv), dev(prefix), dev(tail), dev(tail_len)
    war.war_commit_quant(dev(ids), dev(alen), dev(path), dev(bonus), k_pool, v_pool, dsk, dsv, dev(pt), dpl, dt, dtl)
    torch.cuda.synchronize()
    assert war.war_device_status() == 7
    got_pl, got_t, got_tl = dpl.cpu().numpy(), dt.cpu().numpy(), dtl.cpu().numpy()
    for b in range(B):
        k = int(alen[b])
        if b in (7, 8):
            assert got_pl[b] == prefix[b] and (got_t[b] == tail[b]).all() and got_tl[b] == tail_len[b]
            continue
        O.commit_rows(ck, sk, kv, block, pt[b], int(prefix[b]), path[b, :k])
        O.commit_rows(cv, sv, kv, block, pt[b], int(prefix[b]), path[b, :k])
        text = tail[b, P - tail_len[b]:].tolist() + [int(ids[b, j]) for j in path[b, :k]] + ([int(bonus[b])] if bonus[b] >= 0 else [])
        new = min(P, len(text))
        assert got_pl[b] == prefix[b] + k + (bonus[b] >= 0) and got_tl[b] == new
        assert (got_t[b] == [0] * (P - new) + text[len(text) - new:]).all()
    np.testing.assert_array_equal(Q.codes_of(k_pool), ck)
    np.testing.assert_array_equal(Q.codes_of(v_pool), cv)
    np.testing.assert_array_equal(dsk.cpu().numpy(), sk)
    np.testing.assert_array_equal(dsv.cpu().numpy(), sv)


def test_commit_with_a_bad_page(war):
    rng = np.random.default_rng(3)
    pt, total = Q.pages(rng, np.array([40, 40]), 16)
    ck, sk = Q.cache(rng, "e4m3", total, 1, 16, 16, pow2=True)
    k_pool, v_pool = Q.to_device(ck, "e4m3", False), Q.to_device(ck, "e4m3", False)
    keep = pt[0, 1]
    pt[0, 1] = total
    path = np.array([[2, 5, -1, -1, -1, -1, -1, -1]] * 2, np.int32)
    prefix = np.array([14, 14], np.int32)
    war.war_commit_quant(dev(np.zeros((2, 8), np.int32)), dev(np.array([2, 2], np.int32)), dev(path), dev(np.array([1, 1], np.int32)), k_pool,
                         v_pool, dev(sk), dev(sk), dev(pt), dev(prefix), dev(np.zeros((2, 4), np.int32)), dev(np.zeros(2, np.int32)))
    torch.cuda.synchronize()
    assert war.war_device_status() == 8
    got, s = Q.codes_of(k_pool), sk.copy()
    assert (got[keep] == ck[keep]).all() and (got[pt[0, 0]] == ck[pt[0, 0]]).all()
    O.commit_rows(ck, s, "e4m3", 16, pt[1], 14, [2, 5])
    assert (got[pt[1, 0]] == ck[pt[1, 0]]).all() and (got[pt[1, 1]] == ck[pt[1, 1]]).all()


@pytest.mark.parametrize("kv", ["e4m3", "e5m2"])
def test_whole_steps_in_a_row(war, kv):
    """store -> attention -> target -> accept -> commit, five times on the same buffers: the attention of every step against
    the checker on the values the cache stands for, choices and acceptance against their checkers, and the cache's live rows
    against the rows that were stored (each within the rounding of the coarsest scale its block has seen)."""
    rng = np.random.default_rng(7)
    B, N, Hq, Hkv, page, block, V, P = 5, 12, 8, 2, 16, 16, 500, 32
    prefix = np.array([0, 7, 16, 130, 255], np.int32)
    pt, total = Q.pages(rng, prefix + 6 * N, page)
    ck, sk = Q.cache(rng, kv, total, Hkv, page, block, pow2=True)
    cv, sv = Q.cache(rng, kv, total, Hkv, page, block, pow2=True)
    k_pool, v_pool, dsk, dsv = Q.to_device(ck, kv, False), Q.to_device(cv, kv, False), dev(sk), dev(sv)
    text = [rng.integers(0, V, int(p) + 1).tolist() for p in prefix]
    tail = np.zeros((B, P), np.int32)
    tail_len = np.array([min(P, len(t)) for t in text], np.int32)
    for b in range(B):
        tail[b, P - tail_len[b]:] = text[b][-tail_len[b]:]
    dpl, dt, dtl, dpt = dev(prefix), dev(tail), dev(tail_len), dev(pt)
    inv_freq, factor = war.war_rope_frequencies(128, 10000.0, "ramp", 4.0, 64.0)
    d_freq = inv_freq.to(DEV)
    out = torch.zeros((B, N, Hq, 128), dtype=torch.bfloat16, device=DEV)
    lse = torch.zeros((B, N, Hq), device=DEV)
    q_rot = torch.zeros_like(out)
    target = torch.zeros((B, N), dtype=torch.int32, device=DEV)
    alen, bonus = torch.zeros(B, dtype=torch.int32, device=DEV), torch.zeros(B, dtype=torch.int32, device=DEV)
    path = torch.zeros((B, N), dtype=torch.int32, device=DEV)
    params = war.attn_quant_params(out, k_pool, v_pool, dsk, dsv, dpt, 128 ** -0.5)
    ws = war.new_quant_workspace(params, DEV)
    scale_rows = {}
    for step in range(5):
        g = torch.Generator().manual_seed(step)
        nn, parent = Q.trees(rng, B, N)
        ids = rng.integers(0, V, (B, N)).astype(np.int32)
        q, k, v = (torch.randn((B, N, h, 128), generator=g).to(torch.bfloat16).to(DEV) for h in (Hq, Hkv, Hkv))
        d_nn, d_par, d_ids = dev(nn), dev(parent), dev(ids)
        war.war_rope_store(q, k, v, d_freq, dpt, dpl, d_nn, d_par, k_pool, v_pool, dsk, dsv, q_rot, factor=factor)
        war.war_verify_attn_quant(q_rot, k_pool, v_pool, dsk, dsv, dpt, dpl, d_nn, d_par, params, ws, out, lse)
        torch.cuda.synchronize()
        pl = dpl.cpu().numpy()
        hk, hv, hsk, hsv = Q.codes_of(k_pool), Q.codes_of(v_pool), dsk.cpu().numpy(), dsv.cpu().numpy()
        for b in range(B):
            n, L = int(nn[b]), int(pl[b] + nn[b])
            pos = np.arange(L)
            pg, r = pt[b, pos // page], pos % page
            K = O.decode(hk[pg, :, r], kv) * hsk[pg, :, r // block][..., None]
            Vv = O.decode(hv[pg, :, r], kv) * hsv[pg, :, r // block][..., None]
            want, want_lse = A.verify_attention_request(q_rot[b].double().cpu().numpy(), K, Vv, int(pl[b]), parent[b], n, 128 ** -0.5)
            got = out[b, :n].double().cpu().numpy()
            assert np.linalg.norm(got - want) < 2.0 ** -7 * np.linalg.norm(want)
            np.testing.assert_allclose(lse[b, :n].cpu().numpy(), want_lse, atol=1e-4, rtol=1e-5)
            for h in range(Hkv):                                # rows stored by this step and still there from earlier ones
                for j in range(n):
                    scale_rows[b, h, int(pl[b]) + j] = v[b, j, h].double().cpu().numpy()
                for x in range(int(prefix[b]), L):
                    s = hsv[pt[b, x // page], h, x % page // block]
                    worst = 2.0 ** (-4 if kv == "e4m3" else -3) * np.abs(scale_rows[b, h, x]) + s * 2.0 ** (-10 if kv == "e4m3" else -17)
                    assert (np.abs(Vv[x, h] - scale_rows[b, h, x]) <= 1.01 * worst).all(), (step, b, x)
        # the target agrees with some draft tokens: raise their logits
        logits = torch.randn((B, N, V), generator=g)
        for b in range(B):
            for j in range(1, int(nn[b])):
                if rng.random() < 0.6:
                    logits[b, parent[b, j], ids[b, j]] += 20
        off = np.zeros(B + 1, np.int64)
        off[1:] = np.cumsum([len(t) for t in text])
        war.war_target(logits.to(DEV), d_nn, d_ids, d_par, target, d_ctx=dev(np.concatenate(text).astype(np.int32)), d_ctx_off=dev(off),
                       d_repetition=torch.full((B,), 1.05, device=DEV))
        war.war_accept(d_ids, d_par, d_nn, target, 0, alen, path, bonus)
        torch.cuda.synchronize()
        h_t = target.cpu().numpy()
        w_alen, w_path, w_bonus = ACC.accept_batch(ids, parent, nn, h_t, 0)
        assert (alen.cpu().numpy() == w_alen).all() and (path.cpu().numpy() == w_path).all() and (bonus.cpu().numpy() == w_bonus).all()
        war.war_commit_quant(d_ids, alen, path, bonus, k_pool, v_pool, dsk, dsv, dpt, dpl, dt, dtl)
        torch.cuda.synchronize()
        for b in range(B):
            p = int(pl[b])
            moved = [[scale_rows[b, h, p + int(w_path[b, d])] for d in range(w_alen[b])] for h in range(Hkv)]
            for h in range(Hkv):
                for d in range(int(w_alen[b])):
                    scale_rows[b, h, p + 1 + d] = moved[h][d]
            text[b] += [int(ids[b, j]) for j in w_path[b, :w_alen[b]]] + [int(w_bonus[b])]
            assert int(dpl[b]) == len(text[b]) - 1
        assert war.war_device_status() == 0


@pytest.mark.parametrize("N", [3, 24])                           # 12 and 96 query rows per kv head
def test_pages_far_into_a_pool(war, N):
    """Store, attention and commit in a pool of more than 2^32 bytes give what they give in a small one."""
    rng = np.random.default_rng(61)
    B, Hq, Hkv, page, P = 2, 8, 2, 16, 8
    prefix = np.array([37, 200], np.int32)
    pt, total = Q.pages(rng, prefix + N, page)
    far = (1 << 20) + 40 - total                                 # 4096 bytes a page
    nn, parent = Q.trees(rng, B, N, full=True)
    ck, sk = Q.cache(rng, "e4m3", total, Hkv, page, 16, pow2=True)
    cv, sv = Q.cache(rng, "e4m3", total, Hkv, page, 16, pow2=True)
    g = torch.Generator().manual_seed(61)
    q, k, v = (torch.randn((B, N, h, 128), generator=g).to(torch.bfloat16).to(DEV) for h in (Hq, Hkv, Hkv))
    freq = war.war_rope_frequencies(128, 10000.0)[0].to(DEV)
    alen = dev(np.array([1, 2], np.int32))
    path = np.full((B, N), -1, np.int32)
    path[0, 0], path[1, :2] = 1, [1, 2]
    ids, bonus = dev(rng.integers(0, 99, (B, N)).astype(np.int32)), dev(np.array([5, 6], np.int32))
    results = []
    for shift in (0, far):
        pools = []
        for codes, scale in ((ck, sk), (cv, sv)):
            big, s = torch.empty((shift + total, Hkv, page, 128), dtype=torch.uint8, device=DEV), torch.ones((shift + total, Hkv, 1), device=DEV)
            big[shift:], s[shift:] = dev(codes), dev(scale)
            pools += [big.view(torch.float8_e4m3fn), s]
        kp, ks, vp, vs = pools
        table = dev(np.where(pt < total, pt + shift, pt).astype(np.int32))
        dpl, tail, tl = dev(prefix), torch.zeros((B, P), dtype=torch.int32, device=DEV), dev(np.array([3, 8], np.int32))
        out, lse, q_rot = torch.zeros_like(q), torch.zeros((B, N, Hq), device=DEV), torch.zeros_like(q)
        war.war_rope_store(q, k, v, freq, table, dpl, dev(nn), dev(parent), kp, vp, ks, vs, q_rot)
        params = war.attn_quant_params(q_rot, kp, vp, ks, vs, table, 128 ** -0.5)
        war.war_verify_attn_quant(q_rot, kp, vp, ks, vs, table, dpl, dev(nn), dev(parent), params, war.new_quant_workspace(params, DEV), out, lse)
        war.war_commit_quant(ids, alen, dev(path), bonus, kp, vp, ks, vs, table, dpl, tail, tl)
        torch.cuda.synchronize()
        assert war.war_device_status() == 0
        results.append([out, lse, q_rot, dpl, tail, tl] + [x[shift:].view(torch.uint8) if x.dim() == 4 else x[shift:] for x in pools])
    for a, b in zip(*results):
        assert torch.equal(a, b)


def test_steps_in_graphs_on_two_streams(war):
    """Store, attention, choice and commit of two batches, each captured into a graph with its own buffers and replayed at the
    same time on streams of their own, give what the calls give one after the other."""
    rng = np.random.default_rng(62)
    B, N, Hq, Hkv, page, V, P = 3, 6, 8, 2, 16, 3000, 8

    class Batch:
        def __init__(self, seed):
            prefix = np.array([30, 15, 700], np.int32)
            self.pt, total = Q.pages(rng, prefix + 8 * N, page)
            self.nn, self.parent = Q.trees(rng, B, N, full=True)
            self.start = [Q.to_device(c, "e4m3", False) if c.dtype == np.uint8 else dev(c)
                          for c in (*Q.cache(rng, "e4m3", total, Hkv, page, 16, pow2=True), *Q.cache(rng, "e4m3", total, Hkv, page, 16, pow2=True))]
            g = torch.Generator().manual_seed(seed)
            self.q, self.k, self.v = (torch.randn((B, N, h, 128), generator=g).to(torch.bfloat16).to(DEV) for h in (Hq, Hkv, Hkv))
            self.logits = torch.randn((B, N, V), generator=g).to(DEV)
            self.prefix, self.tail, self.tail_len = prefix, rng.integers(0, V, (B, P)).astype(np.int32), np.full(B, P, np.int32)
            self.ids, self.bonus = dev(rng.integers(0, V, (B, N)).astype(np.int32)), dev(np.array([1, 2, 3], np.int32))
            path = np.full((B, N), -1, np.int32)
            path[:, 0] = 1
            self.path, self.alen = dev(path), dev(np.array([1, 1, 0], np.int32))
            self.table, self.d_nn, self.d_par = dev(self.pt), dev(self.nn), dev(self.parent)
            self.freq = war.war_rope_frequencies(128, 10000.0)[0].to(DEV)
            self.rep = torch.full((B,), 1.2, device=DEV)
            self.ctx, self.off = dev(rng.integers(0, V, 90).astype(np.int32)), dev(np.array([0, 30, 60, 90], np.int64))
            self.out, self.lse, self.q_rot = torch.zeros_like(self.q), torch.zeros((B, N, Hq), device=DEV), torch.zeros_like(self.q)
            self.target = torch.zeros((B, N), dtype=torch.int32, device=DEV)
            self.reset()
            self.params = war.attn_quant_params(self.q_rot, *self.pools[::2], *self.pools[1::2], self.table, 128 ** -0.5)
            self.ws = war.new_quant_workspace(self.params, DEV)

        def reset(self):
            if not hasattr(self, "pools"):
                self.pools = [t.clone() for t in self.start]
                self.pools[0], self.pools[2] = self.pools[0].view(torch.float8_e4m3fn), self.pools[2].view(torch.float8_e4m3fn)
                self.state = [dev(self.prefix), dev(self.tail), dev(self.tail_len)]
            for t, s in zip(self.pools, self.start):
                t.view(torch.uint8).copy_(s.view(torch.uint8))
            for t, s in zip(self.state, (self.prefix, self.tail, self.tail_len)):
                t.copy_(dev(s))

        def step(self):
            kp, ks, vp, vs = self.pools
            war.war_rope_store(self.q, self.k, self.v, self.freq, self.table, self.state[0], self.d_nn, self.d_par, kp, vp, ks, vs, self.q_rot)
            war.war_verify_attn_quant(self.q_rot, kp, vp, ks, vs, self.table, self.state[0], self.d_nn, self.d_par, self.params, self.ws, self.out, self.lse)
            war.war_target(self.logits, self.d_nn, self.ids, self.d_par, self.target, d_ctx=self.ctx, d_ctx_off=self.off, d_repetition=self.rep)
            war.war_commit_quant(self.ids, self.alen, self.path, self.bonus, kp, vp, ks, vs, self.table, *self.state)

        def results(self):
            return [t.clone() for t in (self.out, self.lse, self.q_rot, self.target, *self.state)] + [t.view(torch.uint8).clone() for t in self.pools]

    batches = [Batch(1), Batch(2)]
    want = []
    for b in batches:
        for _ in range(3):                                       # three steps: the prefix advances
            b.step()
        want.append(b.results())
        b.reset()
    torch.cuda.synchronize()
    streams, graphs = [torch.cuda.Stream() for _ in batches], []
    for b in batches:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            b.step()
        graphs.append(g)
    for _ in range(3):
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    assert war.war_device_status() == 0
    for b, w in zip(batches, want):
        for x, y in zip(b.results(), w):
            assert torch.equal(x, y)
