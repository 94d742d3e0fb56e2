"""GPU parity: war_verify_attn_quant against the fp64 checker on the values the 8-bit cache stands for.

Tolerances.  A weight p * (V's scale) reaches the tensor cores as two 8-bit parts that hold it to 2^-8 of itself (high part
e4m3: at most 2^-4 off, the remainder's e5m2 code at most 2^-3 of that, and half a step of 2^-16 at the type's lower end);
the largest weight of a row is scaled to at least 14 (28 times p, and p is relative to a reference at most a factor of 2
above the row's maximum).  The output's bf16 adds 2^-8 of itself.  So per element
    |error| <= 2^-8 |out| + 1.05 * (2^-8 * sum w |v| + keys * 2^-17 / 14 * max |v|)
(w: weights that sum to 1; the last term relative to the sum of weights where the largest counts 1, which is at least 1), and
because the roundings are independent the root mean square over many elements stays below 2^-8 of the output's.  The
log-sum-exp sees only 32-bit arithmetic and queries held to 2^-18 of a row's largest."""
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
    def __init__(self, seed, kv, prefix, N, Hq, Hkv, page, block, token_major=False, spread=0.3, dirty=True, q_scale=1.0, full=False):
        rng = np.random.default_rng(seed)
        self.kv, self.N, self.Hq, self.Hkv = kv, N, Hq, Hkv
        B = len(prefix)
        self.prefix = np.asarray(prefix, np.int32)
        self.nn, self.parent = Q.trees(rng, B, N, full)
        self.pt, total = Q.pages(rng, self.prefix + N, page)
        self.ck, self.sk = Q.cache(rng, kv, total, Hkv, page, block, spread)
        self.cv, self.sv = Q.cache(rng, kv, total, Hkv, page, block, spread)
        if dirty:                                   # rows and scales that no live position uses hold NaN
            live = np.zeros((total, page), bool)
            for i in range(B):
                for x in range(int(self.prefix[i] + self.nn[i])):
                    live[self.pt[i, x // page], x % page] = True
            for c, s in ((self.ck, self.sk), (self.cv, self.sv)):
                c[np.broadcast_to(~live[:, None, :], c.shape[:3])] = 0x7F
                dead = ~live.reshape(total, page // block, block).any(-1)
                s[np.broadcast_to(dead[:, None, :], s.shape)] = np.nan
        g = torch.Generator().manual_seed(seed)
        self.q = (torch.randn((B, N, Hq, 128), generator=g) * q_scale).to(torch.bfloat16)
        self.scale = 1.0 / np.sqrt(128) / q_scale
        self.d_q = self.q.to(DEV)
        self.k, self.v = Q.to_device(self.ck, kv, token_major), Q.to_device(self.cv, kv, token_major)
        t = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(DEV)
        self.dsk, self.dsv, self.dpt, self.dpl, self.dnn, self.dpar = t(self.sk), t(self.sv), t(self.pt), t(self.prefix), t(self.nn), t(self.parent)

    def args(self, war, kernel=0):
        p = war.attn_quant_params(self.d_q, self.k, self.v, self.dsk, self.dsv, self.dpt, self.scale, kernel)
        ws = war.new_quant_workspace(p, DEV)
        out = torch.full(self.d_q.shape, 7.0, dtype=torch.bfloat16, device=DEV)
        lse = torch.full(self.d_q.shape[:3], 7.0, device=DEV)
        return (self.d_q, self.k, self.v, self.dsk, self.dsv, self.dpt, self.dpl, self.dnn, self.dpar, p, ws, out, lse)

    def run(self, war, kernel=0):
        a = self.args(war, kernel)
        war.war_verify_attn_quant(*a)
        torch.cuda.synchronize()
        return a[-2], a[-1]

    def check(self, out, lse, requests=None):
        got, got_lse = out.float().cpu().numpy().astype(np.float64), lse.cpu().numpy()
        page, block = self.ck.shape[2], self.ck.shape[2] // self.sk.shape[2]
        for i in range(len(self.prefix)) if requests is None else requests:
            n, L = int(self.nn[i]), int(self.prefix[i] + self.nn[i])
            pos = np.arange(L)
            pg, r = self.pt[i, pos // page], pos % page
            K = O.decode(self.ck[pg, :, r], self.kv) * self.sk[pg, :, r // block][..., None]
            V = O.decode(self.cv[pg, :, r], self.kv) * self.sv[pg, :, r // block][..., None]
            q = self.q[i].double().numpy()
            want, want_lse = A.verify_attention_request(q, K, V, int(self.prefix[i]), self.parent[i], n, self.scale)
            mass, _ = A.verify_attention_request(q, K, np.abs(V), int(self.prefix[i]), self.parent[i], n, self.scale)
            top = np.repeat(np.abs(V).max(axis=(0, 2)), self.Hq // self.Hkv)[None, :, None]
            bound = 2.0 ** -8 * np.abs(want) + 1.05 * (2.0 ** -8 * mass + L * 2.0 ** -17 / 14 * top)
            err = np.abs(got[i, :n] - want)
            assert (err <= bound).all(), (i, float((err / bound).max()))
            if want.size >= 2048:
                rel = np.linalg.norm(got[i, :n] - want) / np.linalg.norm(want)
                assert rel < 2.0 ** -8, (i, rel)
            np.testing.assert_allclose(got_lse[i, :n], want_lse, atol=1e-4, rtol=1e-5)
            assert (got[i, n:] == 7.0).all() and (got_lse[i, n:] == 7.0).all()


CASES = [
    # seed, kv, prefixes, N, Hq, Hkv, page, block, token_major
    (1, "e4m3", [0, 1, 127, 128, 129, 500], 1, 8, 2, 16, 16, False),
    (2, "e4m3", [0, 15, 16, 300, 1023, 2000], 8, 8, 2, 16, 8, False),
    (3, "e5m2", [700, 3, 0, 255], 32, 8, 2, 32, 32, True),
    (4, "e4m3", [40, 900], 64, 16, 2, 64, 16, True),            # 512 rows per kv head: four row blocks
    (5, "e4m3", [5000], 24, 4, 1, 8, 8, False),
    (6, "e5m2", [260, 1500, 90], 17, 15, 3, 128, 32, False),    # five query heads a group
    (7, "e4m3", [8000, 10], 3, 1, 1, 128, 128, True),
]


@pytest.mark.parametrize("kernel", [1, 0, 2])
@pytest.mark.parametrize("case", CASES, ids=[str(c[0]) for c in CASES])
def test_matches_checker(war, case, kernel):
    c = Case(*case)
    c.check(*c.run(war, kernel))
    assert war.war_device_status() == 0


@pytest.mark.parametrize("seed", range(6))
def test_random_shapes(war, seed):
    rng = np.random.default_rng(900 + seed)
    page = int(rng.choice([8, 16, 32, 64, 128]))
    block = int(rng.choice([b for b in (8, 16, 32, 64, 128) if b <= page]))
    Hkv, G = int(rng.integers(1, 4)), int(rng.choice([1, 2, 3, 7, 8]))
    N = int(rng.integers(1, min(64, 512 // G) + 1))
    prefix = rng.integers(0, 1500, int(rng.integers(1, 6)))
    c = Case(seed, str(rng.choice(["e4m3", "e5m2"])), prefix, N, Hkv * G, Hkv, page, block, bool(rng.integers(2)), spread=1.0)
    c.check(*c.run(war))


def test_long_contexts_split_over_blocks(war):
    c = Case(11, "e4m3", [60000, 100, 20001], 8, 4, 1, 16, 16, full=True)
    out, lse = c.run(war)
    c.check(out, lse)
    out2, lse2 = c.run(war, 2)
    assert torch.equal(out, out2) and torch.equal(lse, lse2)     # where the parts are merged does not matter


def test_contiguous_split(war):
    c = Case(12, "e4m3", [9000, 12000, 15000, 7000, 30000, 11111], 4, 16, 4, 16, 16)
    out, lse = c.run(war)
    c.check(out, lse, requests=[0, 3, 4])
    again = c.run(war)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


def test_more_requests_than_one_launch_takes(war):
    rng = np.random.default_rng(5)
    c = Case(13, "e5m2", rng.integers(0, 400, 70), 5, 4, 2, 16, 16, True)
    c.check(*c.run(war))


def test_wide_range_of_scales(war):
    """Scales of neighbouring blocks that differ by up to 2^20, and blocks whose scale is 0."""
    c = Case(14, "e4m3", [900, 300], 6, 4, 2, 16, 8, spread=4.0, dirty=False)
    c.sv[::7] = 0
    c.sk[::11] = 0
    c.sk = np.minimum(c.sk, 2.0).astype(np.float32)
    c.dsk, c.dsv = torch.from_numpy(c.sk).to(DEV), torch.from_numpy(c.sv).to(DEV)
    for kernel in (1, 0):
        out, lse = c.run(war, kernel)
        c.check(out, lse)


@pytest.mark.parametrize("q_scale", [1e-30, 1e-4, 3000.0, 1e30])
def test_query_magnitudes(war, q_scale):
    c = Case(15, "e4m3", [400, 77], 9, 8, 2, 16, 16, q_scale=q_scale)
    c.check(*c.run(war))


def test_one_key_takes_all_and_zero_queries(war):
    c = Case(16, "e4m3", [3000], 4, 4, 2, 16, 16, full=True)
    c.q[:, 0] = 0
    c.q[:, 1] *= 40                                              # logits of +-100: one weight near 1
    c.d_q = c.q.to(DEV)
    c.check(*c.run(war))


@pytest.mark.parametrize("N,B", [(3, 6), (24, 6), (3, 70)])
def test_requests_without_slots(war, N, B):
    """num_nodes 0: the request's rows of out and lse stay as they are, whatever its prefix."""
    rng = np.random.default_rng(92)
    c = Case(92, "e4m3", rng.integers(0, 900, B).tolist(), N, 8, 2, 16, 16, full=True)
    c.nn[1::3] = 0
    c.dnn = torch.from_numpy(c.nn).to(DEV)
    out, lse = c.run(war)
    c.check(out, lse, [i for i in range(B) if c.nn[i] > 0])
    for i in range(1, B, 3):
        assert (out[i] == 7.0).all() and (lse[i] == 7.0).all()
    assert war.war_device_status() == 0


@pytest.mark.parametrize("kernel", [0, 1])
@pytest.mark.parametrize("N", [4, 8, 24])                       # 16, 32 and 96 query rows
def test_many_small_weights(war, N, kernel):
    """One key with a weight of 1 and 60000 with 2^-14.3 each, which together outweigh it four times: what a long context
    behind its first token looks like.  None of the small ones may be lost, and as they are all the same their roundings
    do not cancel: half a step of 2^-16, relative to at least 14, each."""
    c = Case(90, "e4m3", [60000], N, 4, 1, 64, 64, dirty=False, spread=0.0)
    rng = np.random.default_rng(91)
    code = lambda x: torch.as_tensor(x, dtype=torch.float32).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    c.q = torch.ones_like(c.q)
    c.ck[:] = 0
    c.ck[c.pt[0, 0], 0, 5] = code(0.875)
    c.cv[:] = code(1 + 0.25 * rng.standard_normal(c.cv.shape))
    c.sk[:], c.sv[:] = 1.0, 1.0
    c.d_q, c.k, c.v = c.q.to(DEV), Q.to_device(c.ck, c.kv, False), Q.to_device(c.cv, c.kv, False)
    c.dsk, c.dsv = torch.from_numpy(c.sk).to(DEV), torch.from_numpy(c.sv).to(DEV)
    out, lse = c.run(war, kernel)
    c.check(out, lse)
    n, L = int(c.nn[0]), int(c.prefix[0] + c.nn[0])
    pg, r = c.pt[0, np.arange(L) // 64], np.arange(L) % 64
    K, V = O.decode(c.ck[pg, :, r], c.kv), O.decode(c.cv[pg, :, r], c.kv)
    want, want_lse = A.verify_attention_request(c.q[0].double().numpy(), K, V, 60000, c.parent[0], n, c.scale)
    weight = np.exp(want_lse - 128 * 0.875 * c.scale)[:, :, None]          # of all keys, that of the largest being 1
    bound = 2.0 ** -7 * np.abs(want) + 1.05 * L * 2.0 ** -17 / 14 * np.abs(V).max() / weight
    err = np.abs(out[0, :n].double().cpu().numpy() - want)
    assert (err <= bound).all(), float((err / bound).max())


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_nan_and_infinite_queries_stay_in_their_rows(war, bad):
    c = Case(17, "e4m3", [700], 6, 4, 2, 16, 16, full=True)
    clean = c.run(war)
    c.q[0, 2, 1, 5] = bad
    c.d_q = c.q.to(DEV)
    for kernel in (0, 2):
        out, lse = c.run(war, kernel)
        assert torch.isnan(out[0, 2, 1]).all() and torch.isnan(lse[0, 2, 1])
        keep = torch.ones(out.shape[:3], dtype=torch.bool, device=DEV)
        keep[0, 2, 1] = False
        assert torch.equal(out[keep], clean[0][keep]) and torch.equal(lse[keep], clean[1][keep])


def test_bad_requests_are_left_alone(war):
    c = Case(18, "e4m3", [200, 300, 400, 500], 8, 8, 2, 16, 16, full=True)
    par, nn, pl = c.dpar.clone(), c.dnn.clone(), c.dpl.clone()
    c.dpar[1, 3] = 3                                             # its own parent
    c.dnn[2] = 9                                                 # more than N
    for kernel in (1, 0, 2):
        out, lse = c.run(war, kernel)
        assert (out[1] == 7).all() and (out[2] == 7).all() and (lse[1] == 7).all()
        c.check(out, lse, requests=[0, 3])
        assert war.war_device_status() == 7
    c.dpar, c.dnn = par, nn
    c.dpl = pl.clone(); c.dpl[0] = 100000                        # beyond the page table
    out, _ = c.run(war)
    assert (out[0] == 7).all() and war.war_device_status() == 8
    c.dpl = pl
    c.dpt = c.dpt.clone(); c.dpt[3, 2] = 1 << 20                 # a page outside the pool: reported, others unharmed
    out, lse = c.run(war)
    c.check(out, lse, requests=[0, 1, 2])
    assert war.war_device_status() == 8


def test_graph_replay_and_two_streams(war):
    a, b = Case(19, "e4m3", [4000, 900], 8, 8, 2, 16, 16), Case(20, "e5m2", [3000, 100, 5000], 16, 4, 1, 32, 32, True)
    want = a.run(war), b.run(war)
    args = a.args(war), b.args(war)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        with torch.cuda.stream(s1):
            war.war_verify_attn_quant(*args[0])
        with torch.cuda.stream(s2):
            war.war_verify_attn_quant(*args[1])
    torch.cuda.synchronize()
    for x, w in zip(args, want):
        assert torch.equal(x[-2], w[0]) and torch.equal(x[-1], w[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        war.war_verify_attn_quant(*args[0])
    for _ in range(3):
        args[0][-2].zero_()
        g.replay()
    torch.cuda.synchronize()
    live = torch.arange(a.N, device=DEV) < a.dnn[:, None]
    assert torch.equal(args[0][-2][live], want[0][0][live])


def test_no_lse_and_empty_batch(war):
    c = Case(21, "e4m3", [100], 2, 4, 2, 16, 16)
    a = list(c.args(war))
    a[-1] = None
    war.war_verify_attn_quant(*a)
    c.check(a[-2], c.run(war)[1])
    c.dnn.zero_()
    out, lse = c.run(war)
    assert (out == 7).all() and (lse == 7).all() and war.war_device_status() == 0


@pytest.mark.parametrize("N,B,page", [(3, 33, 32), (24, 8, 16)])
def test_long_units_give_the_same_bits_again_and_again(war, N, B, page):
    """Units of hundreds of tiles over a gigabyte of scattered pages, launched back to back: loads come late and out of order, and
    no launch may use one before it is there."""
    Hq, Hkv, L = 8, 2, 54648
    g = torch.Generator(DEV).manual_seed(93)
    pages = -(-(L + N) // page)
    table = torch.randperm(B * pages, generator=g, device=DEV).to(torch.int32).view(B, pages)
    k, v = (torch.randint(0, 0x78, (B * pages, page, Hkv, 128), generator=g, device=DEV, dtype=torch.uint8).view(torch.float8_e4m3fn).permute(0, 2, 1, 3)
            for _ in range(2))
    ks, vs = (torch.full((B * pages, Hkv, 1), 2.0 ** -8, device=DEV) for _ in range(2))
    q = torch.randn((B, N, Hq, 128), generator=g, device=DEV).to(torch.bfloat16)
    nn, prefix = torch.full((B,), N, dtype=torch.int32, device=DEV), torch.full((B,), L, dtype=torch.int32, device=DEV)
    parent = (torch.arange(N, device=DEV, dtype=torch.int32) - 1).expand(B, N).contiguous()
    params = war.attn_quant_params(q, k, v, ks, vs, table, 0.05)
    ws, out, lse = war.new_quant_workspace(params, DEV), torch.zeros_like(q), torch.zeros((B, N, Hq), device=DEV)
    call = lambda: war.war_verify_attn_quant(q, k, v, ks, vs, table, prefix, nn, parent, params, ws, out, lse)
    call()
    torch.cuda.synchronize()
    first = out.clone(), lse.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(10):
            call()
    for _ in range(5):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1])
    assert war.war_device_status() == 0
