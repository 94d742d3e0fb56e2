"""GPU parity of war_verify_attn_quant where V's scales differ widely between blocks, row by row.

Tolerances.  A weight w = p * (V's scale) reaches the tensor cores as two 8-bit parts.  With u = 448 / (largest w that the row's
reference allows for) and the reference at most 2^4 above the row's largest w (a stale one 2^3, a margin of 2), u * w of the
largest is at least 28.  Its parts: u * w / 256 as a half (2^-11 of itself, or half a step of 2^-16 / 256), rounded to a
high part of 4 bits, or to a step of 2^-9 below 2^-6; the rest, at most half of that step, to a low part of 3 bits, 2^-3 of
itself at most.  So u * w is held to (1 + 2^-3) * 2^-8 of itself, or to (1 + 2^-3) * 2^-14 where it is below 2^-6.  With the
output's own rounding, per element
    |error| <= 2^-8 |out| + 1.05 * sum_k |code_k| * max(1.125 * 2^-8 w_k, 1.125 * 2^-14 / 28 * max_j w_j) / sum p
over the keys that the row sees (1.05: 32-bit arithmetic, queries in two 8-bit parts).  Where many keys of similar weight share
a row the roundings are independent (root mean square 2^-9.6 for a weight, 2^-9.8 for the output's bf16), so a row's error as
a whole stays below 2^-8 of it."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as O
from tests import quant_util as Q
from tests.test_gpu_attention_quant import Case

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ROWS = [4, 8, 24, 64]                             # slots: 16, 32, 96 and (two row blocks) 256 query rows per kv head


@pytest.fixture(scope="module")
def war():
    from paper_2607_17299_b200 import binding
    return binding


def expected(c, i):
    """(out, lse, bound) of request i in 64 bits: [n, Hq, 128], [n, Hq], [n, Hq, 128]."""
    page, block = c.ck.shape[2], c.ck.shape[2] // c.sk.shape[2]
    n, pl = int(c.nn[i]), int(c.prefix[i])
    L, G = pl + n, c.Hq // c.Hkv
    pos = np.arange(L)
    pg, r = c.pt[i, pos // page], pos % page
    see = np.zeros((n, L), bool)
    see[:, :pl] = True
    for j in range(n):
        a = j
        while a >= 0:
            see[j, pl + a] = True
            a = int(c.parent[i, a])
    out, bound, lse = np.zeros((n, c.Hq, 128)), np.zeros((n, c.Hq, 128)), np.zeros((n, c.Hq))
    for h in range(c.Hkv):
        K = O.decode(c.ck[pg, h, r], c.kv) * c.sk[pg, h, r // block, None].astype(np.float64)
        code, s = O.decode(c.cv[pg, h, r], c.kv), c.sv[pg, h, r // block].astype(np.float64)
        for g in range(h * G, (h + 1) * G):
            x = np.where(see, c.q[i, :n, g].double().numpy() @ K.T * c.scale, -np.inf)
            top = x.max(1, keepdims=True)
            p = np.exp(x - top)
            w, total = p * s, p.sum(1, keepdims=True)
            out[:, g] = w @ code / total
            lse[:, g] = top[:, 0] + np.log(total[:, 0])
            held = np.where(see, np.maximum(1.125 * 2.0 ** -8 * w, 1.125 * 2.0 ** -14 / 28 * w.max(1, keepdims=True)), 0)
            bound[:, g] = 2.0 ** -8 * np.abs(out[:, g]) + 1.05 * (held @ np.abs(code)) / total
    return out, lse, bound


def check(c, out, lse, rows=None, whole=True):
    got, got_lse = out.double().cpu().numpy(), lse.cpu().numpy()
    for i in range(len(c.prefix)):
        want, want_lse, bound = expected(c, i)
        j = np.arange(want.shape[0]) if rows is None else np.asarray(rows)
        err = np.abs(got[i, j] - want[j])
        assert (err <= bound[j]).all(), (i, float((err / bound[j]).max()))
        if whole:
            rel = np.linalg.norm(err, axis=-1) / np.linalg.norm(want[j], axis=-1)
            assert rel.max() < 2.0 ** -8, (i, float(rel.max()))
        np.testing.assert_allclose(got_lse[i, j], want_lse[j], atol=1e-4, rtol=1e-5)


def set_keys(c, dots):
    """Keys whose product with queries of ones is dots[position] (rounded to the type), for every request and head."""
    c.q = torch.ones_like(c.q)
    c.scale, c.sk[:] = 1.0 / 128, 1.0
    page = c.ck.shape[2]
    code = torch.as_tensor(np.asarray(dots), dtype=torch.float32).to(Q.KV_DTYPE[c.kv]).view(torch.uint8).numpy()
    for i in range(len(c.prefix)):
        L = int(c.prefix[i] + c.nn[i])
        pos = np.arange(L)
        c.ck[c.pt[i, pos // page], :, pos % page] = code[:L, None, None]


def place(c, token_major=False):
    c.d_q, c.k, c.v = c.q.to(DEV), Q.to_device(c.ck, c.kv, token_major), Q.to_device(c.cv, c.kv, token_major)
    c.dsk, c.dsv = torch.from_numpy(c.sk).to(DEV), torch.from_numpy(c.sv).to(DEV)


def scales_at(c, at, scale, block):
    """The V scales of the blocks that hold positions at."""
    page = c.ck.shape[2]
    for i in range(len(c.prefix)):
        for x in at:
            c.sv[c.pt[i, x // page], :, x % page // block] = scale


@pytest.mark.parametrize("N", ROWS)
@pytest.mark.parametrize("bits", [12, 16, 20, 24, 60])
@pytest.mark.parametrize("kv,where", [("e4m3", 0), ("e5m2", 300), ("e4m3", 690)])
def test_a_large_scale_of_little_weight(war, N, bits, kv, where):
    """One block's V scale is 2^bits times the others', and its keys weigh 2^-(bits + 12) of them: what the row puts on the others
    is held as well as without it, wherever the block stands."""
    c = Case(50, kv, [700], N, 4, 1, 16, 16, dirty=False, full=True)
    dots = np.random.default_rng(51).standard_normal(800)
    block = range(where // 16 * 16, where // 16 * 16 + 16)
    dots[list(block)] = -(bits + 12) * np.log(2)
    set_keys(c, dots)
    scales_at(c, block, c.sv.max() * 2.0 ** bits, 16)
    place(c)
    for kernel in (1, 0, 2):
        check(c, *c.run(war, kernel))
    assert war.war_device_status() == 0


@pytest.mark.parametrize("N", ROWS)
@pytest.mark.parametrize("kv", ["e4m3", "e5m2"])
@pytest.mark.parametrize("prefix", [3, 700])
def test_a_slot_hidden_from_the_others_with_the_largest_scale(war, N, kv, prefix):
    """The last slot is a child of the root and a block of its own with the scale that an infinite value gets from the store; the
    other slots are a chain.  Their rows do not feel it, and the slot's own row has its value."""
    page = 8
    prefix += -(prefix + N - 1) % page
    c = Case(52, kv, [prefix], N, 4, 1, page, 8, dirty=False, full=True)
    c.parent[0] = np.arange(N) - 1
    c.parent[0, N - 1] = 0
    c.dpar = torch.from_numpy(c.parent).to(DEV)
    last = prefix + N - 1
    scales_at(c, [last], 2.0 ** 120, 8)
    c.cv[c.pt[0, last // page], :, 0] = torch.ones(128).to(Q.KV_DTYPE[kv]).view(torch.uint8).numpy()
    place(c)
    for kernel in (1, 0, 2):
        out, lse = c.run(war, kernel)
        check(c, out, lse, rows=range(N - 1), whole=prefix > 100)
        check(c, out, lse, rows=[N - 1], whole=False)


@pytest.mark.parametrize("N", ROWS)
def test_long_contexts_with_a_large_scale_of_little_weight(war, N):
    """Split over thread blocks: some parts hold the large scale, others do not."""
    c = Case(53, "e4m3", [20000, 9000], N, 4, 1, 16, 8, dirty=False, full=True)
    dots = np.random.default_rng(54).standard_normal(20100)
    far = [x for b in range(0, 9000, 1000) for x in range(b, b + 8)]
    dots[far] = -40 * np.log(2)
    set_keys(c, dots)
    scales_at(c, far, 2.0 ** 22, 8)
    place(c)
    for kernel in (0, 2):
        check(c, *c.run(war, kernel))


@pytest.mark.parametrize("N", ROWS)
@pytest.mark.parametrize("low,high", [(-90, -70), (-20, 20), (-60, 100)])
def test_scales_from_tiny_to_huge(war, N, low, high):
    """Random powers of two side by side, with weights that make up for them: every row is made of blocks of all scales."""
    c = Case(55, "e4m3", [900], N, 4, 1, 32, 8, dirty=False, full=True)
    rng = np.random.default_rng(56)
    e = rng.integers(low, high + 1, 124)
    dots = -np.repeat(e - low, 8) * np.log(2) + rng.standard_normal(992)
    set_keys(c, dots)
    for b in range((900 + N + 7) // 8):
        scales_at(c, [8 * b], 2.0 ** int(e[b]), 8)
    place(c)
    for kernel in (1, 0, 2):
        check(c, *c.run(war, kernel), whole=False)


@pytest.mark.parametrize("N", ROWS)
@pytest.mark.parametrize("first,rest", [(-90, -8), (-110, 60), (-61, -59)])
@pytest.mark.parametrize("prefix", [700, 9000])
def test_contexts_that_begin_with_tiny_scales(war, N, first, rest, prefix):
    """The first 200 keys have small scales, the others large ones: some tiles begin a group's or a thread block's share with scales below
    2^-60, others do not, and the parts meet."""
    c = Case(57, "e4m3", [prefix], N, 4, 1, 16, 8, dirty=False, full=True)
    dots = np.random.default_rng(58).standard_normal(prefix + N)
    set_keys(c, dots)
    c.sv[:] = 2.0 ** rest
    scales_at(c, range(0, 200, 8), 2.0 ** first, 8)
    place(c)
    for kernel in (1, 0, 2):
        check(c, *c.run(war, kernel))
