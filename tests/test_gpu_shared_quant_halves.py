"""Attention over shared prefixes on the 8-bit cache above 64 query rows per request and kv head, held to what weights as halves give.

Tolerances.  A weight w = p * (V's scale) is rounded once, to a half that is 2^7 or more for the largest w that the row's reference allows
for (the reference follows the largest p * scale of the keys seen): half a step is 2^-11 of w, or 2^-25 / 2^7 = 2^-32 of that largest one.  p goes
into its sum in 32 bits.  With the output's own rounding, per element
    |error| <= 2^-8 |out| + 1.05 * sum_k |code_k| * max(2^-11 w_k, 2^-32 max_j w_j) / sum p
over the keys that the row sees (1.05: 32-bit arithmetic; the queries here are exact).  Two keys of nearly the same weight and opposite values
leave little of the first term, so that the second one is what is tested: weights held to 2^-8 of themselves miss it by far."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as O
from tests import quant_util as Q
from tests.test_gpu_attention_quant_scales import place, scales_at, set_keys
from tests.test_gpu_shared_quant_scales import Shared

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def war():
    from paper_2607_17299_b200 import binding
    return binding


def expected(c, i, rounded=None):
    """(out, bound) of request i in 64 bits; rounded: what the weights are rounded to."""
    page, block = c.ck.shape[2], c.ck.shape[2] // c.sk.shape[2]
    n, pl = int(c.nn[i]), int(c.prefix[i])
    pos = np.arange(pl + n)
    pg, r = c.pt[i, pos // page], pos % page
    see = np.zeros((n, pl + n), bool)
    see[:, :pl] = True
    for j in range(n):
        a = j
        while a >= 0:
            see[j, pl + a] = True
            a = int(c.parent[i, a])
    out, bound = np.zeros((n, c.Hq, 128)), np.zeros((n, c.Hq, 128))
    K = O.decode(c.ck[pg, 0, r], c.kv) * c.sk[pg, 0, r // block, None].astype(np.float64)
    code, s = O.decode(c.cv[pg, 0, r], c.kv), c.sv[pg, 0, r // block].astype(np.float64)
    for g in range(c.Hq):
        x = np.where(see, c.q[i, :n, g].double().numpy() @ K.T * c.scale, -np.inf)
        p = np.exp(x - x.max(1, keepdims=True))
        w, total = p * s, p.sum(1, keepdims=True)
        if rounded is not None:
            w = torch.from_numpy(w).to(rounded).double().numpy()
        out[:, g] = w @ code / total
        held = np.where(see, np.maximum(2.0 ** -11 * w, 2.0 ** -32 * w.max(1, keepdims=True)), 0)
        bound[:, g] = 2.0 ** -8 * np.abs(out[:, g]) + 1.05 * (held @ np.abs(code)) / total
    return out, bound


def two_keys(seed, kv, N, a, b, dot, values):
    """Nothing counts but positions a and b, whose products with a query of ones are 0 and dot."""
    c = Shared(seed, kv, 712, N, 16, 8)
    dots = np.full(712 + N, -40.0)
    dots[a], dots[b] = 0.0, dot
    set_keys(c, dots)
    rng = np.random.default_rng(seed)
    va = torch.from_numpy(rng.standard_normal(128) * 40)
    for x, v in ((a, va if values else torch.zeros_like(va)), (b, -va if values else torch.full_like(va, 448.0))):
        for i in range(3):
            c.cv[c.pt[i, x // 16], :, x % 16] = v.to(Q.KV_DTYPE[kv]).view(torch.uint8).numpy()
    c.sv[:] = 0.7
    return c


def check(c, out):
    got = out.double().cpu().numpy()
    for i in range(3):
        want, bound = expected(c, i)
        err = np.abs(got[i] - want)
        assert (err <= bound).all(), (i, float((err / bound).max()))


# positions: shared keys lie below 704, a request's own from there on
@pytest.mark.parametrize("N", [17, 24, 64])
@pytest.mark.parametrize("kv", ["e4m3", "e5m2"])
@pytest.mark.parametrize("a,b", [(3, 100), (200, 650), (40, 709), (710, 500), (705, 711)])
def test_two_keys_that_cancel(war, N, kv, a, b):
    c = two_keys(a + N, kv, N, a, b, -0.125, True)
    g = torch.Generator().manual_seed(b)
    c.q = (0.5 + 0.5 * torch.rand((3, N, 4, 1), generator=g)).to(torch.bfloat16).expand(3, N, 4, 128).contiguous()
    if a // 8 != b // 8:
        scales_at(c, [b], np.float32(0.7 * np.exp(0.125 * 0.75)), 8)
    place(c)
    out, _ = c.shared_run(war)
    check(c, out)
    assert war.war_device_status() == 0
    want, bound = expected(c, 0)                                                 # the bound tells weights with eight bits apart
    coarse, _ = expected(c, 0, torch.bfloat16)
    assert (np.abs(coarse - want) > bound).any(-1).mean() > 0.3


@pytest.mark.parametrize("N", [17, 64])
@pytest.mark.parametrize("kv", ["e4m3", "e5m2"])
@pytest.mark.parametrize("a,b", [(3, 100), (40, 709)])
@pytest.mark.parametrize("bits", [4, 12, 18, 20, 22, 24, 26])
def test_a_large_value_of_little_weight(war, N, kv, a, b, bits):
    """A key of weight 1 that is 0, and one of weight 2^-bits: halves below the smallest normal one are there, too."""
    c = two_keys(bits, kv, N, a, b, -bits * np.log(2), False)
    for i in range(3):                                                           # (the others are 0)
        L = int(c.prefix[i]) + N
        for x in range(L):
            if x != b:
                c.cv[c.pt[i, x // 16], :, x % 16] = 0
    place(c)
    out, _ = c.shared_run(war)
    check(c, out)
    assert war.war_device_status() == 0
