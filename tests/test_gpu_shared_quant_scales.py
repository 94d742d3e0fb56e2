"""Attention over shared prefixes on the 8-bit cache where V's scales differ widely between blocks: the cases and bounds of
test_gpu_attention_quant_scales.py (they hold for weights in two 8-bit parts, and for weights as halves, 2^-11, all the more), with two
requests that share the pages of their prefix and one that has its own."""
import numpy as np
import pytest
import torch

from tests import quant_util as Q
from tests.test_gpu_attention_quant import Case
from tests.test_gpu_attention_quant_scales import DEV, check, place, scales_at, set_keys

pytestmark = pytest.mark.gpu
ROWS = [4, 16, 17, 24, 64]                        # slots: 16 to 256 query rows per kv head, around the change of kernels at 64


@pytest.fixture(scope="module")
def war():
    from paper_2607_17299_b200 import binding
    return binding


class Shared(Case):
    def __init__(self, seed, kv, prefix, N, page, block, share=True):
        super().__init__(seed, kv, [prefix] * 3, N, 4, 1, page, block, dirty=False, full=True)
        if share:
            self.pt[1, :prefix // page] = self.pt[0, :prefix // page]
            self.dpt = torch.from_numpy(np.ascontiguousarray(self.pt)).to(DEV)
        self.leader = torch.tensor([0, 0, 2] if share else [0, 1, 2], dtype=torch.int32, device=DEV)
        self.shared = torch.full((3,), prefix // page * page, dtype=torch.int32, device=DEV)

    def shared_run(self, war):
        *first, p, _, out, lse = self.args(war)
        war.war_verify_attn_shared_quant(*first, self.leader, self.shared, p, war.new_shared_quant_workspace(p, DEV), out, lse)
        torch.cuda.synchronize()
        return out, lse


@pytest.mark.parametrize("N", ROWS)
@pytest.mark.parametrize("bits", [12, 24, 60])
@pytest.mark.parametrize("kv,where", [("e4m3", 0), ("e5m2", 304), ("e4m3", 688)])
def test_a_large_scale_of_little_weight(war, N, bits, kv, where):
    c = Shared(50, kv, 704, N, 16, 16)
    dots = np.random.default_rng(51).standard_normal(800)
    block = range(where, where + 16)
    dots[list(block)] = -(bits + 12) * np.log(2)
    set_keys(c, dots)
    scales_at(c, block, c.sv.max() * 2.0 ** bits, 16)
    place(c)
    check(c, *c.shared_run(war))
    assert war.war_device_status() == 0


@pytest.mark.parametrize("N", ROWS)
@pytest.mark.parametrize("kv", ["e4m3", "e5m2"])
@pytest.mark.parametrize("prefix", [3, 700])
def test_a_slot_hidden_from_the_others_with_the_largest_scale(war, N, kv, prefix):
    page = 8
    prefix += -(prefix + N - 1) % page
    c = Shared(52, kv, prefix, N, page, 8)
    c.parent[:] = np.arange(N) - 1
    c.parent[:, N - 1] = 0
    c.dpar = torch.from_numpy(c.parent).to(DEV)
    last = prefix + N - 1
    scales_at(c, [last], 2.0 ** 120, 8)
    for i in range(3):
        c.cv[c.pt[i, last // page], :, 0] = torch.ones(128).to(Q.KV_DTYPE[kv]).view(torch.uint8).numpy()
    place(c)
    out, lse = c.shared_run(war)
    check(c, out, lse, rows=range(N - 1), whole=prefix > 100)
    check(c, out, lse, rows=[N - 1], whole=False)


@pytest.mark.parametrize("N", ROWS)
@pytest.mark.parametrize("low,high", [(-90, -70), (-20, 20), (-60, 100)])
def test_scales_from_tiny_to_huge(war, N, low, high):
    c = Shared(55, "e4m3", 896, N, 32, 8)
    rng = np.random.default_rng(56)
    e = rng.integers(low, high + 1, 124)
    set_keys(c, -np.repeat(e - low, 8) * np.log(2) + rng.standard_normal(992))
    for b in range((896 + N + 7) // 8):
        scales_at(c, [8 * b], 2.0 ** int(e[b]), 8)
    place(c)
    check(c, *c.shared_run(war), whole=False)


@pytest.mark.parametrize("N", ROWS)
@pytest.mark.parametrize("share", [True, False])
@pytest.mark.parametrize("first,rest", [(-90, -8), (-110, 60), (-61, -59)])
@pytest.mark.parametrize("prefix", [704, 9008])
def test_contexts_that_begin_with_tiny_scales(war, N, first, rest, prefix, share):
    c = Shared(57, "e4m3", prefix, N, 16, 8, share)
    set_keys(c, np.random.default_rng(58).standard_normal(prefix + N))
    c.sv[:] = 2.0 ** rest
    scales_at(c, range(0, 200, 8), 2.0 ** first, 8)
    place(c)
    check(c, *c.shared_run(war))


@pytest.mark.parametrize("N", ROWS)
@pytest.mark.parametrize("spread", [1e-30, 1e-3, 1e3, 1e30])
def test_queries_small_and_large(war, N, spread):
    """Rows of all magnitudes, and elements of all magnitudes below a row's largest."""
    c = Shared(59, "e5m2", 400, N, 16, 16)
    g = torch.Generator().manual_seed(60)
    c.q = (c.q.float() * torch.exp2(-torch.randint(0, 30, c.q.shape, generator=g)) * spread).to(torch.bfloat16)
    c.scale = 1.0 / spread / np.sqrt(128)
    c.d_q = c.q.to(DEV)
    out, lse = c.shared_run(war)
    c.check(out, lse)
    assert war.war_device_status() == 0
