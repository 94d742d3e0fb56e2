"""GPU parity: war_target against the plain checker.  Both compute in 32 bits with one rounding per operation, in the
documented order, so choices and processed logits are compared for equality (bf16 output: the same value rounded once)."""
import numpy as np
import pytest
import torch

from oracle import target_oracle as T
from tests import quant_util as Q

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def war():
    from paper_2607_17299_b200 import binding
    return binding


def dev(x):
    return None if x is None else torch.from_numpy(np.ascontiguousarray(x)).to(DEV)


class Case:
    def __init__(self, seed, B, N, V, dtype, ctx=200, bias=5, mask=0.5, shared_mask=False, pad=0, penal=(1.3, 0.5, 0.2), coarse=False):
        rng = np.random.default_rng(seed)
        self.B, self.N, self.V = B, N, V
        self.dtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.nn, self.parent = Q.trees(rng, B, N)
        x = rng.standard_normal((B, N, V)).astype(np.float32) * 3
        if coarse:
            x = np.round(x)                                     # many equal values
        self.logits = torch.from_numpy(x).to(self.dtype)
        buf = torch.full((B, N, V + pad), 99.0, dtype=self.dtype, device=DEV)     # rows that do not start on 16 bytes
        buf[:, :, pad // 2: pad // 2 + V] = self.logits.to(DEV)
        self.d_logits = buf[:, :, pad // 2: pad // 2 + V]
        lens = rng.integers(1, ctx + 1, B)
        self.off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
        self.ctx = (V * rng.random(int(self.off[-1])) ** 3).astype(np.int32)
        self.ctx[rng.random(len(self.ctx)) < 0.02] = V + 3      # outside the vocabulary
        self.prompt = (lens // 2).astype(np.int32)
        self.ids = rng.integers(0, V, (B, N)).astype(np.int32)
        self.ids[:, 1::3] = self.ctx[self.off[:-1]][:, None] % V      # drafts repeat a context token, and each other
        r = lambda k: (np.full(B, k) + 0.1 * rng.random(B)).astype(np.float32)
        self.rep, self.pres, self.freq = (None if k is None else r(k) for k in penal)
        cnt = rng.integers(0, bias + 1, B)
        self.boff = np.concatenate([[0], np.cumsum(cnt)]).astype(np.int64)
        self.bids = rng.integers(-1, V + 1, int(self.boff[-1])).astype(np.int32)
        if len(self.bids) > 1:
            self.bids[1] = self.bids[0]                         # the same token twice
        self.bval = (4 * rng.standard_normal(len(self.bids))).astype(np.float32)
        words = (V + 31) // 32
        self.mask = None
        if mask is not None:
            bits = rng.random((B, 1 if shared_mask else N, words * 32)) < mask
            self.allowed = bits[:, :, :V]
            w = (bits.reshape(*bits.shape[:2], words, 32).astype(np.uint64) << np.arange(32, dtype=np.uint64)).sum(-1).astype(np.uint32).view(np.int32)
            self.mask = dev(w)
            if shared_mask:
                self.mask = self.mask.expand(B, N, words)
                self.allowed = np.broadcast_to(self.allowed, (B, N, V))

    def kw(self):
        return dict(d_ctx=dev(self.ctx), d_ctx_off=dev(self.off), d_prompt_len=dev(self.prompt), d_repetition=dev(self.rep),
                    d_presence=dev(self.pres), d_frequency=dev(self.freq), d_bias_off=dev(self.boff), d_bias_ids=dev(self.bids),
                    d_bias_val=dev(self.bval), d_mask=self.mask)

    def run(self, war, out=None, **over):
        target = torch.full((self.B, self.N), -7, dtype=torch.int32, device=DEV)
        war.war_target(self.d_logits, dev(self.nn), dev(self.ids), dev(self.parent), target, d_out=out, **{**self.kw(), **over})
        torch.cuda.synchronize()
        return target.cpu().numpy()

    def want(self):
        x = self.logits.float().numpy()
        rows, target = {}, np.full((self.B, self.N), -1, np.int32)
        for b in range(self.B):
            ctx = self.ctx[self.off[b]:self.off[b + 1]]
            bias = list(zip(self.bids[self.boff[b]:self.boff[b + 1]].tolist(), self.bval[self.boff[b]:self.boff[b + 1]].tolist()))
            one = lambda a, d: d if a is None else a[b]
            for j in range(int(self.nn[b])):
                path, a = [], j
                while a > 0:
                    path.append(int(self.ids[b, a]))
                    a = int(self.parent[b, a])
                rows[b, j] = T.process_row(x[b, j], ctx, int(self.prompt[b]), path, one(self.rep, 1.0), one(self.pres, 0.0), one(self.freq, 0.0),
                                           bias, None if self.mask is None else self.allowed[b, j])
                target[b, j] = T.choose(rows[b, j])
        return rows, target

    def check(self, war, in_place=False):
        rows, want = self.want()
        got = self.run(war)
        np.testing.assert_array_equal(got, want)
        out = self.d_logits if in_place else torch.full((self.B, self.N, self.V), 55.0, dtype=self.dtype, device=DEV)
        before = self.d_logits.clone()
        np.testing.assert_array_equal(self.run(war, out=out), want)
        h = out.cpu()
        for b in range(self.B):
            for j in range(self.N):
                if j < self.nn[b]:
                    assert torch.equal(h[b, j].nan_to_num(nan=1e9), torch.from_numpy(rows[b, j]).to(self.dtype).nan_to_num(nan=1e9)), (b, j)
                else:
                    assert torch.equal(h[b, j], before[b, j].cpu()) if in_place else (h[b, j] == 55).all()
        assert war.war_device_status() == 0


CASES = [
    # seed, B, N, V, dtype, kwargs
    (1, 3, 1, 32000, "bf16", {}),
    (2, 2, 8, 32000, "bf16", dict(ctx=3000)),
    (3, 2, 5, 1009, "f32", dict(pad=1)),
    (4, 2, 5, 1009, "bf16", dict(pad=3)),
    (5, 2, 64, 77, "bf16", dict(pad=2, coarse=True)),
    (6, 1, 3, 131071, "f32", dict(pad=1, ctx=5000, bias=60)),
    (7, 1, 2, 262144, "bf16", {}),
    (8, 4, 4, 1, "f32", {}),
    (9, 3, 6, 33, "bf16", dict(pad=5, mask=0.03, coarse=True)),       # some rows have nothing left
    (10, 2, 4, 5000, "f32", dict(mask=None, bias=0)),
    (11, 2, 4, 5001, "bf16", dict(shared_mask=True, penal=(1.2, None, None))),
    (12, 2, 7, 4097, "bf16", dict(penal=(None, 0.7, None), pad=1, coarse=True)),
    (13, 2, 7, 9000, "f32", dict(penal=(0.7, -0.5, -0.3), coarse=True)),     # penalties that raise
    (14, 70, 2, 700, "bf16", dict(penal=(None, None, None))),
]


@pytest.mark.parametrize("case", CASES, ids=[str(c[0]) for c in CASES])
def test_matches_checker(war, case):
    Case(*case[:5], **case[5]).check(war)


MORE = [
    (41, 160, 3, 20000, "bf16", dict(coarse=True)),              # many requests: few slices, long pieces, ties across warps
    (42, 8, 12, 40000, "f32", dict(coarse=True, ctx=9000)),
    (43, 2, 9, 30001, "bf16", dict(pad=3, coarse=True, mask=0.002)),      # a grammar that leaves a token in 500
    (44, 2, 9, 30001, "f32", dict(pad=1, mask=0.0005, bias=40)),
    (47, 2, 3, 5000, "bf16", dict(bias=20000)),                  # most tokens have a bias, many have several
]


@pytest.mark.parametrize("case", MORE, ids=[str(c[0]) for c in MORE])
def test_matches_checker_at_size(war, case):
    Case(*case[:5], **case[5]).check(war)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["equal", "rising", "falling"])
def test_rows_that_are_hard_to_dismiss(war, kind, dtype):
    """All logits equal (zeros of both signs: the lowest token allowed wins), and rows where every value is a new largest one."""
    c = Case(45, 3, 7, 25013, dtype, pad=5, mask=0.5 if kind == "equal" else 0.9)
    V = c.V
    if kind == "equal":
        row = torch.where(torch.arange(V) % 3 == 0, torch.tensor(-0.0), torch.tensor(0.0))
    else:
        row = torch.linspace(-8, 8, V) if kind == "rising" else torch.linspace(8, -8, V)
    c.logits = row.to(c.dtype).expand(3, 7, V).clone()
    c.d_logits.copy_(c.logits)
    c.check(war)


@pytest.mark.parametrize("V", [8000, 7770, 8096])
def test_tables_around_the_shared_memory_limit(war, V):
    """A slice whose tables come to just below, about and just above the 48 KB that a launch has to ask for, the kernel's own variables
    included."""
    for W in range(V, V + 64, 32):
        c = Case(49, 1, 1, 4 * W, "bf16", ctx=30, bias=2)
        c.check(war)
    c = Case(50, 120, 1, 4 * V, "bf16", ctx=30, bias=2, mask=None)          # four slices
    c.check(war)


def test_requests_without_slots_and_many_requests(war):
    c = Case(48, 700, 2, 300, "bf16")
    c.nn[::3] = 0
    c.check(war)
    assert (c.run(war)[::3] == -1).all()


def test_logits_far_apart(war):
    """Requests 2^32 elements apart, in and out."""
    c = Case(46, 2, 3, 4001, "bf16")
    step = (1 << 32) + 4096
    buf = torch.empty(step + 3 * 4001, dtype=torch.bfloat16, device=DEV)
    far = buf.as_strided((2, 3, 4001), (step, 4001, 1))
    far.copy_(c.d_logits)
    c.d_logits = far
    rows, want = c.want()
    np.testing.assert_array_equal(c.run(war), want)
    np.testing.assert_array_equal(c.run(war, out=far), want)
    h = far.cpu()
    for (b, j), row in rows.items():
        assert torch.equal(h[b, j].nan_to_num(nan=1e9), torch.from_numpy(row).to(c.dtype).nan_to_num(nan=1e9))


def test_out_in_place(war):
    Case(31, 2, 6, 3001, "bf16", pad=3).check(war, in_place=True)


def test_special_values(war):
    c = Case(32, 1, 8, 2000, "f32", mask=None, bias=0, penal=(1.5, 0.0, 0.0))
    c.nn[:] = 8
    c.parent[0] = [-1, 0, 1, 2, 3, 4, 5, 6]
    x = c.logits
    x[0, 0] = -np.inf                                            # nothing above -inf
    x[0, 1] = np.nan
    x[0, 2, 5] = np.nan; x[0, 2, 7] = np.inf
    x[0, 3] = torch.finfo(torch.float32).min                     # the lowest value is a value
    x[0, 4] = -np.inf; x[0, 4, 1999] = -3e38
    x[0, 5] = -1.0; x[0, 5, 300] = -0.0; x[0, 5, 400] = 0.0      # equal: the lower token
    c.d_logits.copy_(x)
    c.check(war)
    got = c.run(war)[0]
    assert got[0] == -1 and got[1] == -1 and got[2] == 7 and got[4] == 1999


def test_without_trees_and_without_penalties(war):
    c = Case(33, 2, 4, 3000, "bf16", bias=3)
    target = torch.zeros((2, 4), dtype=torch.int32, device=DEV)
    war.war_target(c.d_logits, dev(c.nn), None, None, target)
    x = c.logits.float().numpy()
    for b in range(2):
        for j in range(4):
            assert int(target[b, j]) == (T.choose(x[b, j]) if j < c.nn[b] else -1)
    c.parent[:] = -1; c.parent[:, 1:] = 0; c.ids[:] = -1         # no path tokens either way
    rows, want = c.want()
    war.war_target(c.d_logits, dev(c.nn), None, None, target, **c.kw())
    np.testing.assert_array_equal(target.cpu().numpy(), want)


def test_hot_token_in_a_long_context(war):
    c = Case(34, 2, 2, 1000, "f32", ctx=10)
    c.ctx = np.where(np.random.default_rng(0).random(200000) < 0.5, 17, 900).astype(np.int32)
    c.off = np.array([0, 150000, 200000], np.int64)
    c.prompt = np.array([10, 50000], np.int32)
    c.freq[:] = 1e-4
    c.check(war)


def test_bad_requests(war):
    c = Case(35, 4, 5, 600, "bf16", bias=4)
    c.nn, c.parent = Q.trees(np.random.default_rng(35), 4, 5, full=True)
    rows, want = c.want()
    c.parent[1, 2] = 2
    c.nn[2] = 6
    out = torch.full((4, 5, 600), 55.0, dtype=c.dtype, device=DEV)
    got = c.run(war, out=out)
    assert (got[1] == -1).all() and (got[2] == -1).all() and (out[1] == 55).all() and (out[2] == 55).all()
    np.testing.assert_array_equal(got[[0, 3]], want[[0, 3]])
    assert war.war_device_status() == 7
    c.parent[1, 2] = 0; c.nn[2] = 5
    off = c.off.copy(); off[2] = off[1] - 1
    got = c.run(war, d_ctx_off=dev(off))
    assert (got[1] == -1).all() and war.war_device_status() == 1


def test_graph_replay(war):
    c = Case(36, 3, 4, 20000, "bf16")
    want = c.run(war)
    args = dict(c.kw())
    nn, ids, par = dev(c.nn), dev(c.ids), dev(c.parent)
    target = torch.zeros((3, 4), dtype=torch.int32, device=DEV)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        war.war_target(c.d_logits, nn, ids, par, target, **args)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        war.war_target(c.d_logits, nn, ids, par, target, **args)
    for _ in range(3):
        target.zero_()
        g.replay()
    torch.cuda.synchronize()
    np.testing.assert_array_equal(target.cpu().numpy(), want)
