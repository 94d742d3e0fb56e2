"""Attention over shared prefixes where it could go wrong: groups that break the rules, trees and pages that do, requests that are not
running, values that are no numbers, capture and replay, several streams, the largest batches and pools.

Tolerances are those of test_gpu_attention_shared.py."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as A
from tests.test_gpu_attention_shared import DEV, Case

pytestmark = pytest.mark.gpu
INVALID, BAD_TREE, BAD_PAGE = 1, 7, 8
KINDS = [("bf16", 0), ("e4m3", 16), ("e5m2", 8)]                  # the last one with more than 64 rows per request and kv head


@pytest.fixture(scope="module")
def war():
    from paper_2607_17299_b200 import binding
    return binding


@pytest.fixture(autouse=True)
def clean(war):
    assert war.war_device_status() == 0
    yield
    torch.cuda.synchronize()


def group_case(kv, block, seed=21, **kw):
    return Case(seed, kv, [(256, [0, 130, 17]), (512, [9, 300]), (0, [40])], 6, 32 if block == 8 else 8, 2, 16, block, full=True, **kw)


def put(c):
    """The host's integers into the device's arrays."""
    for d, h in zip(c.ints, (c.pt, c.prefix, c.nn, c.parent, c.leader, c.shared)):
        d.copy_(torch.from_numpy(np.ascontiguousarray(h)))


def members(c):
    sets = {}
    for i, l in enumerate(c.leader.tolist()):
        sets.setdefault(l, []).append(i)
    return sorted([(l, m) for l, m in sets.items() if len(m) > 1], key=lambda x: -len(x[1]))           # (the group of three first)


@pytest.mark.parametrize("kv,block", KINDS)
@pytest.mark.parametrize("how", ["leader behind the last", "leader below 0", "leader that has one", "shared longer than a prefix", "shared below 0",
                                 "shared longer than the leader's"])
def test_members_that_break_the_rules(war, kv, block, how):
    """Their rows stay, the others' are right."""
    c = group_case(kv, block)
    (l0, m0), (l1, m1) = members(c)
    if how == "leader behind the last":
        victims = [next(i for i in m0 if i != l0)]
        c.leader[victims] = len(c.prefix)
    elif how == "leader below 0":
        victims = [next(i for i in m0 if i != l0)]
        c.leader[victims] = -1
    elif how == "leader that has one":                                # a member names a member
        victims = [next(i for i in m0 if i != l0)]
        c.leader[victims] = next(i for i in m1 if i != l1)
    elif how == "shared longer than a prefix":                        # 400 tokens: nobody in the group has them
        victims = [i for i in m0 if i != l0]                          # (the leader is left alone, and so for itself)
        c.shared[l0] = 400
        assert (c.prefix[m0] < 400).all()
    elif how == "shared below 0":
        victims = [i for i in m1 if i != l1]
        c.shared[l1] = -1
    else:
        victims = [i for i in m1 if c.prefix[i] < 528]                # 512 + 9: the short one only
        c.shared[l1] = 528
        assert 0 < len(victims) < len(m1)
    put(c)
    out, lse = c.run(war)
    assert war.war_device_status() == INVALID
    c.check(out, lse, untouched=victims)


@pytest.mark.parametrize("kv,block", KINDS)
def test_malformed_requests(war, kv, block):
    c = group_case(kv, block)
    (l0, m0), (l1, m1) = members(c)
    bad = [next(i for i in m0 if i != l0), l1]
    parent = c.parent.copy()
    c.parent[bad[0], 3] = 3                                           # a slot that is its own parent
    c.nn[bad[1]] = c.N + 1
    put(c)
    a = c.args(war)
    c.call(war, a)
    torch.cuda.synchronize()
    assert war.war_device_status() == BAD_TREE
    c.nn[bad[1]], c.parent = c.N, parent
    c.check(a[-2], a[-1], untouched=bad)
    c.prefix[bad[1]] = -1
    put(c)
    a[-2].fill_(7.0), a[-1].fill_(7.0)
    c.call(war, a)
    torch.cuda.synchronize()
    assert war.war_device_status() == BAD_TREE
    c.prefix[bad[1]] = c.pt.shape[1] * c.page                         # the tree would lie behind the table
    put(c)
    a[-2].fill_(7.0), a[-1].fill_(7.0)
    c.call(war, a)
    torch.cuda.synchronize()
    assert war.war_device_status() == BAD_PAGE
    c.check(a[-2], a[-1], untouched=[bad[1]])


@pytest.mark.parametrize("kv,block", KINDS)
def test_bad_pages(war, kv, block):
    """A page outside the pool is named and not read; requests that do not use it are right."""
    for bad in (-1, 1 << 30):
        c = group_case(kv, block)
        (l0, m0), (l1, m1) = members(c)
        i = m0[1]
        c.pt[i, int(c.prefix[i]) // c.page] = bad                     # behind what it shares
        put(c)
        out, lse = c.run(war)
        assert war.war_device_status() == BAD_PAGE
        c.check(out, lse, requests=[k for k in range(len(c.prefix)) if k != i])


@pytest.mark.parametrize("kv,block", KINDS)
def test_requests_that_are_not_running(war, kv, block):
    for stop in ("leader", "all but one", "a whole group", "everybody"):
        c = group_case(kv, block)
        (l0, m0), (l1, m1) = members(c)
        idx = {"leader": [l0, l1], "all but one": m0[:-1] + m1[1:], "a whole group": m0, "everybody": list(range(len(c.prefix)))}[stop]
        c.nn[idx] = 0
        c.pt[idx] = 1 << 30                                           # their tables are not looked at
        put(c)
        c.check(*c.run(war))
        assert war.war_device_status() == 0


@pytest.mark.parametrize("kv,block", KINDS)
def test_shared_lengths_inside_a_page(war, kv, block):
    """Rounded down to whole pages; what a request alone in its group says about it does not count."""
    c = group_case(kv, block)
    (l0, m0), (l1, m1) = members(c)
    c.shared[l0], c.shared[l1] = 256 + 15, 16 * 7 + 1
    lonely = next(i for i in range(len(c.prefix)) if i not in m0 + m1)
    c.shared[lonely] = -5
    put(c)
    c.check(*c.run(war))
    c.shared[l0], c.shared[l1], c.shared[lonely] = 15, 0, 1 << 30     # not a page: everybody for itself
    put(c)
    c.check(*c.run(war))
    assert war.war_device_status() == 0


def test_hidden_slots_that_are_no_numbers(war):
    """bf16: keys of slots that a row does not see may be anything; V and the cache in front are finite."""
    c = group_case("bf16", 0)
    hit = {}
    for i in range(len(c.prefix)):
        pos = int(c.prefix[i]) + 3
        c.k[c.pt[i, pos // 16], :, pos % 16] = [float("nan"), float("inf"), float("-inf")][i % 3]
        sees = []
        for j in range(int(c.nn[i])):
            k = j
            while k > 3:
                k = int(c.parent[i, k])
            sees.append(k == 3)
        hit[i] = sees
    c.cache[0].copy_(c.k.to(DEV))
    out, lse = c.run(war)
    for i, sees in hit.items():
        n = int(c.nn[i])
        rows = [j for j in range(n) if not sees[j]]
        K, V = c.values(i)
        K[int(c.prefix[i]) + 3] = 0.0                                 # (unseen by the rows that are compared)
        q = c.q[i].double().numpy()
        want, want_lse = A.verify_attention_request(q, K, V, int(c.prefix[i]), c.parent[i], n, c.scale)
        mass, _ = A.verify_attention_request(q, K, np.abs(V), int(c.prefix[i]), c.parent[i], n, c.scale)
        got = out[i].float().cpu().numpy().astype(np.float64)
        assert (np.abs(got[rows] - want[rows]) <= 2.0 ** -8 * np.abs(want[rows]) + 1.05 * 2.0 ** -8 * mass[rows]).all()
        np.testing.assert_allclose(lse[i].cpu().numpy()[rows], want_lse[rows], atol=1e-4, rtol=1e-5)
        if i % 3 == 0:
            assert all(np.isnan(got[j]).all() for j in range(n) if sees[j])


@pytest.mark.parametrize("kv,block", KINDS)
def test_queries_that_are_no_numbers(war, kv, block):
    """A row of NaN gives NaN and changes no other row."""
    c = group_case(kv, block)
    good, good_lse = c.run(war)
    rows = [(i, int(j), int(h)) for i, j, h in zip([0, 1, 2, 4, 5], [0, 5, 2, 1, 3], [0, 7, 3, 4, 2])]
    for i, j, h in rows:
        c.d_q[i, j, h] = float("nan")
    out, lse = c.run(war)
    hit = torch.zeros(out.shape[:3], dtype=torch.bool, device=DEV)
    for i, j, h in rows:
        hit[i, j, h] = True
    assert torch.isnan(out[hit].float()).all() and torch.isnan(lse[hit]).all()
    assert torch.equal(out[~hit], good[~hit]) and torch.equal(lse[~hit], good_lse[~hit])


@pytest.mark.parametrize("kv,block", KINDS)
def test_same_result_every_time(war, kv, block):
    """Units are drawn as they come, sums are not: bit for bit the same, in another workspace too, with or without the log-sum-exp."""
    c = Case(31, kv, [(2048, [0, 700, 3, 90])] * 6, 9 if block == 8 else 8, 16, 2, 16, block)
    first, first_lse = c.run(war)
    for _ in range(5):
        out, lse = c.run(war)
        assert torch.equal(out, first) and torch.equal(lse, first_lse)
    a = c.args(war)
    c.call(war, (*a[:-1], None))
    torch.cuda.synchronize()
    assert torch.equal(a[-2], first) and (a[-1] == 7.0).all()


@pytest.mark.parametrize("kv,block", KINDS)
def test_agrees_with_every_request_for_itself(war, kv, block):
    """The call without groups on the same cache: both are within the bound of the exact result, so within two of each other."""
    c = Case(41, kv, [(1024, [0, 700, 3, 90]), (320, [64, 65])], 9 if block == 8 else 8, 16, 2, 16, block)
    out, lse = c.run(war)
    quant = kv != "bf16"
    p = (war.attn_quant_params if quant else war.attn_params)(c.d_q, *c.cache, c.ints[0], c.scale)
    ws = (war.new_quant_workspace if quant else war.new_workspace)(p, DEV)
    other, other_lse = torch.full_like(out, 7.0), torch.full_like(lse, 7.0)
    (war.war_verify_attn_quant if quant else war.war_verify_attn)(c.d_q, *c.cache, *c.ints[:4], p, ws, other, other_lse)
    torch.cuda.synchronize()
    c.check(out, lse)
    np.testing.assert_allclose(lse.cpu(), other_lse.cpu(), atol=1e-4, rtol=1e-5)
    assert ((out == 7.0) == (other == 7.0)).all()


@pytest.mark.parametrize("kv,block", KINDS)
def test_replay_with_other_inputs(war, kv, block):
    """A captured call looks at the arrays as they are at every replay: groups, lengths and trees may change."""
    c = group_case(kv, block)
    a = c.args(war)
    c.call(war, a)                                                    # (one-time set-up of the device)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=torch.cuda.Stream()):
        c.call(war, a)
    (l0, m0), (l1, m1) = members(c)

    def check():
        put(c)
        a[-2].fill_(7.0), a[-1].fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        c.check(a[-2], a[-1])
    check()
    c.leader[m0] = m0                                                 # the first group falls apart
    check()
    c.nn[m1[0]] = 0
    c.prefix[m0[0]] -= 100
    c.nn[m0[1]] = 1
    check()
    c.leader[:], c.nn[:] = np.arange(len(c.prefix)), 0
    check()
    assert war.war_device_status() == 0


def test_calls_at_the_same_time(war):
    """Two captured calls and two plain ones on streams of their own, each with its workspace."""
    cases = [group_case("e5m2", 8), Case(51, "e4m3", [(2048, [0, 700, 3, 90])] * 4, 8, 16, 2, 16, 16), group_case("bf16", 0, seed=22),
             Case(52, "bf16", [(2048, [0, 700, 3, 90])] * 4, 8, 16, 2, 16)]
    want = [c.run(war) for c in cases]
    args = [c.args(war) for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    graphs = []
    for c, a, s in zip(cases[:2], args, streams):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            c.call(war, a)
        graphs.append(g)
    torch.cuda.synchronize()
    for _ in range(10):
        for k, s in enumerate(streams):
            with torch.cuda.stream(s):
                args[k][-2].fill_(7.0), args[k][-1].fill_(7.0)
                graphs[k].replay() if k < 2 else cases[k].call(war, args[k])
        torch.cuda.synchronize()
        for k in range(4):
            assert torch.equal(args[k][-2], want[k][0]) and torch.equal(args[k][-1], want[k][1]), k
    assert war.war_device_status() == 0


@pytest.mark.parametrize("kv,block", KINDS)
@pytest.mark.parametrize("groups", [[(64, [1] * 8)] * 512, [(160, list(range(4)) * 1024)], [(0, [33])] * 4096], ids=["512 groups", "one group", "no group"])
def test_the_largest_batch(war, kv, block, groups):
    c = Case(61, kv, groups, 2, 34 if block == 8 else 2, 1, 16, block)
    out, lse = c.run(war)
    c.check(out, lse, requests=list(range(0, 4096, 67)) + [4095])
    assert torch.isfinite(out).all()
    assert war.war_device_status() == 0


@pytest.mark.parametrize("kv,block", KINDS)
def test_one_row_and_many_heads(war, kv, block):
    Case(71, kv, [(0, [0])], 1, 1, 1, 16, block).check(*Case(71, kv, [(0, [0])], 1, 1, 1, 16, block).run(war))           # one token in all
    c = Case(72, kv, [(128, [0, 5, 200])], 1, 512, 1, 16, block)                                                         # 512 query heads a kv head
    c.check(*c.run(war))
    c = Case(73, kv, [(128, [0, 5, 200])], 3, 64, 64, 16, block)                                                         # as many as kv heads
    c.check(*c.run(war))
    assert war.war_device_status() == 0


@pytest.mark.parametrize("kv,block", KINDS)
@pytest.mark.parametrize("token_major", [False, True])
def test_pools_past_32_bits(war, kv, block, token_major):
    """Pages at the far end of a pool of more than 2^32 bytes."""
    c = Case(81, kv, [(256, [0, 130, 17]), (0, [40])], 4, 136 if block == 8 else 16, 8, 16, block, token_major)
    size = 2 if kv == "bf16" else 1
    far = (1 << 32) // (8 * 16 * 128 * size) + 100
    small = c.cache
    total = small[0].shape[0]
    shape = (far + total, 16, 8, 128) if token_major else (far + total, 8, 16, 128)
    big = []
    for x in small[:2]:
        y = torch.empty(shape, dtype=torch.uint8 if size == 1 else torch.bfloat16, device=DEV)
        y = y.permute(0, 2, 1, 3) if token_major else y
        y[far:] = x.view(torch.uint8) if size == 1 else x
        big.append(y.view(x.dtype))
    for x in small[2:]:
        s = torch.empty((far + total, *x.shape[1:]), device=DEV)
        s[far:] = x
        big.append(s)
    assert big[0].numel() * size > 1 << 32
    at = c.pt.copy()
    c.cache, c.ints[0] = tuple(big), torch.from_numpy(np.where(at < total, at + far, at).astype(np.int32)).to(DEV)
    out, lse = c.run(war)
    c.check(out, lse)
    assert war.war_device_status() == 0


def test_other_device(war, monkeypatch):
    """Tensors of another device than the current one are refused before anything is launched."""
    from tests import test_pages_cpu_binding as B
    calls = {**B.calls(war), "war_verify_attn_shared": B.attention_args(war, False), "war_verify_attn_shared_quant": B.attention_args(war, True)}
    for name, args in calls.items():
        move = lambda v: v.to(DEV) if isinstance(v, torch.Tensor) else war.Pages(*(x.to(DEV) for x in v)) if isinstance(v, war.Pages) else v
        args = {k: move(v) for k, v in args.items()}
        with monkeypatch.context() as m:
            m.setattr(torch.cuda, "current_device", lambda: 1)
            with pytest.raises(ValueError, match="current device, cuda:1"):
                getattr(war, name)(**args)
        getattr(war, name)(**args)                                    # (no slots, nothing to copy, nobody done)
        torch.cuda.synchronize()
        assert war.war_device_status() == 0, name
