"""What the 8-bit cache, the rotary store and the target choice refuse, and the parts that run on the host."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import cache_oracle as O
from oracle import target_oracle as T


@pytest.fixture(scope="module")
def war():
    from paper_2607_17299_b200.build import build
    build()
    from paper_2607_17299_b200 import binding
    return binding


@pytest.mark.parametrize("kv,dt", [("e4m3", torch.float8_e4m3fn), ("e5m2", torch.float8_e5m2)])
def test_checker_codes_are_the_types(kv, dt):
    np.testing.assert_array_equal(torch.arange(256, dtype=torch.uint8).view(dt).double().numpy(), O.values(kv))
    rng = np.random.default_rng(0)
    x = (rng.standard_normal(20000) * np.exp(4 * rng.standard_normal(20000))).astype(np.float32)
    x = np.concatenate([x, O.values(kv)[np.isfinite(O.values(kv))]]).astype(np.float32).clip(-O.MOST[kv], O.MOST[kv])
    np.testing.assert_array_equal(torch.from_numpy(x).to(dt).view(torch.uint8).numpy(), O.encode(x, kv))
    for a in [O.MOST[kv], O.MOST[kv] * 2.0 ** -7, 1.0, 3e38, 1e-30, 1.1754944e-38]:
        s = O.scale_for(a, kv)
        assert a <= O.MOST[kv] * s and (s == O.SMALLEST_SCALE or a > O.MOST[kv] * s / 2)


def test_checker_commit_keeps_values_under_powers_of_two():
    rng = np.random.default_rng(1)
    codes = O.encode(rng.standard_normal((3, 2, 16, 128)) * 100, "e4m3")
    scale = 2.0 ** rng.integers(-3, 3, (3, 2, 2)).astype(np.float32)
    before = O.decode(codes, "e4m3") * scale.repeat(8, -1)[..., None]
    table = [2, 0, 1]
    O.commit_rows(codes, scale, "e4m3", 8, table, 13, [2, 9, 20])
    after = O.decode(codes, "e4m3") * scale.repeat(8, -1)[..., None]
    at = lambda v, x: v[table[x // 16], :, x % 16]
    for src, dst in ((13, 13), (15, 14), (22, 15), (33, 16)):
        assert np.abs(at(after, dst) - at(before, src)).max() <= 2.0 ** -10 * scale.max()       # subnormal codes may round
    assert (at(after, 0) == at(before, 0)).all()


def test_checker_choice():
    assert T.choose(np.array([1, np.nan, 3, 3], np.float32)) == 2
    assert T.choose(np.array([-np.inf, np.nan], np.float32)) == -1
    x = T.process_row(np.array([2, -2, 1, 1], np.float32), [0, 1, 0], 1, [3], 2.0, 0.5, 0.25, [(2, 1.0), (2, 7.0)], np.array([1, 1, 1, 0], bool))
    np.testing.assert_array_equal(x, np.array([1 - 0.25 - 0.5, -4 - 0.25 - 0.5, 8, -np.inf], np.float32))


def _freq(war, **kw):
    f, factor = war.war_rope_frequencies(**kw)
    return f.double().numpy(), factor


def test_frequencies(war):
    n = 64
    i = np.arange(n)
    plain = 10000.0 ** (-2.0 * i / 128)
    close = lambda a, b: np.testing.assert_allclose(a, b, rtol=2.0 ** -23)
    f, factor = _freq(war, rot_dim=128, base=10000.0)
    close(f, plain)
    assert factor == 1.0
    close(_freq(war, rot_dim=128, base=10000.0, kind="linear", scale=4.0)[0], plain / 4)
    f, _ = _freq(war, rot_dim=128, base=10000.0, kind="base", scale=8.0)
    close(f, (10000.0 * 8.0 ** (128 / 126)) ** (-2.0 * i / 128))
    np.testing.assert_allclose(f[-1], plain[-1] / 8, rtol=1e-6)                 # the slowest wave stretched by the scale
    f, factor = _freq(war, rot_dim=128, base=10000.0, kind="ramp", scale=4.0, original_length=4096.0)
    turns = 4096 * plain / (2 * np.pi)
    close(f[turns > 40], plain[turns > 40])
    close(f[turns < 0.8], plain[turns < 0.8] / 4)
    assert (np.diff(plain / f) > -1e-6).all() and abs(factor - (0.1 * np.log(4) + 1)) < 1e-6
    f, factor = _freq(war, rot_dim=128, base=500000.0, kind="bands", scale=8.0, original_length=8192.0, fast=4.0, slow=1.0)
    plain = 500000.0 ** (-2.0 * i / 128)
    turns = 8192 * plain / (2 * np.pi)
    share = np.clip((turns - 1) / 3, 0, 1)
    close(f, plain / 8 * (1 - share) + plain * share)
    assert factor == 1.0 and len(_freq(war, rot_dim=0, base=2.0)[0]) == 0


@pytest.mark.parametrize("kw", [dict(rot_dim=7, base=1e4), dict(rot_dim=130, base=1e4), dict(rot_dim=64, base=1.0), dict(rot_dim=64, base=float("nan")),
                                dict(rot_dim=64, base=1e4, kind="linear", scale=0.5), dict(rot_dim=64, base=1e4, kind="ramp", scale=2.0),
                                dict(rot_dim=64, base=1e4, kind="bands", scale=2.0, original_length=10.0, fast=1.0, slow=2.0)])
def test_frequency_refusals(war, kw):
    with pytest.raises(war.WarError) as e:
        war.war_rope_frequencies(**kw)
    assert e.value.code == 1


def _store(war):
    p = war.RopeStoreParams()
    p.B, p.N, p.Hq, p.Hkv, p.D, p.page_size, p.max_pages_per_req, p.kv_type, p.scale_block = 2, 8, 8, 2, 128, 16, 10, 1, 16
    p.rot_dim, p.interleaved, p.factor, p.num_pages = 128, 0, 1.0, 40
    for a, s in ((p.q_strides, (8192, 1024, 128, 1)), (p.k_strides, (2048, 256, 128, 1)), (p.v_strides, (2048, 256, 128, 1)),
                 (p.kpool_strides, (4096, 2048, 128, 1)), (p.vpool_strides, (4096, 2048, 128, 1))):
        for i in range(4):
            a[i] = s[i]
    return p


def _call_store(war, p, ptr=1 << 20, **null):
    names = ["q", "k", "v", "f", "pt", "pl", "n", "par", "kp", "vp", "ks", "vs", "qo"]
    a = [None if null.get(x) is None and x in null else null.get(x, ptr) for x in names]
    return war._lib.war_rope_store(*a[:8], C.byref(p) if p is not None else None, *a[8:], None)


def test_store_refusals(war):
    def code(ptr=1 << 20, _null=None, **change):
        p = _store(war)
        for k, v in change.items():
            if isinstance(v, tuple):
                getattr(p, k)[v[0]] = v[1]
            else:
                setattr(p, k, v)
        return _call_store(war, p, ptr, **(_null or {}))
    assert _call_store(war, None) == 1
    for change in (dict(B=-1), dict(N=0), dict(N=65), dict(Hkv=0), dict(rot_dim=3), dict(rot_dim=130), dict(kv_type=3), dict(interleaved=2),
                   dict(factor=float("nan")), dict(factor=float("inf")), dict(num_pages=0), dict(page_size=0), dict(max_pages_per_req=0)):
        assert code(**change) == 1, change
    for change in (dict(D=64), dict(scale_block=24), dict(scale_block=32), dict(scale_block=0), dict(max_pages_per_req=1 << 27), dict(q_strides=(1, 1020)),
                   dict(k_strides=(3, 2)), dict(kpool_strides=(2, 120)), dict(vpool_strides=(0, -4096))):
        assert code(**change) == 6, change
    assert code(ptr=(1 << 20) + 8) == 6                                          # rows off their 16-byte boundaries
    for x in ("q", "k", "v", "f", "pt", "pl", "n", "par", "kp", "vp", "ks", "vs", "qo"):
        assert code(_null={x: None}) == 1, x
    assert code(B=0, _null={"q": None}) == 0


def test_attention_refusals(war):
    def params(**change):
        p = war.AttnQuantParams()
        a = p.attn
        a.B, a.N, a.Hq, a.Hkv, a.D, a.page_size, a.max_pages_per_req, a.kernel, a.num_pages, a.scale = 8, 16, 32, 8, 128, 16, 300, 0, 4000, 0.088
        for i, s in enumerate((16384, 2048, 128, 1)):
            a.k_strides[i] = a.v_strides[i] = s
        p.kv_type, p.scale_block = 1, 16
        for k, v in change.items():
            o = a if hasattr(a, k) else p
            if isinstance(v, tuple):
                getattr(o, k)[v[0]] = v[1]
            else:
                setattr(o, k, v)
        return p
    size = lambda p: war.war_verify_attn_quant_workspace_bytes(p)
    n = size(params())
    assert n > 0 and n % 256 == 0
    def code(p, ptr=1 << 20, null=()):
        a = [None if i in null else ptr for i in range(9)]
        return war._lib.war_verify_attn_quant(*a, C.byref(p), None if 9 in null else ptr, None if 10 in null else ptr, None, None)
    for change in (dict(B=-1), dict(N=65), dict(N=0), dict(Hq=31), dict(kernel=3), dict(scale=0.0), dict(scale=float("nan")), dict(kv_type=0), dict(kv_type=3),
                   dict(num_pages=-1)):
        assert size(params(**change)) == 0 and code(params(**change)) == 1, change
    for change in (dict(D=64), dict(page_size=24), dict(page_size=256), dict(scale_block=32), dict(scale_block=4), dict(Hkv=1, N=17), dict(B=5000),
                   dict(max_pages_per_req=1 << 27), dict(k_strides=(2, 136)), dict(v_strides=(3, 2))):
        assert size(params(**change)) == 0 and code(params(**change)) == 6, change
    for i in range(11):
        assert code(params(), null=(i,)) == 1, i
    assert code(params(), ptr=(1 << 20) + 8) == 1 and code(params(num_pages=0)) == 1
    assert code(params(B=0), null=tuple(range(11))) == 0


def test_target_refusals(war):
    def code(null=(), inputs=(), ptr=1 << 20, **change):
        p = war.TargetParams()
        p.B, p.N, p.V, p.dtype = 2, 4, 1000, 0
        p.logits_strides[0], p.logits_strides[1] = 4000, 1000
        for k, v in change.items():
            if isinstance(v, tuple):
                getattr(p, k)[v[0]] = v[1]
            else:
                setattr(p, k, v)
        t = war.TargetInputs()
        for k in inputs:
            setattr(t, k, ptr)
        a = [None if i in null else ptr for i in range(4)]
        return war._lib.war_target(*a, C.byref(t), C.byref(p), None if 4 in null else ptr, None, None)
    for change in (dict(B=-1), dict(N=0), dict(N=65), dict(V=0), dict(dtype=2), dict(logits_strides=(0, -1)), dict(mask_strides=(1, -1))):
        assert code(**change) == 1, change
    assert code(V=262145) == 6 and code(B=65536) == 6
    assert code(null=(0,)) == 1 and code(null=(1,)) == 1 and code(null=(4,)) == 1
    assert code(ptr=(1 << 20) + 1) == 1
    assert code(inputs=("d_repetition",)) == 1                                   # penalties need the contexts
    assert code(inputs=("d_presence", "d_ctx", "d_ctx_off"), null=(2,)) == 1     # ids and parent come together
    assert code(inputs=("d_bias_off", "d_bias_ids")) == 1
    assert code(B=0, null=(0, 1, 2, 3, 4)) == 0


def test_commit_refusals(war):
    def code(null=(), ptr=1 << 20, **change):
        q = war.CommitQuantParams()
        p = q.commit
        p.B, p.N, p.P, p.Hkv, p.D, p.page_size, p.max_pages_per_req, p.num_pages = 2, 8, 32, 2, 128, 16, 10, 40
        for i, s in enumerate((4096, 2048, 128, 1)):
            p.k_strides[i] = p.v_strides[i] = s
        q.kv_type, q.scale_block = 2, 8
        for k, v in change.items():
            o = p if hasattr(p, k) else q
            if isinstance(v, tuple):
                getattr(o, k)[v[0]] = v[1]
            else:
                setattr(o, k, v)
        a = [None if i in null else ptr for i in range(12)]
        return war._lib.war_commit_quant(*a[:9], C.byref(q), *a[9:], None)
    for change in (dict(B=-1), dict(N=65), dict(P=33), dict(P=0), dict(Hkv=0), dict(kv_type=0), dict(num_pages=0)):
        assert code(**change) == 1, change
    for change in (dict(D=64), dict(scale_block=32), dict(scale_block=7), dict(k_strides=(2, 120)), dict(max_pages_per_req=1 << 27)):
        assert code(**change) == 6, change
    for i in range(12):
        assert code(null=(i,)) == 1, i
    assert code(ptr=(1 << 20) + 4) == 6
    assert code(B=0, null=tuple(range(12))) == 0


def test_binding_refuses_what_does_not_belong_together(war):
    pool = torch.zeros((4, 2, 16, 128), dtype=torch.uint8).view(torch.float8_e4m3fn)
    scale = torch.ones((4, 2, 1))
    assert war._pool_args(pool, pool, scale, scale) == (1, 16)
    assert war._pool_args(pool.view(torch.uint8).view(torch.float8_e5m2), pool.view(torch.float8_e5m2), torch.ones((4, 2, 2)), torch.ones((4, 2, 2))) == (2, 8)
    for bad in ((pool, pool.view(torch.float8_e5m2), scale, scale), (pool, pool, None, scale), (pool, pool, scale, torch.ones((4, 2, 2))),
                (pool, pool, torch.ones((4, 1, 1)), scale), (pool, pool, torch.ones((4, 2, 3)), torch.ones((4, 2, 3))),
                (pool.to(torch.bfloat16), pool.to(torch.bfloat16), scale, None), (pool.to(torch.float16), pool.to(torch.float16), scale, scale)):
        with pytest.raises(ValueError):
            war._pool_args(*bad)
