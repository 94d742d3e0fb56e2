"""What the calls for pages and shared prefixes refuse before anything is launched, in the binding and in the library."""
import ctypes as C

import pytest
import torch

i32 = dict(dtype=torch.int32)
one = lambda *shape: torch.zeros(shape, **i32)
OK, INVALID, UNSUPPORTED = 0, 1, 6
SOME = C.c_void_p(256)                                          # an address that is never used


@pytest.fixture(scope="module")
def war():
    from paper_2607_17299_b200.build import build
    build()
    from paper_2607_17299_b200 import binding
    return binding


def pages_args(war, num_pages=40, B=3, width=5):
    return war.new_pages(num_pages, B, width, "cpu")


@pytest.mark.parametrize("num_pages", [1, 31, 32, 33, 100])
def test_books_of_an_empty_pool(war, num_pages):
    p = war.new_pages(num_pages, 3, 5, "cpu")
    words = [int(x) & 0xffffffff for x in p.free.tolist()]
    assert sum(w << (32 * i) for i, w in enumerate(words)) == (1 << num_pages) - 1
    assert p.refs.shape == (num_pages,) and not p.refs.any() and (p.page_table == -1).all() and not p.held.any()


@pytest.mark.parametrize("field,shape", [("refs", (65,)), ("refs", (40, 1)), ("free", (1,)), ("free", (3,)), ("page_table", (15,)),
                                         ("page_table", (2, 5)), ("held", (4,)), ("held", (3, 1))])
def test_books_that_do_not_belong_together(war, field, shape):
    p = pages_args(war)._replace(**{field: one(*shape)})
    with pytest.raises(ValueError, match="refs .num_pages.|expected shape"):
        war.war_pages_free(p, one(3))


def calls(war):
    p = pages_args(war)
    return {
        "war_pages_grow": dict(pages=p, N=4, page_size=16, d_prefix_len=one(3), d_tail_len=one(3), d_granted=one(3)),
        "war_pages_fork": dict(pages=p, d_src=one(3), page_size=16, d_prefix_len=one(3), d_tail=one(3, 8), d_tail_len=one(3),
                               d_copies=one(3, 3), d_n_copies=one(1), d_ok=one(1)),
        "war_pages_free": dict(pages=p, d_done=one(3), d_tail_len=one(3)),
        "war_pages_compact": dict(pages=p, page_size=16, d_workspace=war.new_compact_workspace(p), d_copies=one(7, 3), d_n_copies=one(1),
                                  d_top=one(1)),
        "war_pages_copy": dict(d_copies=one(7, 3), d_n_copies=one(1), k_pool=torch.zeros((12, 2, 16, 128), dtype=torch.bfloat16),
                               v_pool=torch.zeros((12, 2, 16, 128), dtype=torch.bfloat16)),
        "war_prefix_groups": dict(d_page_table=one(3, 5), d_prefix_len=one(3), d_tail_len=one(3), page_size=16, min_shared=32,
                                  d_leader=one(3), d_shared_len=one(3)),
    }


@pytest.mark.parametrize("name", ["war_pages_grow", "war_pages_fork", "war_pages_free", "war_pages_compact", "war_pages_copy", "war_prefix_groups"])
def test_nothing_but_the_device_is_wrong(war, name):
    with pytest.raises(ValueError, match="CUDA"):
        getattr(war, name)(**calls(war)[name])


@pytest.mark.parametrize("name,arg,shape", [
    ("war_pages_grow", "d_prefix_len", (2,)), ("war_pages_grow", "d_tail_len", (4,)), ("war_pages_grow", "d_granted", (3, 1)),
    ("war_pages_fork", "d_src", (2,)), ("war_pages_fork", "d_prefix_len", (4,)), ("war_pages_fork", "d_tail_len", (2,)),
    ("war_pages_fork", "d_tail", (2, 8)), ("war_pages_fork", "d_tail", (24,)), ("war_pages_fork", "d_copies", (2, 3)),
    ("war_pages_fork", "d_copies", (3, 2)), ("war_pages_fork", "d_copies", (9,)), ("war_pages_fork", "d_n_copies", (2,)), ("war_pages_fork", "d_ok", (0,)),
    ("war_pages_free", "d_done", (2,)), ("war_pages_free", "d_tail_len", (1,)),
    ("war_pages_compact", "d_copies", (7, 2)), ("war_pages_compact", "d_n_copies", (2,)), ("war_pages_compact", "d_top", (2,)),
    ("war_pages_compact", "d_workspace", (10,)), ("war_pages_copy", "d_copies", (21,)),
    ("war_prefix_groups", "d_page_table", (15,)), ("war_prefix_groups", "d_prefix_len", (2,)), ("war_prefix_groups", "d_tail_len", (4,)),
    ("war_prefix_groups", "d_leader", (2,)), ("war_prefix_groups", "d_shared_len", (5,))])
def test_shapes(war, name, arg, shape):
    with pytest.raises(ValueError, match="expected shape|must be|one number|smaller than"):
        getattr(war, name)(**{**calls(war)[name], arg: one(*shape)})


def test_copy_pools_that_do_not_belong_together(war):
    a = calls(war)["war_pages_copy"]
    codes = torch.zeros((12, 2, 16, 128), dtype=torch.uint8).view(torch.float8_e4m3fn)
    scale = torch.ones((12, 2, 1))
    for over in (dict(v_pool=a["v_pool"][:11]), dict(v_pool=codes), dict(k_scale=scale, v_scale=scale), dict(k_pool=codes, v_pool=codes),
                 dict(k_pool=codes, v_pool=codes, k_scale=scale, v_scale=scale[:11]), dict(k_pool=a["k_pool"].float(), v_pool=a["v_pool"].float())):
        with pytest.raises(ValueError):
            war.war_pages_copy(**{**a, **over})


def attention_args(war, quant):
    B, N, Hq, Hkv = 3, 5, 8, 2
    a = dict(d_q=torch.zeros((B, N, Hq, 128), dtype=torch.bfloat16))
    if quant:
        pool = lambda: torch.zeros((12, Hkv, 16, 128), dtype=torch.uint8).view(torch.float8_e4m3fn)
        a.update(k_pool=pool(), v_pool=pool(), k_scale=torch.ones((12, Hkv, 1)), v_scale=torch.ones((12, Hkv, 1)))
        cache = [a[k] for k in ("k_pool", "v_pool", "k_scale", "v_scale")]
    else:
        a.update(d_kpool=torch.zeros((12, Hkv, 16, 128), dtype=torch.bfloat16), d_vpool=torch.zeros((12, Hkv, 16, 128), dtype=torch.bfloat16))
        cache = [a["d_kpool"], a["d_vpool"]]
    a.update(d_page_table=one(B, 4), d_prefix_len=one(B), d_num_nodes=one(B), d_parent=one(B, N), d_leader=one(B), d_shared_len=one(B))
    a["params"] = (war.attn_quant_params if quant else war.attn_params)(a["d_q"], *cache, a["d_page_table"], 0.1)
    a["d_workspace"] = (war.new_shared_quant_workspace if quant else war.new_shared_workspace)(a["params"], "cpu")
    a["d_out"], a["d_lse"] = torch.zeros_like(a["d_q"]), torch.zeros((B, N, Hq))
    return a


def attention(war, quant):
    return war.war_verify_attn_shared_quant if quant else war.war_verify_attn_shared


@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("name,shape", [("d_page_table", (2, 4)), ("d_page_table", (12,)), ("d_prefix_len", (2,)), ("d_num_nodes", (4,)),
                                        ("d_parent", (3, 4)), ("d_parent", (15,)), ("d_leader", (2,)), ("d_leader", (3, 1)), ("d_shared_len", (4,)),
                                        ("d_out", (3, 5, 4, 128)), ("d_lse", (3, 5)), ("d_q", (3, 40, 128))])
def test_attention_shapes(war, quant, name, shape):
    a = attention_args(war, quant)
    with pytest.raises(ValueError, match="expected shape|d_q must be"):
        attention(war, quant)(**{**a, name: torch.zeros(shape, dtype=a[name].dtype)})


@pytest.mark.parametrize("quant", [False, True])
def test_attention_of_other_tensors(war, quant):
    a, call = attention_args(war, quant), attention(war, quant)
    with pytest.raises(ValueError, match="CUDA"):                # nothing but the device is wrong
        call(**a)
    with pytest.raises(ValueError, match="CUDA"):
        call(**{**a, "d_lse": None})
    with pytest.raises(ValueError, match="params do not describe"):
        call(**{**a, "d_page_table": one(3, 3)})
    with pytest.raises(ValueError, match="workspace is smaller"):
        call(**{**a, "d_workspace": a["d_workspace"][:-1]})
    if quant:
        with pytest.raises(ValueError, match="has scales"):
            call(**{**a, "k_scale": None})
    else:
        with pytest.raises(ValueError, match="must be bf16"):
            call(**{**a, "d_kpool": a["d_kpool"].float()})


def attn(war, quant=False, **over):
    q = war.AttnQuantParams() if quant else war.AttnParams()
    p = q.attn if quant else q
    p.B, p.N, p.Hq, p.Hkv, p.D, p.page_size, p.max_pages_per_req, p.kernel, p.num_pages, p.scale = 4, 8, 8, 2, 128, 16, 9, 0, 50, 0.1
    over = dict(over)
    for k, v in over.items():
        if k in ("kv_type", "scale_block"):
            continue
        setattr(p, k, v)
    for i, s in enumerate((p.Hkv * p.page_size * 128, p.page_size * 128, 128, 1)):
        p.k_strides[i] = p.v_strides[i] = s
    if quant:
        q.kv_type, q.scale_block = over.get("kv_type", 1), over.get("scale_block", 16)
    return q


@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("over,status", [(dict(B=-1), INVALID), (dict(N=0), INVALID), (dict(N=65), INVALID), (dict(Hq=9), INVALID), (dict(Hkv=0), INVALID),
                                         (dict(kernel=1), INVALID), (dict(scale=0.0), INVALID), (dict(scale=float("nan")), INVALID),
                                         (dict(max_pages_per_req=-1), INVALID), (dict(num_pages=-1), INVALID), (dict(D=64), UNSUPPORTED),
                                         (dict(page_size=24), UNSUPPORTED), (dict(Hq=160), UNSUPPORTED), (dict(B=4097), UNSUPPORTED),
                                         (dict(B=4096, N=64, Hq=2048, Hkv=2048), UNSUPPORTED), (dict(Hq=65536, Hkv=65536), UNSUPPORTED),
                                         (dict(max_pages_per_req=1 << 26), UNSUPPORTED)])
def test_attention_limits(war, quant, over, status):
    name = "war_verify_attn_shared_quant" if quant else "war_verify_attn_shared"
    size = getattr(war, name + "_workspace_bytes")
    assert size(attn(war, quant)) > 0 and size(attn(war, quant)) % 256 == 0
    q = attn(war, quant, **over)
    assert size(q) == 0
    n = 11 if quant else 9
    assert getattr(war._lib, name)(*[SOME] * n, C.byref(q), SOME, SOME, None, None) == status
    assert getattr(war._lib, name)(*[SOME] * n, None, SOME, SOME, None, None) == INVALID


@pytest.mark.parametrize("quant", [False, True])
def test_attention_addresses(war, quant):
    fn = getattr(war._lib, "war_verify_attn_shared_quant" if quant else "war_verify_attn_shared")
    n, q = 11 if quant else 9, attn(war, quant)
    call = lambda first, ws=SOME, out=SOME: fn(*first, C.byref(q), ws, out, None, None)
    for i in range(n):
        assert call([None if k == i else SOME for k in range(n)]) == INVALID
    assert call([SOME] * n, ws=None) == INVALID and call([SOME] * n, out=None) == INVALID
    assert call([SOME] * n, ws=C.c_void_p(128)) == INVALID           # 256-byte aligned
    assert call([SOME] * n, out=C.c_void_p(8)) == INVALID
    assert call([C.c_void_p(8)] + [SOME] * (n - 1)) == INVALID
    assert call([SOME, C.c_void_p(8)] + [SOME] * (n - 2)) == INVALID
    q = attn(war, quant, B=0)
    assert call([None] * n, None, None) == OK                         # nothing to do


def test_attention_over_an_8_bit_cache_limits(war):
    for over, status in ((dict(kv_type=0), INVALID), (dict(kv_type=3), INVALID), (dict(scale_block=4), UNSUPPORTED), (dict(scale_block=32), UNSUPPORTED)):
        q = attn(war, True, **over)
        assert war.war_verify_attn_shared_quant_workspace_bytes(q) == 0
        assert war._lib.war_verify_attn_shared_quant(*[SOME] * 11, C.byref(q), SOME, SOME, None, None) == status


def books(war, **over):
    p = war.PagesBooks(256, 256, 256, 256, 4, 16, 9, 0, 50)
    for k, v in over.items():
        setattr(p, k, v)
    return p


PAGES = {"war_pages_grow": lambda p: (p, 8, SOME, SOME, SOME, None), "war_pages_fork": lambda p: (p, SOME, 8, SOME, SOME, SOME, SOME, SOME, SOME, None),
         "war_pages_free": lambda p: (p, SOME, SOME, None), "war_pages_compact": lambda p: (p, SOME, 8, SOME, SOME, SOME, None)}


@pytest.mark.parametrize("name", list(PAGES))
@pytest.mark.parametrize("over,status", [(dict(B=-1), INVALID), (dict(page_size=0), INVALID), (dict(max_pages_per_req=0), INVALID), (dict(num_pages=0), INVALID),
                                         (dict(B=4097), UNSUPPORTED), (dict(num_pages=(1 << 30) + 1), UNSUPPORTED), (dict(max_pages_per_req=1 << 29), UNSUPPORTED), (dict(d_refs=None), INVALID),
                                         (dict(d_free=None), INVALID), (dict(d_page_table=None), INVALID), (dict(d_held=None), INVALID)])
def test_books_limits(war, name, over, status):
    assert getattr(war._lib, name)(*PAGES[name](C.byref(books(war, **over)))) == status
    assert getattr(war._lib, name)(*PAGES[name](None)) == INVALID


def test_pages_arguments(war):
    p, lib = C.byref(books(war)), war._lib
    assert lib.war_pages_grow(p, -1, SOME, SOME, SOME, None) == INVALID
    assert lib.war_pages_grow(p, 1 << 30, SOME, SOME, SOME, None) == INVALID
    assert lib.war_pages_grow(p, 8, None, SOME, SOME, None) == INVALID
    assert lib.war_pages_grow(p, 8, SOME, SOME, None, None) == INVALID
    for i in (1, 3, 4, 5, 6, 7, 8):
        assert lib.war_pages_fork(*[None if k == i else x for k, x in enumerate(PAGES["war_pages_fork"](p))]) == INVALID
    for P in (0, -1, 1 << 20):
        assert lib.war_pages_fork(p, SOME, P, SOME, SOME, SOME, SOME, SOME, SOME, None) == INVALID
    assert lib.war_pages_free(p, None, SOME, None) == INVALID
    for i in (1, 3, 4, 5):
        assert lib.war_pages_compact(*[None if k == i else x for k, x in enumerate(PAGES["war_pages_compact"](p))]) == INVALID
    assert lib.war_pages_compact(p, C.c_void_p(258), 8, SOME, SOME, SOME, None) == INVALID
    assert lib.war_pages_compact(p, SOME, -1, SOME, SOME, SOME, None) == INVALID
    empty = C.byref(books(war, B=0))
    assert lib.war_pages_grow(empty, 8, SOME, SOME, SOME, None) == OK and lib.war_pages_free(empty, SOME, SOME, None) == OK
    assert lib.war_pages_compact_workspace_bytes(0) == 0 and lib.war_pages_compact_workspace_bytes((1 << 30) + 1) == 0
    assert lib.war_pages_compact_workspace_bytes(1 << 30) > 0


def test_groups_arguments(war):
    call = lambda B=4, page=16, width=9, least=16, table=SOME, prefix=SOME, leader=SOME, shared=SOME: war._lib.war_prefix_groups(
        table, prefix, None, B, page, width, least, leader, shared, None)
    for over in (dict(B=-1), dict(page=0), dict(width=0), dict(least=0), dict(table=None), dict(prefix=None), dict(leader=None), dict(shared=None)):
        assert call(**over) == INVALID
    assert call(B=4097) == UNSUPPORTED and call(B=0) == OK


def copy_params(war, kv=0, **over):
    q = war.PagesCopyParams(2, 128, 16, kv, 16, 0, 50)
    q.kpool_strides[:] = q.vpool_strides[:] = (4096, 2048, 128, 1)
    for k, v in over.items():
        if k == "strides":
            q.vpool_strides[:] = v
        else:
            setattr(q, k, v)
    return q


def test_copy_arguments(war):
    def call(q, n=8, copies=SOME, count=SOME, k=SOME, v=SOME, ks=SOME, vs=SOME):
        return war._lib.war_pages_copy(copies, count, n, k, v, ks, vs, None if q is None else C.byref(q), None)
    for over, status in ((dict(Hkv=0), INVALID), (dict(page_size=0), INVALID), (dict(num_pages=0), INVALID), (dict(kv_type=3), INVALID), (dict(D=64), UNSUPPORTED),
                         (dict(num_pages=(1 << 30) + 1), UNSUPPORTED), (dict(strides=(4096, 2048, 127, 1)), UNSUPPORTED),
                         (dict(strides=(4096, 2048, 128, 2)), UNSUPPORTED)):
        assert call(copy_params(war, **over)) == status, over
    for kv in (0, 1, 2):
        q = copy_params(war, kv)
        for arg in ("copies", "count", "k", "v") + (("ks", "vs") if kv else ()):
            assert call(q, **{arg: None}) == INVALID
        assert call(q, k=C.c_void_p(8)) == INVALID and call(q, n=-1) == INVALID and call(q, n=0, copies=None) == OK
    assert call(None) == INVALID
    for block, page in ((4, 16), (32, 16), (8, 1024)):
        assert call(copy_params(war, 1, scale_block=block, page_size=page)) == UNSUPPORTED
