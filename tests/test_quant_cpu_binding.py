"""What the binding of the cache and logits calls refuses before anything is launched: arguments that do not belong together."""
import pytest
import torch

i32, f32 = dict(dtype=torch.int32), dict(dtype=torch.float32)


@pytest.fixture(scope="module")
def war():
    from paper_2607_17299_b200.build import build
    build()
    from paper_2607_17299_b200 import binding
    return binding


def target_args(**over):
    B, N, V = 2, 4, 100
    a = dict(d_logits=torch.zeros((B, N, V)), d_num_nodes=torch.zeros(B, **i32), d_ids=torch.zeros((B, N), **i32),
             d_parent=torch.zeros((B, N), **i32), d_target=torch.zeros((B, N), **i32), d_ctx=torch.zeros(7, **i32),
             d_ctx_off=torch.tensor([0, 3, 7]), d_repetition=torch.ones(B), d_bias_off=torch.tensor([0, 1, 2]),
             d_bias_ids=torch.zeros(2, **i32), d_bias_val=torch.zeros(2))
    return {**a, **over}


@pytest.mark.parametrize("penalty", ["d_repetition", "d_presence", "d_frequency"])
def test_penalties_need_the_contexts(war, penalty):
    none = dict(d_ctx=None, d_repetition=None)
    with pytest.raises(ValueError, match="penalties need d_ctx"):
        war.war_target(**target_args(**{**none, penalty: torch.ones(2)}))
    with pytest.raises(ValueError, match="CUDA"):               # without penalties they may be left out
        war.war_target(**target_args(**none))


@pytest.mark.parametrize("length", [1, 3])
def test_bias_lists_are_of_one_length(war, length):
    with pytest.raises(ValueError, match="one length"):
        war.war_target(**target_args(d_bias_val=torch.zeros(length)))
    with pytest.raises(ValueError, match="CUDA"):
        war.war_target(**target_args())


def commit_args(**over):
    B, N, P = 3, 5, 8
    pool = lambda: torch.zeros((12, 2, 16, 128), dtype=torch.uint8).view(torch.float8_e4m3fn)
    one = lambda *shape: torch.zeros(shape, **i32)
    a = dict(d_ids=one(B, N), d_accept_len=one(B), d_accept_path=one(B, N), d_bonus=one(B), k_pool=pool(), v_pool=pool(),
             k_scale=torch.ones((12, 2, 1)), v_scale=torch.ones((12, 2, 1)), page_table=one(B, 4), d_prefix_len=one(B), d_tail=one(B, P),
             d_tail_len=one(B))
    return {**a, **over}


@pytest.mark.parametrize("name,shape", [("d_accept_len", (2,)), ("d_accept_len", (3, 1)), ("d_accept_path", (3, 4)), ("d_accept_path", (2, 5)),
                                        ("d_accept_path", (15,)), ("d_bonus", (4,)), ("d_prefix_len", (2,)), ("d_tail_len", (2,)),
                                        ("d_tail", (2, 8)), ("d_tail", (8,)), ("page_table", (2, 4)), ("page_table", (12,)), ("d_ids", (15,))])
def test_commit_shapes(war, name, shape):
    with pytest.raises(ValueError, match="expected shape|d_ids must be"):
        war.war_commit_quant(**commit_args(**{name: torch.zeros(shape, **i32)}))


def test_commit_shapes_that_belong_together(war):
    with pytest.raises(ValueError, match="CUDA"):                # nothing but the device is wrong
        war.war_commit_quant(**commit_args())


def attention_args(war, **over):
    B, N, Hq, Hkv = 3, 5, 8, 2
    pool = lambda: torch.zeros((12, Hkv, 16, 128), dtype=torch.uint8).view(torch.float8_e4m3fn)
    one = lambda *shape: torch.zeros(shape, **i32)
    a = dict(d_q=torch.zeros((B, N, Hq, 128), dtype=torch.bfloat16), k_pool=pool(), v_pool=pool(), k_scale=torch.ones((12, Hkv, 1)),
             v_scale=torch.ones((12, Hkv, 1)), d_page_table=one(B, 4), d_prefix_len=one(B), d_num_nodes=one(B), d_parent=one(B, N))
    a["params"] = war.attn_quant_params(*(a[k] for k in ("d_q", "k_pool", "v_pool", "k_scale", "v_scale", "d_page_table")), 0.1)
    a["d_workspace"] = torch.zeros(war.war_verify_attn_quant_workspace_bytes(a["params"]), dtype=torch.uint8)
    a["d_out"], a["d_lse"] = torch.zeros_like(a["d_q"]), torch.zeros((B, N, Hq))
    return {**a, **over}


@pytest.mark.parametrize("name,shape", [("d_page_table", (2, 4)), ("d_page_table", (12,)), ("d_prefix_len", (2,)), ("d_num_nodes", (4,)),
                                        ("d_parent", (3, 4)), ("d_parent", (15,)), ("d_out", (3, 5, 4, 128)), ("d_out", (3, 4, 8, 128)),
                                        ("d_lse", (3, 5)), ("d_lse", (3, 5, 4)), ("d_q", (3, 40, 128))])
def test_attention_shapes(war, name, shape):
    a = attention_args(war)
    with pytest.raises(ValueError, match="expected shape|d_q must be"):
        war.war_verify_attn_quant(**{**a, name: torch.zeros(shape, dtype=a[name].dtype)})


def test_attention_params_of_other_tensors(war):
    a = attention_args(war)
    e5m2 = a["k_pool"].view(torch.float8_e5m2)
    wide = torch.zeros((12, 2, 16, 256), dtype=torch.uint8).view(torch.float8_e4m3fn)[..., :128]
    by_token = torch.zeros((12, 16, 2, 128), dtype=torch.uint8).view(torch.float8_e4m3fn).permute(0, 2, 1, 3)
    pages = torch.zeros((9, 2, 16, 128), dtype=torch.uint8).view(torch.float8_e4m3fn)
    fine = torch.ones((12, 2, 2))
    for over in (dict(k_pool=e5m2, v_pool=e5m2), dict(k_pool=wide), dict(v_pool=by_token), dict(k_scale=fine, v_scale=fine),
                 dict(k_pool=pages, v_pool=pages, k_scale=torch.ones((9, 2, 1)), v_scale=torch.ones((9, 2, 1))),
                 dict(d_page_table=torch.zeros((3, 3), **i32)), dict(d_q=a["d_q"][:, :4].contiguous(), d_parent=a["d_parent"][:, :4].contiguous(),
                                                                     d_out=a["d_out"][:, :4].contiguous(), d_lse=None)):
        with pytest.raises(ValueError, match="params do not describe"):
            war.war_verify_attn_quant(**{**a, **over})
    with pytest.raises(ValueError, match="CUDA"):                # nothing but the device is wrong
        war.war_verify_attn_quant(**a)
    a["params"].attn.kernel = 2                                  # the caller's own choices stay
    with pytest.raises(ValueError, match="CUDA"):
        war.war_verify_attn_quant(**a)


def test_tensors_on_another_device_than_the_current_one(war, monkeypatch):
    class On:
        def __init__(self, device):
            self.get_device = lambda: device
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    monkeypatch.setattr(war, "_stream", lambda: 77)
    assert war._stream_of(On(1), None, On(1)) == 77
    for where in ((On(0),), (On(1), On(0)), (None, On(1), On(2))):
        with pytest.raises(ValueError, match="current device, cuda:1"):
            war._stream_of(*where)
