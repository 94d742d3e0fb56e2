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
