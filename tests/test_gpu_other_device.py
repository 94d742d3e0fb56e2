"""The cache and logits calls run on the current device: tensors of another one are refused before anything is launched."""
import pytest
import torch

from tests import test_quant_cpu_binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def war():
    from paper_2607_17299_b200 import binding
    return binding


def store_args(war):
    a = B.attention_args(war)
    B_, N, Hq, _ = a["d_q"].shape
    row = lambda: torch.zeros((B_, N, 2, 128), dtype=torch.bfloat16)
    return dict(d_q=a["d_q"], d_k=row(), d_v=row(), d_inv_freq=torch.ones(64), page_table=a["d_page_table"], d_prefix_len=a["d_prefix_len"],
                d_num_nodes=a["d_num_nodes"], d_parent=a["d_parent"], k_pool=a["k_pool"], v_pool=a["v_pool"], k_scale=a["k_scale"],
                v_scale=a["v_scale"], d_q_out=a["d_out"])


CALLS = {"war_rope_store": store_args, "war_verify_attn_quant": B.attention_args, "war_target": lambda war: B.target_args(),
         "war_commit_quant": lambda war: B.commit_args()}


@pytest.mark.parametrize("name", list(CALLS))
def test_refused(war, monkeypatch, name):
    args = {k: v.to(DEV) if isinstance(v, torch.Tensor) else v for k, v in CALLS[name](war).items()}
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    with pytest.raises(ValueError, match="current device, cuda:1"):
        getattr(war, name)(**args)
    monkeypatch.undo()
    getattr(war, name)(**args)                                   # (no slots, nothing accepted)
    torch.cuda.synchronize()
    assert war.war_device_status() == 0
