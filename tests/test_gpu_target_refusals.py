"""war_target with arrays that are missing or offsets that are malformed: reported, the other requests unharmed, nothing read."""
import ctypes as C

import numpy as np
import pytest
import torch

from tests.test_gpu_target import Case, DEV, dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def war():
    from paper_2607_17299_b200 import binding
    return binding


def run_without_ctx(war, c, off):
    """Straight through the C entry point, d_ctx NULL."""
    keep = [dev(x) for x in (c.nn, c.ids, c.parent, off, c.rep)]
    target = torch.full((c.B, c.N), -7, dtype=torch.int32, device=DEV)
    p = war.TargetParams()
    p.B, p.N, p.V, p.dtype = c.B, c.N, c.V, int(c.dtype == torch.float32)
    p.logits_strides[0], p.logits_strides[1] = c.d_logits.stride()[:2]
    t = war.TargetInputs()
    t.d_ctx_off, t.d_repetition = keep[3].data_ptr(), keep[4].data_ptr()
    code = war._lib.war_target(c.d_logits.data_ptr(), *(x.data_ptr() for x in keep[:3]), C.byref(t), C.byref(p), target.data_ptr(), None,
                               torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    return code, target.cpu().numpy()


def test_a_context_without_its_tokens(war):
    c = Case(61, 3, 4, 500, "bf16", mask=None, bias=0, penal=(1.3, None, None))
    c.off = np.array([0, 0, 40, 40], np.int64)                   # the first and the last request have no context
    code, got = run_without_ctx(war, c, c.off)
    assert code == 0 and war.war_device_status() == 1
    c.ctx, c.prompt = np.zeros(40, np.int32), np.zeros(3, np.int32)
    want = c.want()[1]
    assert (got[1] == -1).all()
    np.testing.assert_array_equal(got[[0, 2]], want[[0, 2]])


def test_no_tokens_at_all(war):
    c = Case(62, 3, 4, 500, "f32", mask=None, bias=0, penal=(1.3, None, None))
    c.off, c.ctx, c.prompt = np.zeros(4, np.int64), np.zeros(0, np.int32), np.zeros(3, np.int32)
    want = c.want()[1]
    code, got = run_without_ctx(war, c, c.off)
    assert code == 0 and war.war_device_status() == 0
    np.testing.assert_array_equal(got, want)
    np.testing.assert_array_equal(c.run(war), want)              # an empty tensor has no address


@pytest.mark.parametrize("which", ["d_ctx_off", "d_bias_off"])
def test_negative_offsets(war, which):
    c = Case(63, 3, 4, 500, "bf16", mask=None, bias=6)
    want = c.want()[1]
    off = (c.off if which == "d_ctx_off" else c.boff).copy()
    off[0] = -2
    got = c.run(war, **{which: dev(off)})
    assert (got[0] == -1).all() and war.war_device_status() == 1
    np.testing.assert_array_equal(got[1:], want[1:])
