"""How much two 8-bit parts hold of a query element and of a softmax weight: the bounds that war_verify_attn_quant states, by the
same steps in numpy (a scaled value is rounded to a high part and the remainder to a low part)."""
import numpy as np
import torch


def e4m3(x):
    return torch.from_numpy(x.astype(np.float32)).to(torch.float8_e4m3fn).double().numpy()


def halves(x):
    return x.astype(np.float16)


def split_query(x, largest):
    """x next to the row's largest element: scaled by the power of two that puts that into [128, 256), two e4m3 parts."""
    f = 2.0 ** (7 - np.floor(np.log2(largest)))
    high = e4m3(x * f)
    return (high + e4m3(x * f - high)) / f


def split_weight(x):
    """An e4m3 part cut out of the half of x / 256 and an e5m2 part cut out of the remainder's half, both rounded half up."""
    y = halves((x / 256).astype(np.float32))
    high = ((y.view(np.uint16).astype(np.uint32) + 0x40) & 0x7F80).astype(np.uint16).view(np.float16)
    rest = halves((y.astype(np.float32) - high.astype(np.float32)) * 256)
    low = ((rest.view(np.uint16).astype(np.uint32) + 0x80) & 0xFF00).astype(np.uint16).view(np.float16)
    codes = ((high.view(np.uint16).astype(np.uint32) * 2) >> 8).astype(np.uint8)
    assert (torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy() == high.astype(np.float64) * 256).all()
    return high.astype(np.float64) * 256 + low.astype(np.float64)


def test_query_elements():
    bf16 = torch.arange(0x3000, 0x3F80, dtype=torch.int32).to(torch.uint16).view(torch.bfloat16).double().numpy()       # 2^-31 .. 1
    for largest in (1.0, 1.25, 1.9921875):
        x = bf16[bf16 <= largest]
        err = np.abs(split_query(x, largest) - x)
        assert (err[x >= largest * 2.0 ** -9] == 0).all()
        assert err.max() <= 2.0 ** -17 * largest
    x = np.array([2.0 ** -10 + 2.0 ** -17])
    assert abs(split_query(x, 1.0) - x) == 2.0 ** -17            # reached


def test_weights():
    for e in range(-16, 9):
        x = (2.0 ** e * (1 + np.arange(100003) / 100003)).astype(np.float32)
        x = x[x <= 448]
        err = np.abs(split_weight(x) - x)
        assert (err <= np.maximum(2.0 ** -7.8 * x, 2.0 ** -13.8)).all(), e
