"""The plain form of the row cache at the ends of the row types' ranges: finite rows stay finite, wider ones convert as they do elsewhere."""
import numpy as np
import pytest
import torch

from oracle import history as oh


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16, torch.float16])
def test_the_largest_values_stay_finite(bits, dt):
    top = torch.finfo(dt).max
    x = (torch.linspace(0.98, 1.0, 57, dtype=torch.float64)[:, None] * top).clamp(max=top).to(dt)
    codes, s = oh.quantise(x.float().numpy(), bits)
    plain = codes * s[:, None].astype(np.float64)
    # what the rounded scale does to them (not in fp32 with 8 bits: the scale 2^121 * 1.015625 takes the largest value to code 126)
    assert (plain > top).any() or (dt, bits) == (torch.float32, 8)
    back = oh.dequantise(codes, s, top)
    assert torch.from_numpy(back).to(dt).isfinite().all() and (back <= top).all()
    assert (np.abs(back - x.double().numpy()) <= s[:, None] * (0.5 + 2.0 ** -20)).all()
    codes, s = oh.quantise(-x.float().numpy(), bits)
    assert np.array_equal(oh.dequantise(codes, s, top), -back)


@pytest.mark.parametrize("bits", [4, 8])
def test_a_scale_is_the_product_with_the_reciprocal_rounded_up(bits):
    """amax = 7 * 1.5 and 127 * 1.5: amax / L is a bf16 number, and the scale is what the definition's product gives, step for step."""
    L = 7 if bits == 4 else 127
    for m in range(128):
        amax = np.float32(L) * np.float32(1 + m / 128)
        s = np.float32(amax * np.float32(np.float32(1) / np.float32(L)))
        up = int(s.view(np.uint32))
        up = (up + 0xFFFF) >> 16 << 16
        assert oh.quantise(np.array([[amax]]), bits)[1][0] == np.uint32(up).view(np.float32)


def test_wider_rows_pass_the_narrower_range():
    codes, s = oh.quantise(np.full((1, 3), 1e5), 8)
    assert (oh.dequantise(codes, s, 65504.0) > 9e4).all()
    codes, s = oh.quantise(np.array([[np.inf, 1.0], [np.nan, 1.0]]), 4)
    assert np.isnan(oh.dequantise(codes, s, 65504.0)).all()
