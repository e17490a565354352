"""The oracle of the 4-bit cache's format, on heads worked out by hand (no GPU needed)."""
import numpy as np
import pytest
import torch

import oracle.kv4_oracle as k4
from kv4_cases import LEAST, hold, read_back, rounder
from kv_cases import TYPES


def _hold(x, dtype):
    z, s, c = k4.hold(np.array([x], dtype=np.float64), rounder(dtype), LEAST[dtype])
    return float(z[0, 0]), float(s[0, 0]), c[0].tolist()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_codes_of_a_step_of_one(dtype):
    """Ties go to the even code."""
    assert _hold([0.0, 15.0, 7.5, 6.5, 0.4, 0.6, 14.4, 1.0], dtype) == (0.0, 1.0, [0, 15, 8, 6, 0, 1, 14, 1])
    assert _hold([-8.0, 7.0, -0.5, 0.5], dtype) == (-8.0, 1.0, [0, 15, 8, 8])


@pytest.mark.parametrize("dtype,step", [("bf16", 1.0703125), ("f16", 1.06640625)])
def test_the_step_is_of_the_type(dtype, step):
    """16 / 15 = 1.06667 lies between 1.0625 and 1.0703125 of bf16, nearer to the second, and between 1.06640625 and
    1.0673828125 of f16, nearer to the first; codes are of the rounded step."""
    z, s, c = _hold([0.0, 16.0, 8.0], dtype)
    assert s == step and z == 0.0
    assert c == [0, 15, round(8 / step)]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_flat_heads_and_steps_too_small(dtype):
    assert _hold([3.5] * 8, dtype) == (3.5, 0.0, [0] * 8)
    tiny = torch.finfo(TYPES[dtype]).tiny                 # the smallest normal number
    if dtype == "bf16":
        assert _hold([0.0, 14 * tiny], dtype)[1:] == (0.0, [0, 0])       # a step below it counts as 0
        assert _hold([0.0, 15 * tiny], dtype)[1:] == (tiny, [0, 15])
    else:
        # a subnormal step is held: 24 units / 15 = 1.6 -> 2 units, so the largest code is 12
        unit = 2.0 ** -24
        assert _hold([0.0, 24 * unit], dtype) == (0.0, 2 * unit, [0, 12])
        # 21 / 15 = 1.4 -> 1 unit: the quotient of 21 is past the last code
        assert _hold([0.0, 21 * unit], dtype) == (0.0, unit, [0, 15])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_heads_that_are_not_finite(dtype, bad):
    z, s, c = _hold([1.0, bad, 2.0], dtype)
    assert np.isnan(z) and s == 0.0 and c == [0, 0, 0]


def test_a_range_past_fp32():
    top = torch.finfo(torch.bfloat16).max
    z, s, _ = _hold([-top, top], "bf16")
    assert np.isnan(z) and s == 0.0
    top = torch.finfo(torch.float16).max
    assert _hold([-top, top], "f16") == (-top, 8736.0, [0, 15])          # 131008 / 15 = 8733.9; steps of 8 there


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_reading_back_is_within_half_a_step(dtype):
    """The bound of the header: (1/2 + 2^-5) s of an element, and the rounding to the type."""
    g = torch.Generator().manual_seed(0)
    x = torch.randn(64, 128, generator=g).to(TYPES[dtype])
    _, s, _ = hold(x, dtype)
    u = torch.finfo(TYPES[dtype]).eps / 2
    y = read_back(x, dtype).double().numpy()
    assert (np.abs(y - x.double().numpy()) <= (0.5 + 2.0 ** -5) * s + u * np.abs(y)).all()
