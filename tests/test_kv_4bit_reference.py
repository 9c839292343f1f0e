"""The reference of the 4-bit cache against fractions, and the bounds that its documentation gives."""
import numpy as np
import pytest

from tests.kv_4bit_reference import BITS, held, held_exactly, round16


def values(dtype, seed, n=40):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((n, 32)) * 2.0 ** rng.integers(-6, 6, (n, 1)) + rng.integers(-3, 4, (n, 1))
    x[::5] = rng.integers(-8, 9, (len(x[::5]), 32))  # ties
    x[1::5] *= 2.0 ** rng.integers(-20, 1, (len(x[1::5]), 32))
    x[2::10] = rng.integers(-20, 20, (len(x[2::10]), 32)) * 2.0 ** BITS[dtype][1]  # next to nothing
    x[7] = 0.75
    x[8], x[9] = 1.5, 1.5  # differences of more bits than 64-bit floats have, next to borders
    x[8, :6] = -7.5, 7.5, 2.0 ** -23, -2.0 ** -23, 0, 2.0 ** -24
    x[9, :6] = (-7.5, 7.5, 2.0 ** -100, -2.0 ** -100, 0, 2.0 ** -60) if dtype == "bfloat16" else x[8, :6]
    return round16(x, dtype)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_reference_is_exact(dtype):
    x = values(dtype, 0)
    got = held(x, dtype)
    for a, b in zip(x, got):
        assert held_exactly(a.tolist(), dtype) == b.tolist()


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_error_is_half_a_step_and_a_rounding(dtype):
    x = values(dtype, 1)
    span = x.max(-1, keepdims=True) - x.min(-1, keepdims=True)
    bits, least, _ = BITS[dtype]
    # half a step, which is at most span / 15 or the least number; at the highest value 15 times what was cut off the step, less than
    # 15 2^(1 - bits) steps (under a half) or 15 least numbers; the held value is rounded
    step = np.maximum(span / 15, 2.0 ** least)
    bound = np.maximum(step / 2, 15 * 2.0 ** least) + np.abs(held(x, dtype)) * 2.0 ** -bits + 2.0 ** (least - 1)
    assert (np.abs(held(x, dtype) - x) <= bound).all()


def test_a_group_that_is_not_finite_is_not_a_number():
    x = np.ones((3, 40))
    x[0, 3], x[1, 35] = np.inf, np.nan
    got = held(x, "bfloat16")
    assert np.isnan(got[0, :32]).all() and (got[0, 32:] == 1).all()
    assert np.isnan(got[1, 32:]).all() and (got[1, :32] == 1).all() and (got[2] == 1).all()
