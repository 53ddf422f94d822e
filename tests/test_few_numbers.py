"""Arithmetic that the products on weight pages rely on, for every number that can occur (CPU only)."""
import numpy as np
import pytest


@pytest.mark.parametrize("bits", [8, 4, 3, 2])
def test_two_fp16_numbers_hold_a_centred_code_times_a_scale(bits):
    """(code - 2^(bits - 1)) * scale for every scale that a block of fp16 weights has, at most 131008 / (2^bits - 1): the nearest
    fp16 number of the product with min(scale, 65504 / 2^(bits - 1)), and what that leaves of the product."""
    half = np.arange(0, 0x7c00, dtype=np.uint16).view(np.float16)
    most, limit = np.float16(65504 / 2 ** (bits - 1)), np.float64(np.float16(131008 / (2 ** bits - 1)))
    assert float(most) * 2 ** (bits - 1) == 65504
    s = half[half.astype(np.float64) <= limit]
    for code in range(-2 ** (bits - 1), 2 ** (bits - 1)):
        product = code * s.astype(np.float64)
        near = (code * np.minimum(s, most).astype(np.float64)).astype(np.float16).astype(np.float64)
        rest = (product - near).astype(np.float16).astype(np.float64)
        assert np.all(np.isfinite(near)) and np.array_equal(near + rest, product)


@pytest.mark.parametrize("low,high,relative,absolute", [(-14, 15.99, 2.0 ** -22, 0), (-40, -14, 0, 2.0 ** -36)])
def test_two_fp16_numbers_hold_22_bits_of_an_activation(low, high, relative, absolute):
    """The nearest number, and 2^11 times what it leaves, as the layer for few tokens keeps silu(gate) * up."""
    rng = np.random.default_rng(5)
    h = (2.0 ** rng.uniform(low, high, 200000)).astype(np.float32)
    near = h.astype(np.float16).astype(np.float32)
    rest = ((h - near) * np.float32(2048)).astype(np.float16)
    assert np.all(np.isfinite(near)) and np.all(np.isfinite(rest))
    error = np.abs(h.astype(np.float64) - near.astype(np.float64) - rest.astype(np.float64) / 2048)
    assert np.all(error <= h.astype(np.float64) * relative + absolute)
