"""The 64-bit form of the microscaled 4-bit format: the format's own examples."""
import math

import pytest

torch = pytest.importorskip("torch")

from mxref import dequantised, quantise  # noqa: E402


def _row(*v):
    x = torch.zeros(1, 32, dtype=torch.float64)
    x[0, :len(v)] = torch.tensor(v, dtype=torch.float64)
    return x


def test_grid_values_are_kept():
    v = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.5, -6.0)
    for s in (1.0, 2.0 ** 100, 2.0 ** -100, 2.0 ** -127):
        x = _row(*v) * s
        assert torch.equal(dequantised(x), x)


def test_ties_go_to_the_even_code_and_values_saturate():
    x = _row(4.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 5.01, 7.99, -0.25, -2.5)
    want = (4.0, 0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 6.0, 6.0, 0.0, -2.0)
    assert dequantised(x)[0, :12].tolist() == list(want)


def test_scale_is_two_below_the_largest_exponent():
    assert int(quantise(_row(1.0))[1]) == 127 - 2
    assert int(quantise(_row(7.99))[1]) == 127
    assert int(quantise(_row(8.0))[1]) == 128
    assert int(quantise(_row(0.0))[1]) == 0
    assert int(quantise(_row(2.0 ** -133))[1]) == 0


def test_a_block_with_an_infinity_or_nan_is_nan():
    for bad in (math.inf, -math.inf, math.nan):
        x = torch.ones(1, 64, dtype=torch.float64)
        x[0, 5] = bad
        v = dequantised(x)
        assert torch.isnan(v[0, :32]).all() and (v[0, 32:] == 1).all()
