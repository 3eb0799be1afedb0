"""The plain model of pools in four bits: pinned by hand, and against its own definition."""
import numpy as np
import pytest

from tests import mxfp_reference as mx


def test_rounding_to_the_grid():
    x = np.zeros(128)
    x[:14] = [6, 0.25, 0.26, 0.75, 0.74, 1.25, 1.26, 1.75, 2.5, 2.51, 3.5, 5.0, 5.01, -3.0]
    rows, scales = mx.quantise(x[None])
    assert scales[0].tolist() == [127, 0, 0, 0]               # (blocks of zeros take the least scale)
    want = [6, 0, 0.5, 1, 0.5, 1, 1.5, 2, 2, 3, 4, 4, 6, -3]
    assert mx.values(rows, scales)[0, :14].tolist() == want
    assert rows[0, 0] == 0x07 and rows[0, 6] == 0xd7          # element 0 in the low half


@pytest.mark.parametrize("top,scale", [(6.0, 0), (6.0001, 1), (4.0, 0), (3.0, -1), (3.0001, 0), (12.0, 1), (1e-40, -127), (6 * 2.0 ** -127, -127),
                                       (6.1 * 2.0 ** -127, -126), (2.0 ** 127, 125), (3.3e38, 126)])
def test_the_scale_is_the_least_that_holds_the_block(top, scale):
    x = np.full((1, 128), top / 7)
    x[0, 77] = -top
    assert mx.quantise(x)[1][0, 2] == scale + 127
    if scale > -127:
        assert top > 6 * 2.0 ** (scale - 1)
    assert top <= 6 * 2.0 ** scale


def test_what_is_not_finite_takes_its_block_along():
    x = np.ones((3, 128))
    x[0, 40], x[1, 127], x[2, 0] = np.nan, np.inf, -np.inf
    rows, scales = mx.quantise(x)
    nan = np.isnan(mx.values(rows, scales)).reshape(3, 4, 32)
    assert nan.all(-1).tolist() == [[False, True, False, False], [False, False, False, True], [True, False, False, False]]
    assert (nan.all(-1) == nan.any(-1)).all()


def test_values_are_their_own_rounding():
    rng = np.random.default_rng(0)
    rows, scales = rng.integers(0, 256, (50, 64)).astype(np.uint8), rng.integers(1, 250, (50, 4)).astype(np.uint8)
    rows[:, ::16] = 0x7f                                      # a 6 in every block
    v = mx.values(rows, scales)
    again = mx.quantise(v)
    np.testing.assert_array_equal(again[1], scales)
    np.testing.assert_array_equal(mx.values(*again), v)


def test_the_error_is_half_a_step():
    x = np.random.default_rng(1).standard_normal((200, 128))
    rows, scales = mx.quantise(x)
    power = np.repeat(2.0 ** (scales.astype(float) - 127), 32, -1)
    step = np.where(np.abs(x) > 4 * power, 2.0, np.where(np.abs(x) > 2 * power, 1.0, 0.5)) * power
    assert (np.abs(mx.values(rows, scales) - x) <= step / 2 + 1e-15).all()
