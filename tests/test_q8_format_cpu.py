"""The 8-bit format's plain forms, against codes and exponents written out by hand."""
import numpy as np
import pytest
import torch

from perf import more_operators
from test_q8_gpu import _q8, _values

TINY, MOST = 2.0 ** -149, float(np.finfo(np.float32).max)
# largest entries, other entries, exponent, codes
CASES = [
    ([0.0, -0.0], -126, [0, 0]),                                    # a zero vector
    ([TINY, -TINY], -126, [0, 0]),                                  # subnormal numbers far below half a unit
    ([2.0 ** -127, 2.0 ** -126, 1.5 * 2.0 ** -126], -126, [0, 1, 2]),      # a tie goes to the even code
    ([2.0 ** -120, 2.0 ** -126], -126, [64, 1]),                    # the first exponent that is not held up
    ([2.0 ** -119, 2.0 ** -126], -125, [64, 0]),
    ([64.0, 0.5, 1.5, 2.5, -0.5, -1.5], 0, [64, 0, 2, 2, 0, -2]),   # ties
    ([63.9999, 0.25], -1, [127, 0]),                                # just below a power of two: 127.9998 is held at 127
    ([float(np.nextafter(np.float32(64), np.float32(0))), -0.5], -1, [127, -1]),
    ([float(np.nextafter(np.float32(64), np.float32(99))), 63.5], 0, [64, 64]),
    ([127.5, -127.49, 126.5, 125.5], 0, [127, -127, 126, 126]),
    ([-127.999, 1.0], 0, [-127, 1]),
    ([128.0, 127.0, 1.0], 1, [64, 64, 0]),                          # 63.5 is a tie
    ([1.0, -1.0 / 64, 3.0 / 128], -6, [64, -1, 2]),
    ([MOST, -MOST, 2.0 ** 121], 121, [127, -127, 1]),
]


@pytest.mark.parametrize("x,exponent,codes", CASES)
def test_codes_and_exponents(x, exponent, codes):
    for shape in ((-1,), (1, -1)):
        c, e = _q8(np.array(x).reshape(shape))
        assert c.reshape(-1).tolist() == codes and e.reshape(-1).tolist() == [exponent]
        assert c.dtype == np.int8 and e.dtype == np.int8
        assert _values(c, e).reshape(-1).tolist() == [v * 2.0 ** exponent for v in codes]
    c, e = more_operators._quantise(torch.tensor([x], dtype=torch.float64))
    assert c.tolist() == [codes] and e.tolist() == [exponent]
    assert more_operators._value(np.array([x])).tolist() == [[v * 2.0 ** exponent for v in codes]]


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf"), 2.0 ** 128])
def test_vectors_that_are_not_finite_are_marked(bad):
    c, e = _q8(np.array([[1.0, bad], [bad, bad], [3.0, 64.0]]))
    assert c.tolist() == [[0, 0], [0, 0], [3, 64]] and e.tolist() == [-128, -128, 0]
    assert np.isnan(_values(c, e)[:2]).all() and _values(c, e)[2].tolist() == [3.0, 64.0]


def test_what_stands_in_eight_bits_keeps_its_codes():
    x = np.random.RandomState(1).normal(size=(500, 64)) * 2.0 ** np.random.RandomState(2).randint(-60, 60, (500, 1))
    c, e = _q8(x)
    assert np.abs(_values(c, e) - x).max(1).tolist() <= (2.0 ** (e.astype(float) - 1) * (1 + 2 * (np.abs(c).max(1) == 127))).tolist()
    for kept in (torch.float32, torch.bfloat16):      # exact in both
        again = torch.as_tensor(_values(c, e)).to(kept).double().numpy()
        assert np.array_equal(_q8(again)[0], c) and np.array_equal(_q8(again)[1], e)
