"""Pins of the oracle of the 8-bit checkpoints at the end of the types' range."""
import numpy as np
import pytest

from oracle import site as os_

FLT_MAX = float(np.finfo(np.float32).max)
BF16_MAX = float.fromhex("0x1.fep127")
BORDER = 127 * 2.0 ** 121          # above it the next scale would make 64 2^122 = 2^128 of the largest value


@pytest.mark.parametrize("top", [FLT_MAX, BF16_MAX, float(np.nextafter(np.float32(BORDER), np.float32(np.inf))), BORDER,
                                 float(np.nextafter(np.float32(BORDER), np.float32(0))), 2.0 ** 127, 2.0 ** 126 * 1.99])
def test_largest_values_stay_finite(top):
    """What a checkpoint of finite values stands for is finite in the layer's types and within 1/127 of the largest."""
    rng = np.random.default_rng(1)
    fields = ((0, 40), (1, 9))
    x = (rng.uniform(-1, 1, (6, 67)) * top).astype(np.float32).astype(np.float64)
    x[0, 3], x[1, 35], x[2, 66], x[3], x[4] = top, -top, top, top, -top
    q, e = os_.pack(fields, x)
    v = os_.unpack(fields, q, e)
    assert np.abs(v).max() <= BF16_MAX and np.abs(q.astype(int)).max() <= 127 and e.max() <= 121 + 127
    b = 0
    for lo, hi in ((0, 32), (32, 40), (40, 67)):
        amax = np.abs(x[:, lo:hi]).max(1, keepdims=True)
        assert np.all(np.abs(v - x)[:, lo:hi] <= amax / 127)
        inside = np.abs(x[:, lo:hi]) <= BORDER
        step = np.exp2(e[:, b:b + 1].astype(float) - 127)
        assert np.all((np.abs(v - x)[:, lo:hi] <= step / 2) | ~inside)
        b += 1
