"""The plain microscaled rows at the end of fp32's range, and the bytes of what is encoded again."""
import numpy as np
import pytest

from oracle import mx


@pytest.mark.parametrize("fmt,most", [(0, 1.5), (1, 1.875)])
def test_no_finite_number_is_held_as_an_infinity(fmt, most):
    m = np.array([1.0, 1.5, 1.74, 1.75, 1.76, 1.875, 1.93, 1.9375, 1.94, 1.99999988])
    y = mx.decode(mx.encode(m[:, None] * 2.0 ** 127, fmt), fmt, 1)[:, 0] / 2.0 ** 127
    assert y.max() == most
    assert (np.abs(y - m) <= (0.25, 0.0625)[fmt] * m).all()


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("cols", [1, 7, 32, 33, 100])
def test_encoding_again_gives_the_same_bytes(fmt, cols):
    """where the block's largest element, as held, still wants the same scale: it is more than half of the format's largest"""
    x = np.random.default_rng(cols).standard_normal((200, cols)) * np.exp(np.random.default_rng(cols + 1).standard_normal((200, 1)) * 5)
    rows = mx.encode(x, fmt)
    y = mx.decode(rows, fmt, cols)
    again, n, kept = mx.encode(y, fmt), mx.code_bytes(fmt, cols), 0
    for b in range((cols + 31) // 32):
        v = np.abs(y[:, 32 * b:32 * b + 32]).max(1)
        same = v > mx.GRID[fmt][-1] / 2 * 2.0 ** (rows[:, n + b].astype(float) - 127)
        at = slice(16 * b, min(16 * b + 16, n)) if fmt == 0 else slice(32 * b, min(32 * b + 32, n))
        assert np.array_equal(again[same, n + b], rows[same, n + b])
        assert np.array_equal(again[same, at], rows[same, at])
        kept += same.sum()
    assert kept > 100
