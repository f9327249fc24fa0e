"""The plain microscaled rows of oracle/mx.py, against what the formats' definitions say by themselves."""
import numpy as np
import pytest
import torch

from oracle import mx


def test_eight_bit_grid_is_torchs():
    codes = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(codes, mx.E4M3)
    assert mx.E4M3[-1] == 448


def test_nearest_is_torchs_eight_bit_rounding():
    rng = np.random.default_rng(1)
    u = np.concatenate([rng.uniform(0, 448, 4000), 2.0 ** rng.uniform(-12, 8, 4000), (mx.E4M3[1:] + mx.E4M3[:-1]) / 2]).astype(np.float32)
    want = torch.from_numpy(u).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(mx.nearest(u.astype(np.float64), mx.MXFP8), want)


@pytest.mark.parametrize("u,code", [(0.25, 0), (0.2500001, 1), (0.75, 2), (1.25, 2), (1.75, 4), (2.5, 4), (3.5, 6), (5.0, 6), (5.01, 7), (6.0, 7)])
def test_ties_go_to_the_even_code(u, code):
    assert mx.nearest(np.array([u]), mx.MXFP4)[0] == code


@pytest.mark.parametrize("fmt,top,t", [(0, 6.0, 0), (0, 6.0000001, 1), (0, 3.0, -1), (0, 1e-45, -126), (0, 0.0, -126), (0, 3.4e38, 126),
                                       (1, 448.0, 0), (1, 448.1, 1), (1, 1.0, -8), (1, 0.875, -9), (1, 3.4e38, 120)])
def test_scale_is_the_smallest_that_does_not_saturate(fmt, top, t):
    assert mx.scale_exponent(top, fmt) == t


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("cols", [1, 7, 8, 31, 32, 33, 100])
def test_round_trip_is_within_half_a_step(fmt, cols):
    rng = np.random.default_rng(cols)
    x = rng.standard_normal((20, cols)) * np.exp(rng.standard_normal((20, 1)) * 5)
    rows = mx.encode(x, fmt)
    assert rows.shape[1] == mx.row_bytes(fmt, cols) and rows.shape[1] % 4 == 0
    y = mx.decode(rows, fmt, cols)
    top = np.stack([np.abs(x[:, c // 32 * 32:c // 32 * 32 + 32]).max(1) for c in range(cols)], 1)
    # relative half step of the format, or half of its smallest step at the block's scale (2^t < 2 top / MAX)
    half, least = (2.0 ** -2, 0.25 * 2 / 6) if fmt == 0 else (2.0 ** -4, 2.0 ** -10 * 2 / 448)
    assert (np.abs(y - x) <= np.maximum(half * np.abs(x), least * top)).all()
    assert np.array_equal(mx.encode(y, fmt)[:, :mx.code_bytes(fmt, cols)].size, rows[:, :mx.code_bytes(fmt, cols)].size)
    assert np.array_equal(mx.decode(mx.encode(y, fmt), fmt, cols), y)          # what is held is held again


def test_infinities_and_nan_take_their_block():
    x = np.ones((3, 70))
    x[0, 3], x[1, 40], x[2, 69] = np.inf, np.nan, -np.inf
    for fmt in (0, 1):
        bad = np.isnan(mx.decode(mx.encode(x, fmt), fmt, 70))
        want = np.zeros((3, 70), bool)
        want[0, :32] = want[1, 32:64] = want[2, 64:] = True
        assert np.array_equal(bad, want)
