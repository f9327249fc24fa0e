"""Microscaled rows in plain numpy, 64 bits: the definition, written apart from the library (test infrastructure)."""
import numpy as np

MXFP4, MXFP8 = 0, 1
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
E4M3 = np.array([(c & 7) / 8 * 2.0 ** -6 if c < 8 else (1 + (c & 7) / 8) * 2.0 ** ((c >> 3) - 7) for c in range(127)])
GRID = {MXFP4: E2M1, MXFP8: E4M3}


def code_bytes(fmt, cols):
    return (cols + 7) // 8 * 4 if fmt == MXFP4 else (cols + 3) // 4 * 4


def row_bytes(fmt, cols):
    return (code_bytes(fmt, cols) + (cols + 31) // 32 + 3) // 4 * 4


def scale_exponent(top, fmt):
    """smallest t >= -126 with top <= 2^t * MAX (numbers or arrays)"""
    most, top = GRID[fmt][-1], np.asarray(top, np.float64)
    t = np.maximum(np.ceil(np.log2(np.maximum(top, 2.0 ** -140) / most)), -126.0)
    t = np.where((t > -126) & (top <= most * 2.0 ** (t - 1)), t - 1, t)          # (the logarithm is rounded: its neighbours are looked at)
    return np.where(top > most * 2.0 ** t, t + 1, t).astype(np.int64)


def nearest(u, fmt):
    """codes of the magnitudes u <= MAX: nearest value, of two as near the even code"""
    grid = GRID[fmt]
    low = np.clip(np.searchsorted(grid, u, side="right") - 1, 0, len(grid) - 1)
    high = np.minimum(low + 1, len(grid) - 1)
    a, b = u - grid[low], grid[high] - u
    return np.where((b < a) | ((a == b) & (high % 2 == 0)), high, low)


def encode(x, fmt):
    """x [R, C] -> uint8 [R, row_bytes]; what is nearest to 2^128, past fp32's range, gets the code below"""
    x = np.asarray(x, np.float64)
    R, C = x.shape
    n = code_bytes(fmt, C)
    out = np.zeros((R, row_bytes(fmt, C)), np.uint8)
    codes = np.zeros((R, (C + 31) // 32 * 32), np.uint8)
    for b in range((C + 31) // 32):
        v = x[:, 32 * b:32 * b + 32]
        bad = ~np.isfinite(v).all(1)
        t = scale_exponent(np.where(bad, 1.0, np.abs(v).max(1)), fmt)
        out[:, n + b] = np.where(bad, 255, t + 127)
        u = np.where(bad[:, None], 0.0, np.abs(v)) / 2.0 ** t[:, None].astype(np.float64)
        c = nearest(u, fmt)
        c = np.where(GRID[fmt][c] * 2.0 ** t[:, None].astype(np.float64) >= 2.0 ** 128, c - 1, c)
        c = c | np.signbit(v).astype(np.int64) << (3 if fmt == MXFP4 else 7)
        codes[:, 32 * b:32 * b + v.shape[1]] = np.where(bad[:, None], 0 if fmt == MXFP4 else 0x7F, c)
    if fmt == MXFP4:
        codes = codes[:, 0::2] | codes[:, 1::2] << 4
    out[:, :n] = codes[:, :n]
    return out


def decode(rows, fmt, C):
    """uint8 [R, >= row_bytes] -> float64 [R, C]"""
    n = code_bytes(fmt, C)
    code = rows[:, :n]
    if fmt == MXFP4:
        code = np.stack([code & 15, code >> 4], 2).reshape(rows.shape[0], -1)
        v = E2M1[code & 7] * np.where(code & 8, -1.0, 1.0)
    else:
        mag = np.append(E4M3, np.nan)[code & 127]
        v = mag * np.where(code & 128, -1.0, 1.0)
    s = rows[:, n:n + (C + 31) // 32].astype(np.int64)
    scale = np.where(s == 255, np.nan, 2.0 ** (s - 127.0))
    return v[:, :C] * np.repeat(scale, 32, axis=1)[:, :C]
