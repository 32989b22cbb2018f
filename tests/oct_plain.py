"""8-bit rows restated in numpy in 64 bits from their definition."""
from __future__ import annotations

import numpy as np

STEP = 128


def code_values():
    """What the 256 codes stand for."""
    b = np.arange(256)
    e, m = (b >> 3 & 15).astype(np.float64), (b & 7).astype(np.float64)
    v = np.where(e > 0, np.exp2(e - 7) * (1 + m / 8), m * 2.0 ** -9)
    v[[127, 255]] = np.nan
    return np.where(b >= 128, -v, v)


def quantize(x):
    """(codes, scale bytes in whole fours) of the rows of a float64 array: the least exponent by search, the nearest code by
    comparison with all of them, the even one of two that are as near."""
    n, d = x.shape
    steps = -(-d // STEP)
    padded = np.zeros((n, STEP * steps))
    padded[:, :d] = x
    b = padded.reshape(n, steps, STEP)
    levels = code_values()[:127]  # ascending
    middles = (levels[1:] + levels[:-1]) / 2
    with np.errstate(all="ignore"):
        most = np.abs(b).max(axis=2)
        fine = np.isfinite(most)
        e = np.full(most.shape, -127)
        for k in range(-127, 128):
            e = np.where(np.where(fine, most, 0.0) > 448.0 * 2.0 ** k, k + 1, e)
        y = np.where(fine[..., None], np.nan_to_num(b) / np.exp2(e.astype(np.float64))[..., None], 0.0)
    mag = np.abs(y)
    low = np.searchsorted(middles, mag, side="left")  # codes whose middle to the next lies below
    tie = (low < 126) & (mag == middles[np.minimum(low, 125)])
    code = (low + (tie & (low % 2 == 1))).astype(np.uint8)
    code |= np.signbit(np.where(fine[..., None], b, 0.0)).astype(np.uint8) << 7
    scales = np.zeros((n, -(-steps // 4) * 4), np.uint8)
    scales[:, :steps] = np.where(fine, e + 127, 255)
    return code.reshape(n, -1), scales


def values(codes, scales, d):
    steps = codes.shape[1] // STEP
    s = scales[:, :steps].astype(np.float64)
    s = np.where(s == 255, np.nan, np.exp2(s - 127))
    return (code_values()[codes].reshape(-1, steps, STEP) * s[..., None]).reshape(codes.shape[0], -1)[:, :d]
