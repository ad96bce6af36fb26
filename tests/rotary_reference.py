"""The rotation of head vectors in float64, and the bounds that the fp32 kernel is held to."""
from __future__ import annotations

import numpy as np


def rotate(x, positions, table, interleaved):
    """x float64 [T][H][D], positions [T], table [positions][R/2][2] -> (rotated x, the sum of the
    magnitudes of the two products of each element, 0 where nothing is rotated)."""
    half = table.shape[1]
    c = table[positions, :, 0].astype(np.float64)[:, None, :]
    s = table[positions, :, 1].astype(np.float64)[:, None, :]
    ia = np.arange(half) * 2 if interleaved else np.arange(half)
    ib = ia + (1 if interleaved else half)
    y, mag = x.copy(), np.zeros_like(x)
    a, b = x[..., ia], x[..., ib]
    y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
    mag[..., ia], mag[..., ib] = np.abs(a * c) + np.abs(b * s), np.abs(b * c) + np.abs(a * s)
    return y, mag


def fp32_error(y, mag):
    """One rounded product and one rounded fused multiply-add, each off by at most 2^-24 of its value
    (and the smallest subnormal)."""
    return 2.0 ** -24 * (mag + np.abs(y)) * (1 + 2.0 ** -20) + 2.0 ** -148


def bf16_bound(y, mag):
    """The fp32 error, then half a bf16 step: 2^-8 of the value (half the smallest subnormal below)."""
    e = fp32_error(y, mag)
    return e + 2.0 ** -8 * (np.abs(y) + e) + 2.0 ** -134


def e4m3_bound(y, mag, inv):
    """Of y * inv (one more fp32 rounding, then clamped to 448): half an E4M3 step, 2^-4 of the power of
    two below the value, 2^-10 among the subnormals. Returns (reference, bound)."""
    v = y * float(inv)
    e = fp32_error(y, mag) * float(inv)
    e = e + 2.0 ** -24 * (np.abs(v) + e)
    ref = np.clip(v, -448.0, 448.0)
    top = np.minimum(np.abs(ref) + e, 448.0)
    half_step = 2.0 ** (np.floor(np.log2(np.maximum(top, 2.0 ** -6))) - 4)
    return ref, half_step + e


def positions_of(prefix_lens, new_lens):
    return np.concatenate([np.arange(p, p + n) for p, n in zip(prefix_lens, new_lens)] + [np.zeros(0, np.int64)]).astype(np.int64)
