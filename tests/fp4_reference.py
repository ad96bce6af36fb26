"""4-bit pools in float64: the quantisation by distances to the sixteen numbers, pools built from a workload, and the
values that pools stand for. Everything is exact (no rounding but the quantisation's own)."""
from __future__ import annotations

import numpy as np

from paper_2505_23970_amd import workloads as W

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
VALUES = np.concatenate([MAGNITUDES, -MAGNITUDES])
NAN_SCALE = 255


def scale_code(top):
    """Exponent code of the least s = 2^(c - 127) with top < 7 s, c in 3 .. 252."""
    c = 3
    while c < 252 and not top < 7.0 * 2.0 ** (c - 127):
        c += 1
    return c


def scale_codes(tops):
    """scale_code of an array of finite magnitudes."""
    tops = np.asarray(tops, np.float64)
    c = np.full(tops.shape, 3, np.int64)
    for code in range(3, 252):
        c += ~(tops < 7.0 * 2.0 ** (code - 127))
    return c


def quantise(x):
    """x float64 [..., D] -> (codes uint8 [..., D], one a byte; scale codes uint8 [..., D / 32])."""
    x = np.asarray(x, np.float64)
    b = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    bad = np.isnan(b).any(axis=-1)
    b = np.where(bad[..., None], 0.0, b)
    top = np.abs(b).max(axis=-1)
    c = scale_codes(top)
    with np.errstate(invalid="ignore"):
        y = np.abs(b) / 2.0 ** (c[..., None] - 127.0)
    y = np.minimum(y, 6.0)   # (infinities are the largest numbers)
    best = np.full(y.shape, np.inf)
    code = np.zeros(y.shape, np.uint8)
    for k, m in enumerate(MAGNITUDES):
        d = np.abs(y - m)
        nearer = (d < best) | ((d == best) & (k % 2 == 0))
        best, code = np.where(nearer, d, best), np.where(nearer, k, code).astype(np.uint8)
    code = np.where(np.signbit(b), code + 8, code).astype(np.uint8)
    code = np.where(bad[..., None], 0, code).astype(np.uint8)
    return code.reshape(x.shape), np.where(bad, NAN_SCALE, c).astype(np.uint8)


def pack(codes):
    return (codes[..., 0::2] | codes[..., 1::2] << 4).astype(np.uint8)


def unpack(packed):
    return np.stack([packed & 15, packed >> 4], axis=-1).reshape(*packed.shape[:-1], 2 * packed.shape[-1])


def values(packed, scales):
    """float64 [..., D] of codes [..., D / 2] and scale codes [..., D / 32] (NaN blocks: NaN)."""
    v = VALUES[unpack(packed)]
    s = np.where(scales == NAN_SCALE, np.nan, 2.0 ** (scales.astype(np.float64) - 127.0))
    return v * np.repeat(s, 32, axis=-1)


def rows_of(bits):
    return W.bf16_bits_to_f32(bits).astype(np.float64)


def pools(w: W.Workload, rng=None):
    """The initial pools of a workload (prefixes resident): k4, v4 [NB][Hkv][16][D / 2], scales [NB][Hkv][16][D / 32][2].
    Every other slot holds random codes under NaN scales."""
    k = rows_of(w.k_pool)
    v = rows_of(w.v_pool).transpose(0, 1, 3, 2)
    out, scales = [], []
    rng = rng or np.random.default_rng(w.seed + 17)
    for x in (k, v):
        code, s = quantise(x)
        stale = np.isnan(x).all(axis=-1)
        code = np.where(stale[..., None], rng.integers(0, 16, code.shape), code).astype(np.uint8)
        out.append(pack(code))
        scales.append(s)
    return out[0], out[1], np.stack(scales, axis=-1)


def slots(w: W.Workload):
    """(block, slot) of every new token."""
    block, slot = [], []
    for r in range(w.batch):
        pos = np.arange(int(w.prefix_lens[r]), int(w.prefix_lens[r] + w.new_lens[r]))
        block.append(w.block_tables[r][pos // 16])
        slot.append(pos % 16)
    return np.concatenate(block + [np.zeros(0, np.int64)]).astype(np.int64), np.concatenate(slot + [np.zeros(0, np.int64)]).astype(np.int64)


def append(w: W.Workload, k4, v4, scales, keys=None):
    """Copies of the pools after the new tokens' append (keys: float64 [T][Hkv][D] in place of w.k_new)."""
    k4, v4, scales = k4.copy(), v4.copy(), scales.copy()
    block, slot = slots(w)
    ok = (block >= 0) & (block < w.num_blocks)
    keys = rows_of(w.k_new) if keys is None else keys
    for i, (pool, x) in enumerate(((k4, keys), (v4, rows_of(w.v_new)))):
        code, s = quantise(x)
        pool[block[ok], :, slot[ok]] = pack(code)[ok]
        scales[block[ok], :, slot[ok], :, i] = s[ok]
    return k4, v4, scales


def as_bf16_pools(k4, v4, scales):
    """bf16 bit patterns in the bf16 pools' layout of the very same numbers (they are bf16 numbers)."""
    def bits(x):
        b = W.f32_to_bf16_bits(np.nan_to_num(x, nan=0.0).astype(np.float32))
        assert np.array_equal(W.bf16_bits_to_f32(b), np.nan_to_num(x, nan=0.0).astype(np.float32))
        return np.where(np.isnan(x), W.BF16_NAN, b).astype(np.uint16)
    k, v = values(k4, scales[..., 0]), values(v4, scales[..., 1])
    return bits(k), np.ascontiguousarray(bits(v).transpose(0, 1, 3, 2))
