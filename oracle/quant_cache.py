"""The packed cache in 8 bits, fp64 on the CPU.

TEST INFRASTRUCTURE, NOT PRODUCT: only tests may use this module.

Every 32 rows of a segment, counted from its first row, are a block; K and V have a scale each per block: the smallest power
of two s with max|x| <= Q s (Q = 448 for e4m3, 127 for int8), at least 2^-126, 0 for a block without a finite value other than
0.  A code is x / s rounded to the nearest number of the format, ties to the even one; NaN is 0, infinities are the largest.
Block b of segment s, whose first row is cap[s], has scale number cap[s] // 32 + s + b.

The e4m3 numbers are listed from the format's definition (sign, 4 exponent bits with bias 7, 3 mantissa bits, no infinities,
the all-ones code is NaN) and rounding looks them up, so nothing here shares a shortcut with the kernels.

Pins: tests/test_oracle_quant_cache.py.
"""
from __future__ import annotations

import math

import numpy as np

from . import lkv_oracle as O

BLOCK = 32
E4M3, INT8 = 0, 1


def _e4m3_magnitudes() -> np.ndarray:
    out = []
    for code in range(127):
        e, m = code >> 3, code & 7
        out.append(math.ldexp(m / 8, -6) if e == 0 else math.ldexp(1 + m / 8, e - 7))
    return np.array(out)


_MAGNITUDES = {E4M3: _e4m3_magnitudes(), INT8: np.arange(128, dtype=np.float64)}


def numbers(codes: np.ndarray, fmt: int) -> np.ndarray:
    """The numbers that uint8 codes stand for, in units of the scale."""
    c = np.asarray(codes, dtype=np.uint8)
    if fmt == INT8:
        return c.view(np.int8).astype(np.float64)
    m = np.append(_MAGNITUDES[E4M3], np.nan)[c & 127]
    return np.where(c & 128, -m, m)


def block_scale(x: np.ndarray, fmt: int) -> float:
    a = np.abs(np.asarray(x, dtype=np.float64))
    a = a[np.isfinite(a)]
    top = a.max() if a.size else 0.0
    if top == 0.0:
        return 0.0
    k = -126
    while _MAGNITUDES[fmt][-1] * math.ldexp(1.0, k) < top:
        k += 1
    return math.ldexp(1.0, k)


def encode(x: np.ndarray, scale, fmt: int) -> np.ndarray:
    """uint8 codes of x (fp64) with this scale."""
    x = np.asarray(x, dtype=np.float64)
    table = _MAGNITUDES[fmt]
    if scale == 0.0:   # zeros keep their sign, as everywhere
        return np.where((x == 0) & np.signbit(x) & (fmt == E4M3), 128, 0).astype(np.uint8)
    y = np.where(np.isnan(x), 0.0, x) / scale
    a = np.minimum(np.abs(y), table[-1])
    hi = np.minimum(np.searchsorted(table, a), table.size - 1)
    lo = np.maximum(hi - 1, 0)
    up, down = table[hi] - a, a - table[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)) | (table[hi] == a), hi, lo)
    if fmt == INT8:
        return np.where(y < 0, -code, code).astype(np.int8).view(np.uint8)
    return (code | np.where(np.signbit(y), 128, 0)).astype(np.uint8)


def scale_count(n_segments: int, rows: int) -> int:
    return rows // BLOCK + n_segments


def scale_number(cap: int, s: int, row: int) -> int:
    """Number of the scale of row `row` of segment s, which starts at row cap."""
    return int(cap) // BLOCK + int(s) + int(row) // BLOCK


def write_segment(x: np.ndarray, cap: int, s: int, codes: np.ndarray, scales: np.ndarray, fmt: int) -> None:
    """Quantises the rows x (fp64 [n, 128]) of segment s into its first rows."""
    for at in range(0, x.shape[0], BLOCK):
        part = x[at:at + BLOCK]
        t = block_scale(part, fmt)
        codes[cap + at:cap + at + part.shape[0]] = encode(part, t, fmt)
        scales[scale_number(cap, s, at)] = t


def read_segment(codes, scales, cap: int, s: int, n: int, fmt: int) -> np.ndarray:
    t = np.array([scales[scale_number(cap, s, i)] for i in range(n)], dtype=np.float64).reshape(-1, 1)
    return numbers(codes[cap:cap + n], fmt) * t


def append_row(x: np.ndarray, used: int, cap: int, s: int, codes, scales, fmt: int) -> None:
    """Row `used` of segment s becomes x (fp64 [128]); the block's rows follow its scale where that has to grow."""
    at = scale_number(cap, s, used)
    first = used // BLOCK * BLOCK
    need = block_scale(x, fmt)
    old = float(scales[at]) if used > first else 0.0
    t = max(old, need)
    if old < t and used > first:
        held = numbers(codes[cap + first:cap + used], fmt) * old
        codes[cap + first:cap + used] = encode(held, t, fmt)
    scales[at] = t
    codes[cap + used] = encode(x, t, fmt)


def unpack(codes, scales, cap, lengths, fmt: int) -> np.ndarray:
    """All rows in use as fp64, segment after segment without spare rows."""
    parts = [read_segment(codes, scales, int(cap[s]), s, int(n), fmt) for s, n in enumerate(lengths)]
    return np.concatenate(parts) if parts else np.zeros((0, 128))


def decode(q64, k_codes, v_codes, k_scale, v_scale, cap, lengths, H: int, scale: float, fmt: int):
    """Decode attention (lkv_oracle.decode_attn) over the values that the cache stands for.  q64 [L, Hq, d]."""
    offsets = np.concatenate([[0], np.cumsum(np.asarray(lengths, dtype=np.int64))])
    return O.decode_attn(q64, unpack(k_codes, k_scale, cap, lengths, fmt), unpack(v_codes, v_scale, cap, lengths, fmt), offsets, H, scale)
