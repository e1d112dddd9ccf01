"""Rotary positions, fp64 on the CPU.

TEST INFRASTRUCTURE, NOT PRODUCT: only tests may use this module.

Pair i of a head's first `rotary_dim` channels is a complex number that position p turns by p w_i; the channels are 2i and
2i + 1 (pairs) or i and i + rotary_dim / 2 (halves).  The gradient goes through the conjugate.  Written with complex numbers, which the
kernels do not use.  Pins: tests/test_oracle_rotary.py.
"""
from __future__ import annotations

import numpy as np


def channels(rotary_dim: int, pairs: bool):
    i = np.arange(rotary_dim // 2)
    return (2 * i, 2 * i + 1) if pairs else (i, i + rotary_dim // 2)


def rotate(x, positions, inv_freq, factor=1.0, pairs=False, backward=False) -> np.ndarray:
    """x [..., T, 128], positions broadcastable to [..., T], inv_freq [rotary_dim / 2]."""
    x = np.asarray(x, dtype=np.float64)
    w = np.asarray(inv_freq, dtype=np.float64)
    a, b = channels(2 * w.size, pairs)
    turn = factor * np.exp(1j * (np.asarray(positions, dtype=np.float64)[..., None] * w))
    z = (x[..., a] + 1j * x[..., b]) * (np.conj(turn) if backward else turn)
    y = x.copy()
    y[..., a], y[..., b] = z.real, z.imag
    return y
