"""Pins of the rotary oracle, and the library's frequency tables (host arithmetic) against their formulas.  No GPU needed."""
import math

import numpy as np
import pytest

from oracle import rotary as R
from paper_2605_06676_amd import lkv


def _w(r, base=10000.0):
    return base ** (-np.arange(0, r, 2) / r)


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("r", [2, 34, 128])
def test_rotation_is_one_and_dot_products_depend_on_the_distance_alone(pairs, r):
    rng = np.random.default_rng(r)
    x, y = rng.normal(size=(2, 128))
    w = _w(r)
    for p, q in [(0, 0), (5, 2), (1000, 997), (-7, 3)]:
        a, b = R.rotate(x[None], [p], w, pairs=pairs)[0], R.rotate(y[None], [q], w, pairs=pairs)[0]
        assert np.isclose(np.linalg.norm(a), np.linalg.norm(x))
        assert np.isclose(a @ b, R.rotate(x[None], [p - q], w, pairs=pairs)[0] @ y)
        assert np.array_equal(a[r:], x[r:])
    assert np.array_equal(R.rotate(x[None], [0], w, pairs=pairs)[0], x)


@pytest.mark.parametrize("pairs", [False, True])
def test_one_pair_by_hand(pairs):
    x = np.zeros(128)
    a, b = R.channels(8, pairs)
    x[a[1]], x[b[1]] = 2.0, 3.0
    y = R.rotate(x[None], [4], _w(8), factor=1.5, pairs=pairs)[0]
    t = 4 * 10000.0 ** (-2 / 8)
    assert np.isclose(y[a[1]], 1.5 * (2 * math.cos(t) - 3 * math.sin(t))) and np.isclose(y[b[1]], 1.5 * (3 * math.cos(t) + 2 * math.sin(t)))
    assert np.count_nonzero(y) == 2


def test_backward_is_the_transpose():
    rng = np.random.default_rng(0)
    x, g = rng.normal(size=(2, 3, 128))
    for pairs in (False, True):
        y = R.rotate(x, [1, 9, 77], _w(96), 1.3, pairs)
        dx = R.rotate(g, [1, 9, 77], _w(96), 1.3, pairs, backward=True)
        assert np.isclose((y * g).sum(), (x * dx).sum())


def test_plain_linear_and_base_frequencies():
    w, f = lkv.lkv_rope_frequencies(lkv.ROPE_PLAIN, 128, 10000.0)
    assert f == 1.0 and np.allclose(w, _w(128), rtol=1e-14)
    w, f = lkv.lkv_rope_frequencies(lkv.ROPE_LINEAR, 96, 10000.0, stretch=4.0)
    assert f == 1.0 and np.allclose(w, _w(96) / 4, rtol=1e-14)
    w, f = lkv.lkv_rope_frequencies(lkv.ROPE_BASE, 64, 10000.0, stretch=8.0)
    # the base is chosen so that the slowest pair is stretched by exactly 8 and the fastest not at all
    assert f == 1.0 and np.isclose(w[-1], _w(64)[-1] / 8) and w[0] == 1.0


def test_by_parts_frequencies():
    r, base, s, n = 128, 10000.0, 16.0, 4096.0
    w, f = lkv.lkv_rope_frequencies(lkv.ROPE_PARTS, r, base, s, n, 1.0, 32.0)
    plain = _w(r, base)
    turns = n * plain / (2 * math.pi)
    share = (plain / w - 1) / (s - 1)                     # 0: kept, 1: stretched; between them 1 / w is not linear but w is
    assert np.isclose(f, 0.1 * math.log(16.0) + 1)
    first, last = int(np.searchsorted(-turns, -32.0)) - 1, int(np.searchsorted(-turns, -1.0))
    assert np.allclose(w[:first + 1], plain[:first + 1], rtol=1e-14) and np.allclose(w[last:], plain[last:] / s, rtol=1e-14)
    ramp = (np.arange(64) - first) / (last - first)
    mid = slice(first, last + 1)
    assert np.allclose(w[mid], (plain * (1 - ramp) + plain / s * ramp)[mid], rtol=1e-13)
    assert (share >= -1e-12).all() and (share <= 1 + 1e-12).all() and first < last


def test_wavelength_frequencies():
    r, base, s, n = 128, 500000.0, 8.0, 8192.0
    w, f = lkv.lkv_rope_frequencies(lkv.ROPE_WAVELENGTHS, r, base, s, n, 1.0, 4.0)
    plain = _w(r, base)
    length = 2 * math.pi / plain
    for i in range(64):
        if length[i] < n / 4:
            want = plain[i]
        elif length[i] > n / 1:
            want = plain[i] / s
        else:
            t = (n / length[i] - 1) / (4 - 1)
            want = (1 - t) * plain[i] / s + t * plain[i]
        assert np.isclose(w[i], want, rtol=1e-13)
    assert f == 1.0


@pytest.mark.parametrize("bad", [dict(kind=5), dict(kind=-1), dict(rotary_dim=0), dict(rotary_dim=3), dict(rotary_dim=130), dict(base=1.0),
                                 dict(base=float("nan")), dict(base=float("inf")), dict(kind=1, stretch=0.5), dict(kind=1, stretch=float("nan")),
                                 dict(kind=2, rotary_dim=2, stretch=2.0), dict(kind=3, stretch=2.0, trained_len=0.0, low=1, high=32),
                                 dict(kind=3, stretch=2.0, trained_len=4096.0, low=4.0, high=4.0),
                                 dict(kind=4, stretch=2.0, trained_len=4096.0, low=0.0, high=4.0)])
def test_frequency_arguments_are_checked(bad):
    with pytest.raises(lkv.LkvError) as e:
        lkv.lkv_rope_frequencies(**{**dict(kind=0, rotary_dim=128, base=10000.0), **bad})
    assert e.value.status == 1


def test_scale_counts_and_null_contexts():
    lib = lkv.load_library()
    assert lkv.lkv_quant_scales(256, 1258291) == 1258291 // 32 + 256 and lkv.lkv_quant_scales(1, 0) == 1
    assert lkv.lkv_quant_scales(0, 100) == 0 and lkv.lkv_quant_scales(3, -1) == 0
    n = lkv.lkv_decode_quant_workspace_bytes(256, 1258291, 32, 8)
    assert n % 256 == 0 and n >= 256 * 4 * 130 * 4
    assert lkv.lkv_decode_quant_workspace_bytes(-1, 10, 32, 8) == 0 and lkv.lkv_decode_quant_workspace_bytes(1, 10, 4, 8) == 0
    assert lib.lkv_compact_quant(None, None, None, None, None, 0, 0, None, None, None, None, None) == 1
    assert lib.lkv_append_quant(None, 1, 1, 1, 128, None, None, None, None, None, None, None, None, None, None, None) == 1
    assert lib.lkv_decode_attn_quant(None, 1, 1, 1, 1, 128, None, None, None, None, 0, 1.0, None, None, None, 0, None) == 1
    assert lib.lkv_reevict_quant(None, 1, 128, None, None, None, None, None, None, 0, None, None, None, None, None, None, None, None) == 1
    assert lib.lkv_rope(None, None, 0, 1, 1, 1, 128, None, None, None, None, None, 0, 0, 0, None) == 1
    assert lib.lkv_rope_frequencies(None, None, None) == 1
