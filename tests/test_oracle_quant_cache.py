"""Pins of the 8-bit cache's oracle: its number formats, scales, block numbers and error bounds.  No GPU needed."""
import math

import numpy as np
import pytest
import torch

from oracle import quant_cache as Q

FORMATS = [Q.E4M3, Q.INT8]


def test_e4m3_numbers_are_those_of_an_independent_implementation():
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(Q.numbers(codes, Q.E4M3), want, equal_nan=True)


@pytest.mark.parametrize("fmt", FORMATS)
def test_codes_are_the_nearest_numbers_and_ties_go_to_the_even_one(fmt):
    every = np.array([c for c in range(256) if not np.isnan(Q.numbers(np.uint8([c]), fmt)[0])], dtype=np.uint8)
    if fmt == Q.INT8:
        every = every[every != 128]                         # -128 is not used
    every = every[np.argsort(Q.numbers(every, fmt), kind="stable")]
    n = Q.numbers(every, fmt)
    rng = np.random.default_rng(0)
    x = np.concatenate([n, (n[1:] + n[:-1]) / 2, rng.uniform(-n.max(), n.max(), 2000), rng.normal(size=500) * 1e-3])
    got = Q.numbers(Q.encode(x, 1.0, fmt), fmt)
    best = np.abs(x[:, None] - n[None, :]).min(axis=1)
    assert np.array_equal(np.abs(got - x), best)
    for y, c in zip(x, Q.encode(x, 1.0, fmt)):              # where two are as near, the even code
        near = n[np.abs(n - y) == np.abs(n - y).min()]
        if np.unique(near).size == 2:
            assert c % 2 == 0, y
    if fmt == Q.E4M3:                                       # and the cast of a library, on every tie and number
        cast = torch.from_numpy(x).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
        exact = x.astype(np.float32) == x
        assert np.array_equal(cast[exact], Q.encode(x, 1.0, fmt)[exact])


@pytest.mark.parametrize("fmt", FORMATS)
def test_a_scale_is_the_smallest_power_of_two_that_holds_the_block(fmt):
    most = 448.0 if fmt == Q.E4M3 else 127.0
    for top in [1.0, 448.0, 448.5, 127.0, 127.5, 3.0e38, 1e-30, 1.1754944e-38 * 500, 0.7, most * 2.0 ** -20, most * 2.0 ** 30]:
        s = Q.block_scale(np.array([0.0, -top, top / 3]), fmt)
        assert math.frexp(s)[0] == 0.5 and top <= most * s and top > most * s / 2
    assert Q.block_scale(np.zeros(5), fmt) == 0.0
    assert Q.block_scale(np.array([1e-44]), fmt) == 2.0 ** -126
    assert Q.block_scale(np.array([np.inf, np.nan, 1.0]), fmt) == Q.block_scale(np.array([1.0]), fmt)
    got = Q.numbers(Q.encode(np.array([np.inf, -np.inf, np.nan]), 1.0, fmt), fmt)
    assert np.array_equal(got, [most, -most, 0.0])


def test_scale_numbers_of_segments_never_meet():
    rng = np.random.default_rng(1)
    for _ in range(200):
        n = int(rng.integers(1, 40))
        room = rng.integers(0, rng.choice([2, 33, 200]), n)
        cap = np.concatenate([[0], np.cumsum(room)])
        seen = [Q.scale_number(cap[s], s, row) for s in range(n) for row in range(0, room[s], Q.BLOCK)]
        assert len(set(seen)) == len(seen) and all(0 <= x < Q.scale_count(n, int(cap[-1])) for x in seen)
        assert seen == sorted(seen)


@pytest.mark.parametrize("fmt", FORMATS)
def test_a_growing_block_stays_within_one_step_of_its_last_scale(fmt):
    # int8: every rounding to a scale t is off by at most t / 2, and the scales at least double: the sum stays below t.
    # e4m3: the codes are floating-point numbers, a growing scale only moves small ones out of range: half a step of 2^-9 t each
    rng = np.random.default_rng(2)
    x = rng.normal(size=(32, 128)) * np.exp2(np.arange(32) / 4.0)[:, None]
    codes, scales = np.zeros((32, 128), dtype=np.uint8), np.zeros(2)
    for i in range(32):
        Q.append_row(x[i], i, 0, 0, codes, scales, fmt)
    got = Q.read_segment(codes, scales, 0, 0, 32, fmt)
    t = scales[0]
    assert t == Q.block_scale(x, fmt)
    bound = t if fmt == Q.INT8 else 2.0 ** -4 * np.abs(x) + 2.0 ** -9 * t
    assert (np.abs(got - x) < bound).all()
    # rows that need no larger scale are the rows of a block quantised at once
    codes2, scales2 = np.zeros((32, 128), dtype=np.uint8), np.zeros(2)
    Q.write_segment(x[::-1], 0, 0, codes2, scales2, fmt)
    codes3, scales3 = np.zeros((32, 128), dtype=np.uint8), np.zeros(2)
    for i in range(32):
        Q.append_row(x[31 - i], i, 0, 0, codes3, scales3, fmt)
    if scales2[0] == Q.block_scale(x[31], fmt):
        assert np.array_equal(codes2, codes3) and np.array_equal(scales2, scales3)


@pytest.mark.parametrize("fmt,bound", [(Q.E4M3, 2.0 ** -4), (Q.INT8, 1 / 127)])
def test_error_of_the_formats(fmt, bound):
    rng = np.random.default_rng(3)
    x = rng.normal(size=(96, 128))
    codes, scales = np.zeros((96, 128), dtype=np.uint8), np.zeros(4)
    Q.write_segment(x, 0, 0, codes, scales, fmt)
    err = np.abs(Q.read_segment(codes, scales, 0, 0, 96, fmt) - x)
    top = np.abs(x).reshape(3, -1).max(axis=1).repeat(32)[:, None]
    assert (err <= (bound * np.maximum(np.abs(x), 2.0 ** -6 / 448 * 2 * top) if fmt == Q.E4M3 else bound * top)).all()
