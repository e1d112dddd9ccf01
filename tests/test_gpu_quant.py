"""The packed cache in 8 bits on the GPU against the 64-bit oracle: compaction, appending, re-eviction (codes, scales, scores
and layout bit for bit) and decode attention.

Decode tolerance.  Per query head, with S = sum_c |q_c k_c| over the 128 channels: the scores are fp32 sums of exact products,
off by at most 2^-24 (128 + 4) scale S (one rounding for each of the 128 additions, four for the scales) = d.  A softmax weight then
is off by at most 2 d relative, plus 2^-21 for exp2 and its argument (whose rounding is counted in d) and 2^-16 for the weights in
two parts (each rounded at 2^-9: 2^-18 and the sums' 2^-24 per row, n rows and a chunk's merge).  The output is a mean of values no
larger than max|v|: |out - ref| <= (2 d + 2^-16 + (n + 64) 2^-24) max|v|, and the log-sum-exp is off by d + 2^-21 + (n + 64) 2^-24 + 2^-22 |lse|.
"""
import numpy as np
import pytest
import torch

from oracle import lkv_oracle as O
from oracle import quant_cache as Q
from oracle import rotary as R
from paper_2605_06676_amd import lkv
from paper_2605_06676_amd import workloads as W

import gpu_util as G

pytestmark = pytest.mark.gpu

KINDS = {Q.E4M3: torch.float8_e4m3fn, Q.INT8: torch.int8}
FORMATS = [pytest.param(Q.E4M3, id="e4m3"), pytest.param(Q.INT8, id="int8")]
GUARD_CODE, GUARD_SCALE = 0x5A, -7.5


@pytest.fixture(scope="module")
def ctx():
    c = lkv.Context(0)
    yield c
    c.close()


def bf16(x):
    return torch.from_numpy(np.asarray(x, dtype=np.float32)).to(torch.bfloat16)


def i32(x):
    return torch.from_numpy(np.asarray(x, dtype=np.int32)).cuda()


class Packed:
    """A packed 8-bit cache on the GPU, full of guard values, next to the same arrays on the host."""

    def __init__(self, rows, n_seg, fmt, extra=2):
        self.fmt, self.rows = fmt, rows
        n = Q.scale_count(n_seg, rows) + extra
        self.kc, self.vc = (np.full((rows + extra, 128), GUARD_CODE, dtype=np.uint8) for _ in range(2))
        self.ks, self.vs = (np.full(n, GUARD_SCALE) for _ in range(2))
        self.dev = [torch.from_numpy(x.copy()).cuda() for x in (self.kc, self.vc)] + [torch.from_numpy(x).float().cuda() for x in (self.ks, self.vs)]
        self.c = lkv.QuantRows(self.dev[0].view(KINDS[fmt]), self.dev[1].view(KINDS[fmt]), self.dev[2], self.dev[3])

    def upload(self):
        for d, x in zip(self.dev, (self.kc, self.vc, self.ks, self.vs)):
            d.copy_(torch.from_numpy(x).to(d.dtype))
        return self

    def assert_same(self, what=""):
        torch.cuda.synchronize()
        for name, d, x in zip(("k", "v", "k_scale", "v_scale"), self.dev, (self.kc, self.vc, self.ks, self.vs)):
            got = d.cpu().numpy()
            assert np.array_equal(got.astype(np.float64), x.astype(np.float64)), \
                f"{what} {name}: {(got != x).sum()} differ, first at {np.argwhere(got != x)[:3].tolist()}"


def _filled(lengths, slack, fmt, seed, spread=1.0):
    """A packed cache with these rows in use; returns it with cap_offsets."""
    rng = np.random.default_rng(seed)
    lengths = np.asarray(lengths)
    cap = np.concatenate([[0], np.cumsum(lengths + slack)])
    p = Packed(int(cap[-1]), len(lengths), fmt)
    for s, n in enumerate(lengths):
        for codes, scales in ((p.kc, p.ks), (p.vc, p.vs)):
            x = rng.normal(size=(int(n), 128)) * np.exp(rng.normal(size=(int(n), 1)) * 0.5)
            x[:, rng.integers(0, 128, 2)] *= 10 * spread
            Q.write_segment(bf16(x).double().numpy(), int(cap[s]), s, codes, scales, fmt)
    return p.upload(), cap


def _cache(Ts, L, H, seed, special=False):
    rng = np.random.default_rng(seed)
    ks, vs = [], []
    for T in Ts:
        for dst in (ks, vs):
            x = rng.normal(size=(L, H, T, 128)) * np.exp2(rng.integers(-3, 4, size=(L, H, T, 1)))
            x[..., 5] *= 10
            x = bf16(x)
            if special:                                       # zeros, tiny values, the largest ones, NaN and infinities
                f = x.reshape(-1, 128)
                f[:40] = 0.0
                f[40:80] *= 2.0 ** -130
                f[80] = 3.3e38
                f[120, 3], f[121, 4], f[122, 5] = float("nan"), float("inf"), float("-inf")
                f[160:200] = float("nan")
            dst.append(x)
    return ks, vs


def _select(Ts, budgets, L, H, seed):
    """Ascending row numbers of every segment and the offsets."""
    rng = np.random.default_rng(seed)
    idx = [np.sort(rng.choice(T, int(b), replace=False)) for T, bs in zip(Ts, budgets) for b in np.asarray(bs).reshape(-1)]
    off = np.concatenate([[0], np.cumsum([len(i) for i in idx])])
    return np.concatenate(idx + [np.zeros(0, dtype=int)]), off


def _compact_case(ctx, Ts, L, H, budgets, fmt, slack, seed, with_up=True, special=False, stream=None):
    ks, vs = _cache(Ts, L, H, seed, special)
    idx, off = _select(Ts, budgets, L, H, seed + 1)
    n_seg, total = len(off) - 1, int(off[-1])
    u = [np.random.default_rng(seed + 2 + i).normal(size=(L, H, T)).astype(np.float32) for i, T in enumerate(Ts)]
    rows = total + n_seg * slack
    p = Packed(rows, n_seg, fmt)
    cap = off + slack * np.arange(n_seg + 1)
    up_ref = np.full(rows + 1, -3.0, dtype=np.float32)
    for s in range(n_seg):
        q, lh = divmod(s, L * H)
        sel = idx[off[s]:off[s + 1]]
        for src, codes, scales in ((ks, p.kc, p.ks), (vs, p.vc, p.vs)):
            Q.write_segment(src[q].reshape(L * H, Ts[q], 128)[lh][torch.from_numpy(sel)].double().numpy(), int(cap[s]), s, codes, scales, fmt)
        up_ref[cap[s]:cap[s] + len(sel)] = u[q].reshape(L * H, Ts[q])[lh][sel]
    cache = lkv.Cache([k.cuda() for k in ks], [v.cuda() for v in vs], H)
    d_idx, d_off = i32(np.append(idx, 0)), i32(off)
    up = torch.full((rows + 1,), -3.0, device="cuda")
    d_cap, d_len = i32(np.full(n_seg + 1, -1)), i32(np.full(n_seg, -1))
    kw = dict(scores=[torch.from_numpy(x).cuda() for x in u], up=up) if with_up else {}
    if slack or with_up:
        kw.update(cap_offsets=d_cap, lengths=d_len)
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())
    lkv.lkv_compact_quant(ctx, cache, d_idx, d_off, total, p.c, slack=slack, stream=stream, **kw)
    if stream is not None:
        stream.synchronize()
    p.assert_same("compact")
    if with_up:
        assert np.array_equal(up.cpu().numpy(), up_ref)
    if "lengths" in kw:
        assert np.array_equal(d_cap.cpu().numpy(), cap) and np.array_equal(d_len.cpu().numpy(), np.diff(off))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("slack,with_up", [(0, False), (0, True), (1, True), (45, False), (32, True)])
def test_compaction(ctx, fmt, slack, with_up):
    Ts, L, H = [333, 64, 1], 2, 3
    budgets = [[[0, 1, 31], [32, 33, 333]], [[64, 0, 63], [7, 40, 1]], [[1, 1, 0], [0, 1, 1]]]
    _compact_case(ctx, Ts, L, H, budgets, fmt, slack, 11 + slack, with_up)


@pytest.mark.parametrize("fmt", FORMATS)
def test_compaction_of_values_at_the_ends_of_their_range(ctx, fmt):
    _compact_case(ctx, [400], 1, 2, [[[400, 123]]], fmt, 3, 5, special=True)


@pytest.mark.parametrize("fmt", FORMATS)
def test_compaction_of_more_sequences_than_a_launch_describes(ctx, fmt):
    rng = np.random.default_rng(3)
    Ts = rng.integers(1, 60, 70).tolist()
    budgets = [rng.integers(0, T + 1, (1, 2)) for T in Ts]
    _compact_case(ctx, Ts, 1, 2, budgets, fmt, 5, 21)


def test_compaction_of_nothing(ctx):
    _compact_case(ctx, [50, 3], 1, 2, [[[0, 0]], [[0, 0]]], Q.INT8, 4, 2)
    _compact_case(ctx, [50, 3], 1, 2, [[[0, 0]], [[0, 0]]], Q.E4M3, 0, 2, with_up=False)


def test_compaction_on_another_stream_and_of_many_segments(ctx):
    rng = np.random.default_rng(4)
    _compact_case(ctx, [90], 37, 31, [rng.integers(0, 91, (37, 31)) // rng.integers(1, 9, (37, 31))], Q.E4M3, 2, 9, stream=torch.cuda.Stream())


# ---- decode ---------------------------------------------------------------------------------------


def _decode(ctx, p, cap, lengths, q, H, scale, d_len=True, stream=None):
    """q: bf16 host [n_seq, L, Hq, 128]."""
    n_seq, L, Hq, _ = q.shape
    n_seg, rows = n_seq * L * H, int(cap[-1])
    need = lkv.lkv_decode_quant_workspace_bytes(n_seg, rows, Hq, H)
    ws = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device="cuda")   # NaN where it is read unwritten
    out = torch.full((n_seq, L, Hq, 128), float("nan"), device="cuda")
    lse = torch.full((n_seq, L, Hq), float("nan"), device="cuda")
    dq, dcap, dlen = q.cuda(), i32(cap), i32(lengths) if d_len else None
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())
    lkv.lkv_decode_attn_quant(ctx, n_seq, L, H, Hq, 128, dq, p.c, dcap, dlen, rows, scale, out, lse, ws[:need], stream=stream)
    if stream is not None:
        stream.synchronize()
    torch.cuda.synchronize()
    assert (ws[need:] == 0xFF).all()
    return out.cpu().numpy().reshape(-1, 128), lse.cpu().numpy().reshape(-1)


def _assert_decode(p, cap, lengths, q, H, scale, out, lse):
    n_seq, L, Hq, _ = q.shape
    g = Hq // H
    q64 = q.double().numpy().reshape(-1, g, 128)
    for s, n in enumerate(lengths):
        o, z = out[s * g:(s + 1) * g], lse[s * g:(s + 1) * g]
        if n == 0:
            assert (o == 0).all() and np.isneginf(z).all(), s
            continue
        k = Q.read_segment(p.kc, p.ks, int(cap[s]), s, int(n), p.fmt)
        v = Q.read_segment(p.vc, p.vs, int(cap[s]), s, int(n), p.fmt)
        a = scale * (q64[s] @ k.T)
        top = a.max(axis=1, keepdims=True)
        e = np.exp(a - top)
        ref, zr = (e / e.sum(axis=1, keepdims=True)) @ v, top[:, 0] + np.log(e.sum(axis=1))
        d = 132 * 2.0 ** -24 * abs(scale) * (np.abs(q64[s]) @ np.abs(k).T).max(axis=1)
        tol = (2 * d + 2.0 ** -16 + (n + 64) * 2.0 ** -24)[:, None] * np.abs(v).max()
        assert (np.abs(o - ref) <= tol).all(), f"segment {s} of {n} rows: {(np.abs(o - ref) / np.maximum(tol, 1e-300)).max():.3g} of the tolerance"
        ztol = d + 2.0 ** -21 + (n + 64) * 2.0 ** -24 + 2.0 ** -22 * np.abs(zr)
        assert (np.abs(z - zr) <= ztol).all(), f"segment {s} of {n} rows: lse"


def _queries(n_seq, L, Hq, seed, size=1.0):
    return bf16(np.random.default_rng(seed).normal(size=(n_seq, L, Hq, 128)) * size)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("H,g", [(8, 4), (4, 7), (3, 1), (2, 16)])
@pytest.mark.parametrize("slack", [0, 13])
def test_decode_of_short_and_empty_segments(ctx, fmt, H, g, slack):
    lengths = np.array([0, 1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 0, 500, 3, 17, 96, 97, 1, 256, 257, 0, 40])
    lengths = np.resize(lengths, 24 if 24 % H == 0 else 24 // H * H)
    p, cap = _filled(lengths, slack, fmt, 100 * H + slack)
    q = _queries(1, len(lengths) // H, H * g, 7)
    out, lse = _decode(ctx, p, cap, lengths, q, H, 128 ** -0.5, d_len=slack > 0)
    _assert_decode(p, cap, lengths, q, H, 128 ** -0.5, out, lse)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("lengths", [[40000], [5, 30000, 0, 9000], [1] * 7 + [70000], [3000] * 16])
def test_decode_of_long_segments(ctx, fmt, lengths):
    p, cap = _filled(lengths, 3, fmt, len(lengths))
    q = _queries(1, 1, 4 * len(lengths), 8, 3.0)
    out, lse = _decode(ctx, p, cap, lengths, q, len(lengths), 128 ** -0.5)
    _assert_decode(p, cap, lengths, q, len(lengths), 128 ** -0.5, out, lse)


@pytest.mark.parametrize("fmt", FORMATS)
def test_decode_of_many_segments(ctx, fmt):
    rng = np.random.default_rng(5)
    lengths = (rng.exponential(40.0, 3 * 7 * 100)).astype(int)
    p, cap = _filled(lengths, 0, fmt, 6)
    q = _queries(3, 100, 14, 9)
    out, lse = _decode(ctx, p, cap, lengths, q, 7, 128 ** -0.5, d_len=False)
    _assert_decode(p, cap, lengths, q, 7, 128 ** -0.5, out, lse)
    again = _decode(ctx, p, cap, lengths, q, 7, 128 ** -0.5, d_len=False, stream=torch.cuda.Stream())
    assert np.array_equal(out, again[0]) and np.array_equal(lse, again[1])


@pytest.mark.parametrize("fmt", FORMATS)
def test_decode_with_scales_of_any_kind(ctx, fmt):
    # scales that are no powers of two, blocks of zeros, and value scales far apart from block to block
    lengths = [300, 33, 64, 700]
    p, cap = _filled(lengths, 5, fmt, 12)
    rng = np.random.default_rng(13)
    own = p.ks != GUARD_SCALE
    p.ks[own] = (p.ks[own] * rng.uniform(0.3, 1.0, own.sum())).astype(np.float32)
    p.vs[own] = (p.vs[own] * np.exp2(rng.integers(-12, 13, own.sum())) * rng.uniform(0.5, 1.0, own.sum())).astype(np.float32)
    p.vs[np.flatnonzero(own)[::5]] = 0.0
    p.ks[np.flatnonzero(own)[::7]] = 0.0
    p.vs[np.flatnonzero(own)[:3]] = 0.0
    p.upload()
    q = _queries(2, 1, 8, 14)
    for scale in (128 ** -0.5, 0.5, -0.1, 0.0):
        out, lse = _decode(ctx, p, cap, lengths, q, 2, scale)
        _assert_decode(p, cap, lengths, q, 2, scale, out, lse)


@pytest.mark.parametrize("fmt", FORMATS)
def test_decode_with_scales_below_the_normal_numbers(ctx, fmt):
    lengths = [40, 100, 33, 64]
    p, cap = _filled(lengths, 5, fmt, 17)
    own = np.flatnonzero(p.ks != GUARD_SCALE)
    tiny = [1e-40, 3e-39, 2.0 ** -149, 1e-40, 0.0, 0.25, 1e-40, 2e-42, 1e-40, 2.0 ** -149]   # 2 + 4 + 2 + 2 blocks
    assert len(own) == len(tiny)
    p.vs[own] = np.float32(tiny)
    p.ks[own[::2]] = np.float32(1e-42)
    p.upload()
    q = _queries(1, 1, 8, 18)
    out, lse = _decode(ctx, p, cap, lengths, q, 4, 128 ** -0.5)
    _assert_decode(p, cap, lengths, q, 4, 128 ** -0.5, out, lse)


@pytest.mark.parametrize("fmt", FORMATS)
def test_decode_with_one_scale_of_no_power_of_two_in_many_blocks(ctx, fmt):
    """A wave with 1024 tiles, the same scale c in all of them, where c (1 / c) is 1 - 2^-24: nothing may be lost from tile to tile.
    All scores are 0 and the codes are small whole numbers, so that their sums times 2^15 are exact.  What is off: the weights,
    1 / c and its product with c and the second parts that the sums swallow, 3 * 2^-24; c and the quotient at the end, 2 * 2^-24."""
    c, n = np.float32(0.013), 32 * 1024
    assert c * (np.float32(1.0) / c) != 1
    rows = 2048 * 1024 * 32 - 32          # spare but for the first n; 2048 waves have 1024 blocks each
    codes = np.array([0x38, 0x40, 0x44, 0x48], dtype=np.uint8) if fmt == Q.E4M3 else np.array([1, 2, 3, 4], dtype=np.uint8)
    pick = np.random.default_rng(19).integers(0, 4, (n, 128))
    k, v = (torch.empty((rows, 128), dtype=torch.uint8, device="cuda") for _ in range(2))
    k[:n].zero_()
    v[:n].copy_(torch.from_numpy(codes[pick]))
    ks, vs = (torch.full((Q.scale_count(1, rows),), float(c), device="cuda") for _ in range(2))
    p = lkv.QuantRows(k.view(KINDS[fmt]), v.view(KINDS[fmt]), ks, vs)
    q = _queries(1, 1, 2, 20).cuda()
    ws = torch.empty((lkv.lkv_decode_quant_workspace_bytes(1, rows, 2, 1),), dtype=torch.uint8, device="cuda")
    out = torch.full((1, 1, 2, 128), float("nan"), device="cuda")
    lkv.lkv_decode_attn_quant(ctx, 1, 1, 1, 2, 128, q, p, i32([0, rows]), i32([n]), rows, 128 ** -0.5, out, None, ws)
    ref = (pick + 1).mean(axis=0) * float(c)
    assert np.abs(out.cpu().numpy()[0, 0] / ref - 1).max() <= 5 * 2.0 ** -24


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("ahead", [0.0, 3.0, 10.5, 14.0, 18.0])
def test_decode_of_one_large_weight_and_many_small_ones(ctx, fmt, ahead):
    """One row is `ahead` in its score and has value 0, fifty thousand have score 0 and value 1: what the output holds comes from
    weights of e^-ahead.  All terms are positive, so the sums are off by their depth: 32 rows of a tile, 4 waves, 13 and 32 pieces,
    100 * 2^-24, and a weight by 2^-20 (exp2 of an argument up to 26, 22 bits of the weight)."""
    n = 50000
    p = Packed(n, 1, fmt)
    k, v = np.zeros((n, 128)), np.ones((n, 128))
    k[77, 3], v[77] = 1.0, 0.0
    Q.write_segment(k, 0, 0, p.kc, p.ks, fmt)
    Q.write_segment(v, 0, 0, p.vc, p.vs, fmt)
    p.upload()
    q = torch.zeros((1, 1, 2, 128), dtype=torch.bfloat16)
    q[..., 3] = 1.0
    out, lse = _decode(ctx, p, [0, n], [n], q, 1, ahead)
    rest = (n - 1) * np.exp(-ahead)
    assert np.abs(out / (rest / (1 + rest)) - 1).max() <= 100 * 2.0 ** -24 + 2.0 ** -20
    assert np.abs(lse - (ahead + np.log1p(rest))).max() <= 100 * 2.0 ** -24 + 2.0 ** -20


@pytest.mark.parametrize("fmt", FORMATS)
def test_decode_reads_nothing_of_spare_rows(ctx, fmt):
    lengths = [70, 0, 31]
    p, cap = _filled(lengths, 40, fmt, 15)
    q = _queries(1, 1, 12, 16)
    out, lse = _decode(ctx, p, cap, lengths, q, 3, 0.1)
    for s, n in enumerate(lengths):
        p.kc[cap[s] + n:cap[s + 1]] = 0x7F
        p.vc[cap[s] + n:cap[s + 1]] = 0x7F
    own = {Q.scale_number(cap[s], s, i) for s, n in enumerate(lengths) for i in range(n)}
    free = [i for i in range(len(p.ks)) if i not in own]
    p.ks[free], p.vs[free] = np.nan, np.nan
    p.upload()
    again = _decode(ctx, p, cap, lengths, q, 3, 0.1)
    assert np.array_equal(out, again[0]) and np.array_equal(lse, again[1])


@pytest.mark.parametrize("fmt", FORMATS)
def test_rows_past_two_to_the_31_bytes(ctx, fmt):
    """Two segments, the second 17 million rows further on: decode, append and re-eviction reach it; and a compaction from a head
    of 9 million tokens."""
    gap = 17_000_000
    cap, lengths = np.array([0, gap, gap + 200]), np.array([70, 90])
    n = Q.scale_count(2, int(cap[-1]))
    codes = [torch.zeros((int(cap[-1]), 128), dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.zeros(n, device="cuda") for _ in range(2)]
    rows = lkv.QuantRows(codes[0].view(KINDS[fmt]), codes[1].view(KINDS[fmt]), *scales)
    small, small_cap = _filled(lengths, 110, fmt, 17)                    # the same values in a small cache
    for s, m in enumerate(lengths):
        for big, bs, sc, ss in ((codes[0], scales[0], small.kc, small.ks), (codes[1], scales[1], small.vc, small.vs)):
            big[cap[s]:cap[s] + m] = torch.from_numpy(sc[small_cap[s]:small_cap[s] + m]).cuda()
            for b in range(0, m, 32):
                bs[Q.scale_number(cap[s], s, b)] = float(ss[Q.scale_number(small_cap[s], s, b)])
    q = _queries(1, 1, 8, 18).cuda()
    d_cap, d_len, total = i32(cap), i32(lengths), int(cap[-1])
    out, lse = torch.full((8, 128), float("nan"), device="cuda"), torch.full((8,), float("nan"), device="cuda")
    ws = torch.empty(lkv.lkv_decode_quant_workspace_bytes(2, total, 8, 2), dtype=torch.uint8, device="cuda")
    lkv.lkv_decode_attn_quant(ctx, 1, 1, 2, 8, 128, q, rows, d_cap, d_len, total, 0.09, out, lse, ws)
    _assert_decode(small, small_cap, lengths, q.cpu(), 2, 0.09, out.cpu().numpy(), lse.cpu().numpy())
    new = torch.randn((2, 1, 1, 2, 128), generator=torch.Generator().manual_seed(19)).to(torch.bfloat16).cuda()
    small_len = i32(lengths)
    lkv.lkv_append_quant(ctx, 1, 1, 2, 128, new[0], new[1], rows, d_cap, d_len)
    lkv.lkv_append_quant(ctx, 1, 1, 2, 128, new[0], new[1], small.c, i32(small_cap), small_len)
    assert torch.equal(d_len, small_len)
    up = torch.zeros(total, device="cuda")
    up[cap[1]:cap[1] + 91] = torch.randn(91, generator=torch.Generator().manual_seed(20)).cuda()
    small_up = torch.zeros(small.rows, device="cuda")
    small_up[small_cap[1]:small_cap[1] + 91] = up[cap[1]:cap[1] + 91]
    got = []
    for src, u, c, ln in ((rows, up, d_cap, d_len), (small.c, small_up, i32(small_cap), small_len)):
        p = Packed(60, 2, fmt)
        u2, c2, l2, idx, off = torch.zeros(60, device="cuda"), i32([0, 0, 0]), i32([0, 0]), i32(np.zeros(60)), i32([0, 0, 0])
        lkv.lkv_reevict_quant(ctx, 128, src, u, c, ln, [71, 91], [15, 41], 2, idx, off, p.c, u2, c2, l2)
        got.append([x.clone() for x in p.dev] + [u2, c2, l2])
    assert all(torch.equal(a, b) for a, b in zip(*got))
    del rows, codes, scales, up, got
    torch.cuda.empty_cache()
    T = 9_000_000
    k = torch.zeros((1, 1, T, 128), dtype=torch.bfloat16, device="cuda")
    pick = torch.tensor([0, 5, T - 70, T - 3, T - 1])
    k[0, 0, pick] = torch.randn((5, 128), generator=torch.Generator().manual_seed(21)).to(torch.bfloat16).cuda()
    p = Packed(5, 1, fmt)
    Q.write_segment(k[0, 0, pick].double().cpu().numpy(), 0, 0, p.kc, p.ks, fmt)
    p.vc[:5], p.vs[0] = p.kc[:5], p.ks[0]
    lkv.lkv_compact_quant(ctx, lkv.Cache([k], [k], 1), pick.int().cuda(), i32([0, 5]), 5, p.c)
    p.assert_same("compact")


@pytest.mark.parametrize("fmt", FORMATS)
def test_lengths_beyond_their_segment_are_cut(ctx, fmt):
    lengths = [40, 64, 7]
    p, cap = _filled(lengths, 0, fmt, 22)
    q = _queries(1, 1, 6, 23)
    out, lse = _decode(ctx, p, cap, [40, 1000, -5], q, 3, 0.1)
    _assert_decode(p, cap, [40, 64, 0], q, 3, 0.1, out, lse)


def test_decode_of_an_empty_cache(ctx):
    p, cap = _filled([0, 0], 0, Q.E4M3, 1)
    out, lse = _decode(ctx, p, cap, [0, 0], _queries(1, 1, 2, 1), 2, 0.1)
    assert (out == 0).all() and np.isneginf(lse).all()


# ---- appending ------------------------------------------------------------------------------------


def _scorer(L, H, kind, seed, per_head=False):
    rng = np.random.default_rng(seed)
    hidden = 0 if kind == "linear" else int(kind)
    shape = (L, H if per_head else 1)
    sc = {"kind": "mlp" if hidden else "linear", "act": "gelu" if per_head else "silu", "hidden": hidden, "per_head": per_head,
          "w1": W.f32_to_bf16_bits((rng.normal(size=shape + ((hidden,) if hidden else ()) + (256,)) * 0.05).astype(np.float32)),
          "b1": (rng.normal(size=shape + ((hidden,) if hidden else ())) * 0.1).astype(np.float32),
          "w2": (rng.normal(size=shape + (hidden,))).astype(np.float32) if hidden else None,
          "b2": rng.normal(size=shape).astype(np.float32) if hidden and per_head else None}
    return sc


class Growing:
    """A packed 8-bit cache that grows, on the GPU and in the oracle."""

    def __init__(self, ctx, n_seq, L, H, lengths, slack, fmt, seed, scorer=None):
        self.ctx, self.n_seq, self.L, self.H, self.fmt = ctx, n_seq, L, H, fmt
        self.p, self.cap = _filled(lengths, slack, fmt, seed)
        self.len = np.asarray(lengths).copy()
        self.sc = scorer
        self.d_sc = None if scorer is None else G.scorer_to_gpu(scorer)
        self.up = np.random.default_rng(seed + 50).normal(size=self.p.rows).astype(np.float32)
        self.d_up, self.d_cap, self.d_len = torch.from_numpy(self.up.copy()).cuda(), i32(self.cap), i32(self.len)
        self.overflow = i32([0])

    def append(self, seed, size=1.0, rotary=None, positions=None, stream=None):
        rng = np.random.default_rng(seed)
        shape = (self.n_seq, self.L, self.H, 128)
        k, v = (bf16(rng.normal(size=shape) * size * np.exp2(rng.integers(-4, 5, shape[:3] + (1,)))) for _ in range(2))
        dk, dv, dpos = k.cuda(), v.cuda(), None if rotary is None else i32(positions)
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        lkv.lkv_append_quant(self.ctx, self.n_seq, self.L, self.H, 128, dk, dv, self.p.c, self.d_cap, self.d_len,
                             scorer=self.d_sc, up=None if self.sc is None else self.d_up, rotary=None if rotary is None else rotary["gpu"],
                             positions=dpos, overflow=self.overflow, stream=stream)
        if stream is not None:
            stream.synchronize()
        if rotary is not None:   # the rotated key in bf16 is what the rotation's own call returns
            y = torch.empty_like(dk).reshape(self.n_seq, self.L * self.H, 1, 128)
            lkv.lkv_rope(self.ctx, rotary["gpu"], dk.reshape(y.shape), y, positions=dpos.reshape(-1, 1))
            y = y.cpu().reshape(shape)
            want = R.rotate(k.double().numpy(), np.asarray(positions)[:, None, None], rotary["w"], rotary["factor"], rotary["pairs"])
            size_of = np.abs(k.double().numpy()).max(axis=-1, keepdims=True) * 2 * abs(rotary["factor"])
            assert (np.abs(y.double().numpy() - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -21 * size_of + 2.0 ** -130).all()
            k = y
        k64, v64 = k.double().numpy().reshape(-1, 128), v.double().numpy().reshape(-1, 128)
        torch.cuda.synchronize()
        got_up = self.d_up.cpu().numpy()
        full = False
        if self.sc is not None:
            u_ref = np.stack([O.score(k.double().numpy()[i][:, :, None], v.double().numpy()[i][:, :, None], G.scorer_to_oracle(self.sc))[..., 0]
                              for i in range(self.n_seq)]).reshape(-1)
        for s in range(len(self.len)):
            row = self.cap[s] + self.len[s]
            if row >= self.cap[s + 1]:
                full = True
                continue
            Q.append_row(k64[s], int(self.len[s]), int(self.cap[s]), s, self.p.kc, self.p.ks, self.fmt)
            Q.append_row(v64[s], int(self.len[s]), int(self.cap[s]), s, self.p.vc, self.p.vs, self.fmt)
            if self.sc is not None:
                assert abs(got_up[row] - u_ref[s]) <= G.SCORE_RTOL * max(abs(u_ref[s]), 0.05)
                self.up[row] = got_up[row]
            self.len[s] += 1
        self.p.assert_same("append")
        assert np.array_equal(self.d_len.cpu().numpy(), self.len) and np.array_equal(got_up, self.up)
        return full


def _rotary(r, pairs, factor=1.0, base=10000.0):
    w = base ** (-np.arange(0, r, 2) / r)
    return {"w": w, "factor": factor, "pairs": pairs, "gpu": lkv.Rotary(torch.from_numpy(w).cuda(), pairs=pairs, factor=factor)}


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("kind,per_head", [("linear", False), ("64", False), ("100", True), (None, False)])
def test_append_over_block_borders_until_full(ctx, fmt, kind, per_head):
    sc = None if kind is None else _scorer(2, 3, kind, 1, per_head)
    g = Growing(ctx, 1, 2, 3, [0, 1, 30, 31, 32, 63], 40, fmt, 31, sc)
    for i in range(40):
        assert not g.append(1000 + i, size=2.0 ** (i % 7 - 3)), i
        assert int(g.overflow.item()) == 0
    assert g.append(2000) and int(g.overflow.item()) == 1     # full: nothing is written


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("r,pairs,factor", [(128, False, 1.0), (128, True, 1.25), (96, False, 1.0), (34, True, 0.5), (2, False, 1.0)])
def test_append_with_the_rotation(ctx, fmt, r, pairs, factor):
    g = Growing(ctx, 3, 2, 2, np.arange(12) * 7, 3, fmt, 32, _scorer(2, 2, "linear", 2))
    for i, pos in enumerate([[0, 1, 2], [1000000, 77, 131071], [2 ** 31 - 1, 5, 40000]]):
        g.append(3000 + i, rotary=_rotary(r, pairs, factor), positions=pos)


@pytest.mark.parametrize("fmt", FORMATS)
def test_append_of_zeros_and_of_rows_out_of_range(ctx, fmt):
    g = Growing(ctx, 1, 1, 4, [0, 32, 5, 31], 6, fmt, 33)
    for size in (0.0, 1e-30, 0.0, 3e36, 1.0):
        g.append(4000, size=size)


def test_append_on_another_stream(ctx):
    g = Growing(ctx, 2, 5, 3, np.arange(30), 5, Q.INT8, 34, _scorer(5, 3, "16", 3))
    for i in range(3):
        g.append(5000 + i, stream=torch.cuda.Stream())


# ---- re-eviction ------------------------------------------------------------------------------------


def _reevict(g, budgets, slack):
    """Shrinks a Growing cache on both sides."""
    fmt, n_seg = g.fmt, len(g.len)
    nb = np.asarray(budgets)
    cap = np.concatenate([[0], np.cumsum(nb + slack)])
    new = Packed(int(cap[-1]), n_seg, fmt)
    up = np.full(new.rows, -3.0, dtype=np.float32)
    for s in range(n_seg):
        a, n = int(g.cap[s]), int(g.len[s])
        keep = O.select(g.up[a:a + n], int(nb[s]))
        up[cap[s]:cap[s] + len(keep)] = g.up[a:a + n][keep]
        for codes, scales, dst, dst_scales in ((g.p.kc, g.p.ks, new.kc, new.ks), (g.p.vc, g.p.vs, new.vc, new.vs)):
            Q.write_segment(Q.read_segment(codes, scales, a, s, n, fmt)[keep], int(cap[s]), s, dst, dst_scales, fmt)
    total = int(nb.sum())
    d_up, d_cap, d_len = torch.full((max(new.rows, 1),), -3.0, device="cuda"), i32(np.full(n_seg + 1, -1)), i32(np.full(n_seg, -1))
    idx, off = i32(np.full(total + 8, -9)), i32(np.full(n_seg + 1, -1))
    kept = lkv.lkv_reevict_quant(g.ctx, 128, g.p.c, g.d_up, g.d_cap, g.d_len, g.len, nb, slack, idx, off, new.c, d_up, d_cap, d_len)
    assert kept == total
    new.assert_same("re-eviction")
    g.p.assert_same("the old cache")
    assert np.array_equal(d_up.cpu().numpy()[:new.rows], up) and (idx.cpu().numpy()[total:] == -9).all()
    assert np.array_equal(d_cap.cpu().numpy(), cap) and np.array_equal(d_len.cpu().numpy(), nb)
    g.p, g.cap, g.len, g.up, g.d_up, g.d_cap, g.d_len = new, cap, nb.copy(), up, d_up, d_cap, d_len


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("slack", [0, 1, 37])
def test_reeviction(ctx, fmt, slack):
    lengths = np.array([0, 1, 31, 32, 33, 64, 100, 700])
    g = Growing(ctx, 1, 2, 4, lengths, 9, fmt, 41 + slack)
    g.up = np.round(g.up * 4).astype(np.float32) / 4            # many ties
    g.d_up.copy_(torch.from_numpy(g.up))
    _reevict(g, [0, 1, 0, 31, 33, 40, 99, 333], slack)


@pytest.mark.parametrize("fmt", FORMATS)
def test_keeping_every_row_keeps_every_value(ctx, fmt):
    g = Growing(ctx, 1, 1, 3, [64, 33, 5], 7, fmt, 51)
    before = [Q.unpack(c, s, g.cap, g.len, fmt) for c, s in ((g.p.kc, g.p.ks), (g.p.vc, g.p.vs))]
    _reevict(g, g.len, 11)
    for x, c, s in zip(before, (g.p.kc, g.p.vc), (g.p.ks, g.p.vs)):
        assert np.array_equal(x, Q.unpack(c, s, g.cap, g.len, fmt))


# ---- together, captured, refused --------------------------------------------------------------------


@pytest.mark.parametrize("fmt", FORMATS)
def test_a_sequence_from_prefill_to_a_second_eviction(ctx, fmt):
    """Scores, top-k, compaction into 8 bits, tokens generated with rotated queries and keys, decode after each, and again after the
    cache has shrunk."""
    w = W.scaled(W.CONFIGS[1], L=2, H=4, Hq=16, b_min=4, R=0.2)
    T, slack = 700, 35
    (Kb, Vb), Qb, Bu, sc = W.draw_kv(w, T, 0, 3), W.draw_q(w, 0, 3), W.draw_budgets(w, T, 0, 3), W.draw_scorer(w, 3)
    run = G.GpuRun(ctx, [Kb], [Vb], [Qb], sc, [Bu], w.Hq)
    run.score(); run.select()
    n_seg = w.L * w.H
    g = Growing(ctx, 1, w.L, w.H, np.asarray(Bu).reshape(-1), slack, fmt, 1, sc)
    lkv.lkv_compact_quant(ctx, run.cache, run.idx, run.offsets, run.total, g.p.c, slack=slack, scores=run.scores, up=g.d_up,
                          cap_offsets=g.d_cap, lengths=g.d_len)
    torch.cuda.synchronize()
    idx, off, u = run.idx.cpu().numpy(), run.offsets.cpu().numpy(), run.scores[0].cpu().numpy().reshape(n_seg, T)
    for s in range(n_seg):
        rows = idx[off[s]:off[s + 1]]
        for bits, codes, scales in ((Kb, g.p.kc, g.p.ks), (Vb, g.p.vc, g.p.vs)):
            Q.write_segment(O.bf16_bits_to_f64(bits).reshape(n_seg, T, 128)[s][rows], int(g.cap[s]), s, codes, scales, fmt)
        g.up[g.cap[s]:g.cap[s] + len(rows)] = u[s][rows]
    g.p.assert_same("compact")
    rot = _rotary(128, False)
    for step in range(slack):
        g.append(7000 + step, rotary=rot, positions=[T + step])
        if step % 9 == 0 or step == slack - 1:
            q = _queries(1, w.L, w.Hq, 8000 + step).cuda()
            lkv.lkv_rope(ctx, rot["gpu"], q.reshape(1, w.L * w.Hq, 1, 128), q.reshape(1, w.L * w.Hq, 1, 128), first_position=T + step)
            out, lse = _decode(ctx, g.p, g.cap, g.len, q.cpu(), w.H, 128 ** -0.5)
            _assert_decode(g.p, g.cap, g.len, q.cpu(), w.H, 128 ** -0.5, out, lse)
    _reevict(g, np.maximum(1, g.len * 2 // 3), 4)
    g.append(9000, rotary=rot, positions=[T + slack])
    q = _queries(1, w.L, w.Hq, 9001)
    out, lse = _decode(ctx, g.p, g.cap, g.len, q, w.H, 128 ** -0.5)
    _assert_decode(g.p, g.cap, g.len, q, w.H, 128 ** -0.5, out, lse)


@pytest.mark.parametrize("fmt", FORMATS)
def test_captured_steps_replay_to_the_eager_result(ctx, fmt):
    """Rotation of the query, append and decode in one graph, replayed with new inputs in place and eager work between."""
    lengths = np.array([5, 40, 31, 900, 0, 64])
    eager, captured = (Growing(ctx, 1, 2, 3, lengths, 8, fmt, 61, _scorer(2, 3, "linear", 6)) for _ in range(2))
    rot = _rotary(64, True)["gpu"]
    q0 = [_queries(1, 2, 12, 900 + i) for i in range(5)]
    new = [[_queries(1, 2, 3, 950 + 2 * i + j, 2.0 ** i) for j in range(2)] for i in range(5)]
    need = lkv.lkv_decode_quant_workspace_bytes(6, int(eager.cap[-1]), 12, 3)

    def buffers():
        f = dict(device="cuda")
        return {"q": torch.empty((1, 2, 12, 128), dtype=torch.bfloat16, **f), "k": torch.empty((1, 2, 3, 128), dtype=torch.bfloat16, **f),
                "v": torch.empty((1, 2, 3, 128), dtype=torch.bfloat16, **f), "pos": torch.empty(1, dtype=torch.int32, **f),
                "out": torch.empty((1, 2, 12, 128), **f), "lse": torch.empty((1, 2, 12), **f), "ws": torch.empty(need, dtype=torch.uint8, **f)}

    def step(g, b):
        x = b["q"].reshape(1, 24, 1, 128)
        lkv.lkv_rope(ctx, rot, x, x, positions=b["pos"].reshape(1, 1))
        lkv.lkv_append_quant(ctx, 1, 2, 3, 128, b["k"], b["v"], g.p.c, g.d_cap, g.d_len, scorer=g.d_sc, up=g.d_up, rotary=rot, positions=b["pos"])
        lkv.lkv_decode_attn_quant(ctx, 1, 2, 3, 12, 128, b["q"], g.p.c, g.d_cap, g.d_len, int(g.cap[-1]), 0.09, b["out"], b["lse"], b["ws"])

    def fill(b, i):
        b["q"].copy_(q0[i]); b["k"].copy_(new[i][0]); b["v"].copy_(new[i][1]); b["pos"].fill_(1000 + i)

    be, bc = buffers(), buffers()
    fill(be, 0); fill(bc, 0)
    step(eager, be); step(captured, bc)                       # also warms up
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step(captured, bc)
    torch.cuda.synchronize()
    for i in range(1, 5):
        fill(be, i); fill(bc, i)
        step(eager, be)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(be["out"], bc["out"]) and torch.equal(be["lse"], bc["lse"]), i
        assert torch.equal(eager.d_len, captured.d_len) and torch.equal(eager.d_up, captured.d_up)
        assert all(torch.equal(x, y) for x, y in zip(eager.p.dev, captured.p.dev)), i


def _refused(status, call, *args, **kw):
    with pytest.raises(lkv.LkvError) as e:
        call(*args, **kw)
    assert e.value.status == status, str(e.value)


def test_refusals(ctx):
    """Every refusal is the host's, before anything is enqueued: the caches stay as they are."""
    import ctypes as C

    g = Growing(ctx, 1, 1, 2, [5, 40], 3, Q.INT8, 71, _scorer(1, 2, "linear", 7))
    lib, p = ctx.lib, g.p.c
    z = torch.zeros((1, 1, 2, 128), dtype=torch.bfloat16, device="cuda")
    ptr = lambda t: C.c_void_p(t.data_ptr())  # noqa: E731
    sc = lkv._scorer_struct(g.d_sc)
    rot = _rotary(64, False)["gpu"]
    pos = i32([1])

    def struct(**kw):
        s = lkv._QuantRows(p.c.format, p.c.k, p.c.v, p.c.k_scale, p.c.v_scale)
        for k, v in kw.items():
            setattr(s, k, v)
        return s

    def append(want, n=(1, 1, 2), d=128, scorer=sc, up=g.d_up, rotary=None, positions=None, k=z, packed=None, cap=g.d_cap):
        st = lib.lkv_append_quant(ctx.h, *n, d, None if scorer is None else C.byref(scorer), None if rotary is None else C.byref(rotary),
                                  None if positions is None else ptr(positions), None if k is None else ptr(k), ptr(z),
                                  C.byref(packed if packed is not None else p.c), None if up is None else ptr(up), None if cap is None else ptr(cap),
                                  ptr(g.d_len), None, None)
        assert st == want, lib.lkv_last_error(ctx.h)

    bad_rotary = lambda **kw: lkv._Rotary(**{**dict(layout=0, rotary_dim=64, inv_freq=rot.c.inv_freq, factor=1.0), **kw})  # noqa: E731
    append(1, n=(0, 1, 2)); append(2, d=64); append(1, scorer=None); append(1, up=None); append(1, k=None); append(1, cap=None)
    append(1, packed=struct(format=2)); append(1, packed=struct(k=None)); append(1, packed=struct(v_scale=p.c.v_scale + 4))
    append(1, rotary=rot.c); append(1, rotary=bad_rotary(layout=2), positions=pos); append(1, rotary=bad_rotary(rotary_dim=63), positions=pos)
    append(1, rotary=bad_rotary(rotary_dim=130), positions=pos); append(1, rotary=bad_rotary(inv_freq=None), positions=pos)
    append(1, rotary=bad_rotary(factor=float("nan")), positions=pos)

    need = lkv.lkv_decode_quant_workspace_bytes(2, 51, 8, 2)
    ws, out, q = torch.empty(need + 256, dtype=torch.uint8, device="cuda"), torch.zeros((8, 128), device="cuda"), torch.zeros((8, 128), dtype=torch.bfloat16, device="cuda")

    def decode(want, n=(1, 1, 2, 8), d=128, packed=None, rows=51, scale=0.1, ws_at=ws, ws_bytes=need, query=q):
        st = lib.lkv_decode_attn_quant(ctx.h, *n, d, None if query is None else ptr(query), C.byref(packed if packed is not None else p.c), ptr(g.d_cap),
                                       ptr(g.d_len), rows, scale, ptr(out), None, ptr(ws_at), ws_bytes, None)
        assert st == want, lib.lkv_last_error(ctx.h)

    decode(1, n=(1, 1, 0, 8)); decode(1, n=(1, 1, 2, 7)); decode(2, n=(1, 1, 2, 34)); decode(2, d=64); decode(1, rows=-1); decode(1, rows=1 << 31)
    decode(1, scale=float("nan")); decode(1, scale=float("inf")); decode(3, ws_bytes=need - 1); decode(3, ws_at=ws[16:]); decode(1, query=None)
    decode(1, packed=struct(format=-1)); decode(1, packed=struct(v=None)); decode(2, n=(1 << 10, 1 << 10, 2, 8))

    cache = lkv.Cache([torch.zeros((1, 2, 30, 128), dtype=torch.bfloat16, device="cuda")] * 1, [torch.zeros((1, 2, 30, 128), dtype=torch.bfloat16, device="cuda")], 2)
    idx, off = i32(np.arange(10)), i32([0, 5, 10])
    for kw in (dict(slack=-1), dict(slack=2), dict(up=g.d_up), dict(cap_offsets=g.d_cap), dict(lengths=g.d_len)):
        st = lib.lkv_compact_quant(ctx.h, C.byref(cache.c), None, ptr(idx), ptr(off), 10, kw.get("slack", 0), C.byref(p.c),
                                   *[None if kw.get(n) is None else ptr(kw[n]) for n in ("up", "cap_offsets", "lengths")], None)
        assert st == 1, kw
    for args in ((ptr(idx), ptr(off), -1), (ptr(idx), ptr(off), 1 << 31), (None, ptr(off), 10), (ptr(idx), None, 10)):
        assert lib.lkv_compact_quant(ctx.h, C.byref(cache.c), None, *args, 0, C.byref(p.c), None, None, None, None) == 1
    with pytest.raises(AssertionError):                        # a cache too small for the rows
        lkv.lkv_compact_quant(ctx, cache, idx, off, 5000, p)

    other = Packed(60, 2, Q.E4M3)
    args = (128, p, g.d_up, g.d_cap, g.d_len)
    tail = (i32(np.zeros(60)), i32([0, 0, 0]), other.c, g.d_up, i32([0, 0, 0]), i32([0, 0]))
    _refused(2, lkv.lkv_reevict_quant, ctx, *args, [5, 40], [2, 3], 1, *tail)            # another format
    same = Packed(60, 2, Q.INT8)
    tail = tail[:2] + (same.c,) + tail[3:]
    _refused(1, lkv.lkv_reevict_quant, ctx, *args, [5, 40], [6, 3], 1, *tail)
    _refused(1, lkv.lkv_reevict_quant, ctx, *args, [5, 40], [-1, 3], 1, *tail)
    _refused(1, lkv.lkv_reevict_quant, ctx, *args, [5, -1], [0, 0], 1, *tail)
    _refused(1, lkv.lkv_reevict_quant, ctx, *args, [5, 40], [2, 3], -1, *tail)
    _refused(2, lkv.lkv_reevict_quant, ctx, 64, *args[1:], [5, 40], [2, 3], 1, *tail)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):              # uploads host tables: refused while the stream is captured
            _refused(2, lkv.lkv_reevict_quant, ctx, *args, [5, 40], [2, 3], 1, *tail)
            tail[0].add_(0)                                     # a graph with something in it
    torch.cuda.synchronize()
    g.p.assert_same("after the refusals")
    same.assert_same("after the refusals")
    assert np.array_equal(g.d_len.cpu().numpy(), g.len)
