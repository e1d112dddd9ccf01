"""The 8-bit packed cache and the rotary positions: what is measured of them, and their plain forms.

Each case is one pass through one operator:

* ``rope``     rotary positions of queries, keys or their gradients,
* ``compact``  the kept rows of a prefilled bf16 cache gathered into the packed cache in 8 bits,
* ``append``   one generated token per segment joins a packed 8-bit cache, its key rotated on the way,
* ``decode``   one decode step of grouped-query attention over a packed 8-bit cache,
* ``reevict``  a packed 8-bit cache shrunk to smaller budgets.

The packed cache in 8 bits holds e4m3 or int8 codes, one fp32 scale for every 32 rows of a segment and for K and V each.
A scale is the smallest power of two that brings the block's largest magnitude to at most 448 (e4m3) or 127 (int8), at
least 2^-126, and 0 for a block of zeros; a code is the value over the scale, rounded to nearest even.  Block b of segment
s, whose rows start at row cap[s], has scale number cap[s] // 32 + s + b.

Caches come back as their codes (e4m3 numbers, or whole numbers) in units of the scales that come back beside them.
"""
import math

import numpy as np
import torch

own = False

D = 128
BLOCK = 32
SCALE = 1.0 / math.sqrt(D)
_DEVICE = "cuda:0"
_ctx = None


def listed():
    return [
        # one layer's query heads of four sequences at one decode step, far positions: a launch and its latency
        {"name": "rope-step", "op": "rope", "B": 4, "heads": 32, "T": 1, "f32": False, "pairs": False, "rotary_dim": 128,
         "stretch": 8.0, "far": 1 << 20, "backward": False},
        # one layer's queries of a long training sample
        {"name": "rope-16k", "op": "rope", "B": 1, "heads": 32, "T": 16384, "f32": False, "pairs": False, "rotary_dim": 128,
         "stretch": 1.0, "far": 0, "backward": False},
        # the gradient of the queries of an odd sample, fp32 as the attention's backward pass leaves it, half the head rotated
        {"name": "rope-grad-8191", "op": "rope", "B": 1, "heads": 28, "T": 8191, "f32": True, "pairs": True, "rotary_dim": 64,
         "stretch": 4.0, "far": 0, "backward": True},
        # all layers of a 32k prompt, 15 % kept, packed without spare rows
        {"name": "compact-32k-e4m3", "op": "compact", "n_seq": 1, "L": 32, "H": 8, "T": 32768, "R": 0.15, "int8": False,
         "slack": 0},
        # a few layers of a batch of odd lengths, spare rows behind every segment
        {"name": "compact-ragged-int8", "op": "compact", "n_seq": 4, "L": 8, "H": 8, "T": 9001, "R": 0.15, "int8": True,
         "slack": 67},
        # a generated token of one sequence joins all layers and heads
        {"name": "append-256", "op": "append", "n_seq": 1, "L": 32, "H": 8, "rows": 700, "slack": 128, "int8": False,
         "hidden": 0, "pairs": False, "rotary_dim": 128},
        # the same for a batch, MLP scorer, part of the head rotated
        {"name": "append-batch", "op": "append", "n_seq": 16, "L": 28, "H": 4, "rows": 333, "slack": 40, "int8": True,
         "hidden": 64, "pairs": True, "rotary_dim": 96},
        # one layer of one decode step on a short prompt
        {"name": "decode-layer-4k", "op": "decode", "n_seq": 1, "L": 1, "H": 8, "G": 4, "rows": 614, "int8": False,
         "slack": 0},
        # all layers of a 32k prompt
        {"name": "decode-32k-e4m3", "op": "decode", "n_seq": 1, "L": 32, "H": 8, "G": 4, "rows": 4915, "int8": False,
         "slack": 0},
        # all layers of a batch that has generated tokens, seven query heads to a KV head
        {"name": "decode-batch-int8", "op": "decode", "n_seq": 8, "L": 28, "H": 4, "G": 7, "rows": 3276, "int8": True,
         "slack": 64},
        # all layers of a 32k prompt's cache shrink when their spare rows are used up
        {"name": "reevict-32k-e4m3", "op": "reevict", "n_seq": 1, "L": 32, "H": 8, "rows": 4915, "keep": 0.8, "slack": 128,
         "int8": False},
        # one layer of a batch, most rows dropped
        {"name": "reevict-layer-int8", "op": "reevict", "n_seq": 16, "L": 1, "H": 4, "rows": 901, "keep": 0.35, "slack": 33,
         "int8": True},
    ]


def _log_int(rng, lo, hi):
    """A whole number in [lo, hi], spread over its logarithm; odd in half of the draws."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 0.5:
        v |= 1
    return max(lo, min(hi, v))


def draw(rng):
    op = rng.choice(["rope", "rope", "compact", "append", "decode", "decode", "reevict"])
    H, G = rng.choice([(8, 4), (8, 4), (4, 7), (2, 8), (8, 1), (1, 16)])
    n_seq, L, int8 = rng.choice([1, 1, 2, 8, 16]), rng.choice([1, 1, 8, 28, 32]), rng.random() < 0.5
    segments = n_seq * L * H
    if op == "rope":
        B, heads = rng.choice([1, 1, 4, 16]), rng.choice([1, 4, 8, 28, 32])
        return {"op": op, "B": B, "heads": heads, "T": _log_int(rng, 1, max(1, (32 * 16384) // (B * heads * 2))),
                "f32": rng.random() < 0.4, "pairs": rng.random() < 0.5, "rotary_dim": rng.choice([128, 128, 96, 64, 34, 2]),
                "stretch": rng.choice([1.0, 1.0, 4.0, 32.0]), "far": rng.choice([0, 0, 1 << 20]), "backward": rng.random() < 0.5}
    if op == "compact":
        R = rng.choice([0.05, 0.1, 0.15, 0.5])
        return {"op": op, "n_seq": n_seq, "L": L, "H": H,
                "T": _log_int(rng, 64, max(128, min(131072, int(256 * 32768 * min(1.0, 0.125 / R)) // segments))), "R": R, "int8": int8,
                "slack": rng.choice([0, 0, 1, 64])}
    if op == "append":
        return {"op": op, "n_seq": n_seq, "L": L, "H": H, "rows": _log_int(rng, 1, max(2, min(8192, (1 << 20) // segments))),
                "slack": rng.choice([1, 33, 128]), "int8": int8, "hidden": rng.choice([0, 64, 128]), "pairs": rng.random() < 0.5,
                "rotary_dim": rng.choice([128, 128, 96, 64, 2])}
    if op == "decode":
        return {"op": op, "n_seq": n_seq, "L": L, "H": H, "G": G, "rows": _log_int(rng, 8, max(16, min(65536, (5 << 18) // segments))),
                "int8": int8, "slack": rng.choice([0, 0, 17, 128])}
    return {"op": op, "n_seq": n_seq, "L": L, "H": H, "rows": _log_int(rng, 8, max(16, min(32768, (1 << 20) // segments))),
            "keep": rng.choice([0.1, 0.5, 0.8, 1.0]), "slack": rng.choice([0, 17, 128]), "int8": int8}


# ---- inputs -------------------------------------------------------------------------------------


def _gen(seed, tag):
    g = torch.Generator(device=_DEVICE)
    g.manual_seed(int(seed) * 64 + tag)
    return g


def _normal(shape, seed, tag, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device=_DEVICE).normal_(generator=_gen(seed, tag))


def _uniform(shape, seed, tag):
    return torch.rand(shape, dtype=torch.float32, device=_DEVICE, generator=_gen(seed, tag))


def _ints(values):
    return torch.as_tensor(np.asarray(values), dtype=torch.int32, device=_DEVICE)


def _seq_lengths(case):
    """Prompt lengths: fixed by the case, so that every seed is the same amount of work."""
    return [case["T"] - (case["T"] // 2) * i // case["n_seq"] - (i * 13) % 29 for i in range(case["n_seq"])]


def _skewed(n, mean, least, most, seed):
    """n whole numbers in [least, most] of about this mean, unevenly spread as budgets are; the seed turns their order only."""
    share = np.random.default_rng([n, int(mean)]).exponential(1.0, n) ** 1.5
    v = np.clip(np.floor(share * (mean / share.mean())), least, most).astype(np.int64)
    return np.roll(v, int(seed))


def _kept_rows(budgets, T, seed, tag):
    """Ascending row numbers, budgets[s] of the T of every segment."""
    b = torch.as_tensor(budgets, device=_DEVICE)
    order = _uniform((len(budgets), T), seed, tag).argsort(dim=1)
    keep = torch.zeros((len(budgets), T), dtype=torch.bool, device=_DEVICE)
    keep.scatter_(1, order, torch.arange(T, device=_DEVICE)[None, :] < b[:, None])
    return keep.nonzero()[:, 1].to(torch.int32)


def _outliers(x, seed, tag):
    """A few channels ten times as large, as keys have them."""
    x[..., torch.randint(0, D, (2,), generator=_gen(seed, tag), device=_DEVICE)] *= 10.0
    return x


def _frequencies(case):
    """Radians per position of every pair, fp64: base 500000, stretched evenly."""
    i = torch.arange(0, case["rotary_dim"], 2, dtype=torch.float64, device=_DEVICE)
    return 500000.0 ** (-i / case["rotary_dim"]) / case.get("stretch", 1.0)


def _cache_tensors(rows, slots, int8):
    """Codes of K and V and their scales, all zero."""
    kind = torch.int8 if int8 else torch.float8_e4m3fn
    new = lambda: torch.zeros((rows, D), dtype=torch.int8, device=_DEVICE).view(kind)  # noqa: E731
    s = lambda: torch.zeros(slots, dtype=torch.float32, device=_DEVICE)  # noqa: E731
    return {"k": new(), "v": new(), "k_scale": s(), "v_scale": s()}


def _filled_cache(s, lengths, slack, seed, tag):
    """A packed cache with these rows in use, as earlier steps have left it."""
    case = s["case"]
    cap = np.concatenate([[0], np.cumsum(lengths + slack)])
    s["cap"], s["lengths"], s["rows"] = _ints(cap), _ints(lengths), int(cap[-1])
    slots = s["rows"] // BLOCK + len(lengths)
    s.update(_cache_tensors(s["rows"], slots, case["int8"]))
    for i, name in enumerate(("k", "v")):
        x = _normal((s["rows"], D), seed, tag + i)
        x = _outliers(x, seed, tag + 8) if i == 0 else x
        _write_blocks(x.float(), s["cap"], s["lengths"], s[name], s[name + "_scale"])


def prepare(case, seed):
    s = {"op": case["op"], "case": case, "int8": bool(case.get("int8"))}
    f32 = dict(dtype=torch.float32, device=_DEVICE)
    if case["op"] == "rope":
        kind = torch.float32 if case["f32"] else torch.bfloat16
        shape = (case["B"], case["heads"], case["T"], D)
        s["x"], s["y"] = _normal(shape, seed, 0, kind), torch.empty(shape, dtype=kind, device=_DEVICE)
        first = torch.randint(0, case["far"] + 1, (case["B"], 1), generator=_gen(seed, 1), device=_DEVICE)
        s["positions"] = (first + torch.arange(case["T"], device=_DEVICE)).to(torch.int32)
        s["inv_freq"], s["factor"] = _frequencies(case), 1.0 + 0.1 * math.log(case["stretch"])
        return s
    segments = case["n_seq"] * case["L"] * case["H"]
    per_seq = case["L"] * case["H"]
    if case["op"] == "compact":
        lens = _seq_lengths(case)
        budgets = [_skewed(per_seq, case["R"] * T, min(T, 8), T, seed) for T in lens]
        s["kv"] = [tuple(_outliers(_normal((case["L"], case["H"], T, D), seed, 4 * i + j), seed, 60 + j) if j == 0 else
                         _normal((case["L"], case["H"], T, D), seed, 4 * i + j) for j in (0, 1)) for i, T in enumerate(lens)]
        s["idx"] = torch.cat([_kept_rows(b, T, seed, 4 * i + 2) for i, (b, T) in enumerate(zip(budgets, lens))])
        offsets = np.concatenate([[0], np.cumsum(np.concatenate(budgets))])
        s["offsets"], s["total"] = _ints(offsets), int(offsets[-1])
        rows = s["total"] + segments * case["slack"]
        s.update(_cache_tensors(rows, rows // BLOCK + segments, case["int8"]))
        if case["slack"]:
            s["scores"] = [_normal((case["L"], case["H"], T), seed, 4 * i + 3, torch.float32) for i, T in enumerate(lens)]
            s["up"] = torch.zeros(rows, **f32)
            s["cap"] = torch.empty(segments + 1, dtype=torch.int32, device=_DEVICE)
            s["lengths"] = torch.empty(segments, dtype=torch.int32, device=_DEVICE)
        return s
    held = _skewed(segments, case["rows"], 1, 64 * case["rows"], seed)
    _filled_cache(s, held, case["slack"], seed, 0)
    if case["op"] == "decode":
        s["q"] = _normal((case["n_seq"], case["L"], case["H"] * case["G"], D), seed, 20)
        s["out"] = torch.empty((case["n_seq"], case["L"], case["H"] * case["G"], D), **f32)
        s["lse"] = torch.empty((case["n_seq"], case["L"], case["H"] * case["G"]), **f32)
        return s
    s["up"] = _normal((s["rows"],), seed, 21, torch.float32)
    s["up"][::7] = (s["up"][::7] * 8).round() / 8                      # ties
    if case["op"] == "append":
        shape = (case["n_seq"], case["L"], case["H"], D)
        s["k_new"], s["v_new"] = _outliers(_normal(shape, seed, 22), seed, 23), _normal(shape, seed, 24)
        s["positions"] = torch.randint(1, 1 << 17, (case["n_seq"],), generator=_gen(seed, 25), device=_DEVICE).to(torch.int32)
        s["inv_freq"], s["factor"] = _frequencies(case), 1.0
        hidden = case["hidden"]
        w1 = _normal((case["L"], 1, max(hidden, 1), 2 * D), seed, 26, torch.float32) * 0.02
        s["scorer"] = {"kind": "mlp" if hidden else "linear", "act": "silu", "hidden": hidden, "per_head": False,
                       "w1": w1.to(torch.bfloat16), "b1": _normal((case["L"], 1, max(hidden, 1)), seed, 27, torch.float32) * 0.02,
                       "w2": _normal((case["L"], 1, hidden), seed, 28, torch.float32) * 0.02 if hidden else None, "b2": None}
        s["lengths_before"] = s["lengths"].clone()
        return s
    s["held"] = held.astype(np.int32)                                   # the caller's own count of the rows in use
    s["budgets"] = np.maximum(1, np.floor(held * case["keep"])).astype(np.int32)
    s["total"] = int(s["budgets"].sum())
    rows = s["total"] + segments * case["slack"]
    s["new"] = {**_cache_tensors(rows, rows // BLOCK + segments, case["int8"]), "up": torch.zeros(rows, **f32),
                "cap": torch.empty(segments + 1, dtype=torch.int32, device=_DEVICE),
                "lengths": torch.empty(segments, dtype=torch.int32, device=_DEVICE)}
    s["idx"] = torch.empty(s["total"], dtype=torch.int32, device=_DEVICE)
    s["offsets"] = torch.empty(segments + 1, dtype=torch.int32, device=_DEVICE)
    return s


# ---- plain forms --------------------------------------------------------------------------------


def _power_scale(top, int8):
    """The smallest power of two s with top <= 448 s or 127 s, at least 2^-126; 0 where top is 0."""
    m, e = torch.frexp(top)                             # top = m 2^e, 1/2 <= m < 1
    k = (e - 7) + (m > 127 / 128) if int8 else (e - 9) + (m > 448 / 512)
    return torch.where(top > 0, ((k.clamp(min=-126) + 127) << 23).view(torch.float32), 0.0)


def _codes(x, scale, int8):
    y = x * torch.where(scale > 0, 1.0 / scale, 0.0)
    return y.round().to(torch.int8) if int8 else y.to(torch.float8_e4m3fn).view(torch.int8)


def _blocks(cap, lengths, rows):
    """Of every scale number: its segment, its 32 rows and which of them are in use."""
    cap, lengths = cap.long(), lengths.long()
    first = cap[:-1] // BLOCK + torch.arange(lengths.numel(), device=_DEVICE)
    number = torch.arange(rows // BLOCK + lengths.numel(), device=_DEVICE)
    seg = (torch.searchsorted(first, number, right=True) - 1).clamp(min=0)
    at = (number - first[seg])[:, None] * BLOCK + torch.arange(BLOCK, device=_DEVICE)
    used = at < lengths[seg][:, None]
    return seg, (cap[seg][:, None] + at).clamp(max=max(rows - 1, 0)), used


def _write_blocks(x, cap, lengths, codes, scales):
    """Quantises the fp32 rows x in use into codes and scales; other rows and scales stay."""
    int8 = codes.dtype == torch.int8
    seg, rows, used = _blocks(cap, lengths, x.shape[0])
    top = torch.where(used, x.abs().amax(dim=1)[rows], 0.0).amax(dim=1)
    s = _power_scale(top, int8)
    scales.copy_(torch.where(used.any(dim=1), s, scales))
    of_row = torch.zeros(x.shape[0] + 1, dtype=torch.float32, device=_DEVICE)
    row_used = torch.zeros(x.shape[0] + 1, dtype=torch.bool, device=_DEVICE)
    at = torch.where(used, rows, x.shape[0]).reshape(-1)
    of_row[at] = s[:, None].expand(-1, BLOCK).reshape(-1)
    row_used[at] = True
    flat = codes.view(torch.int8)
    flat.copy_(torch.where(row_used[:-1, None], _codes(x, of_row[:-1, None], int8), flat))


def _rotate(x, positions, s, backward):
    """x [B, heads, T, 128] in fp32, positions [B, T]; angles in fp64."""
    angle = positions.double()[:, None, :, None] * s["inv_freq"]
    c, n = (torch.cos(angle) * s["factor"]).float(), (torch.sin(angle) * s["factor"]).float()
    n = -n if backward else n
    r = s["case"]["rotary_dim"]
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if s["case"]["pairs"] else (x[..., :r // 2], x[..., r // 2:r])
    y, z = a * c - b * n, b * c + a * n
    turned = torch.stack((y, z), dim=-1).flatten(-2) if s["case"]["pairs"] else torch.cat((y, z), dim=-1)
    return torch.cat((turned, x[..., r:]), dim=-1)


def _plain_rope(s):
    s["y"].copy_(_rotate(s["x"].float(), s["positions"], s, s["case"]["backward"]))
    return s["y"]


def _plain_compact(s):
    case, slack = s["case"], s["case"]["slack"]
    o = s["offsets"].long()
    n = o.numel() - 1
    per_seq = case["L"] * case["H"]
    seg = torch.searchsorted(o, torch.arange(s["total"], device=_DEVICE), right=True) - 1
    cap, lengths = o + slack * torch.arange(n + 1, device=_DEVICE), o[1:] - o[:-1]
    lens = torch.as_tensor(_seq_lengths(case), device=_DEVICE)
    start = torch.cumsum(lens, 0) - lens                # of each sequence's rows in the joined caches below
    q = seg // per_seq
    src = start[q] * per_seq + (seg % per_seq) * lens[q] + s["idx"].long()
    dst = torch.arange(s["total"], device=_DEVICE) + slack * seg
    for i, name in enumerate(("k", "v")):
        whole = s["kv"][0][i].reshape(-1, D) if case["n_seq"] == 1 else torch.cat([kv[i].reshape(-1, D) for kv in s["kv"]])
        x = torch.zeros(s[name].shape, dtype=torch.float32, device=_DEVICE)
        x[dst] = whole[src].float()
        _write_blocks(x, cap, lengths, s[name], s[name + "_scale"])
    if slack:
        s["up"][dst] = torch.cat([u.reshape(-1) for u in s["scores"]])[src]
        s["cap"].copy_(cap)
        s["lengths"].copy_(lengths)
    return _compacted(s)


def _compacted(s):
    return {name: s[name] for name in ("k", "v", "k_scale", "v_scale", "up", "cap", "lengths") if name in s}


def _plain_append(s):
    case = s["case"]
    n_seq, per_seq, L, H = case["n_seq"], case["L"] * case["H"], case["L"], case["H"]
    # the step of the same cache each time
    s["lengths"].copy_(s["lengths_before"])
    k = _rotate(s["k_new"].float().reshape(n_seq, per_seq, 1, D), s["positions"][:, None], s, False)
    k = k.to(torch.bfloat16).float().reshape(-1, D)
    v = s["v_new"].float().reshape(-1, D)
    sc = s["scorer"]
    x = torch.cat((k, v), dim=1).reshape(n_seq, L, H, 2 * D)
    z = (x[:, :, :, None, :] * sc["w1"].float()[None]).sum(-1) + sc["b1"][None]           # [n_seq, L, H, hidden]
    u = z[..., 0] if not case["hidden"] else (z * torch.sigmoid(z) * sc["w2"][None]).sum(-1)
    cap, used = s["cap"].long(), s["lengths"].long()
    number = torch.arange(used.numel(), device=_DEVICE)
    row, inside = cap[:-1] + used, used % BLOCK
    slot = cap[:-1] // BLOCK + number + used // BLOCK
    at = torch.arange(BLOCK, device=_DEVICE)[None, :]
    held = at < inside[:, None]
    rows = torch.where(held, (row - inside)[:, None] + at, row[:, None])                 # the others: the new row again
    for name, new in (("k", k), ("v", v)):
        int8, flat, scales = s["int8"], s[name].view(torch.int8), s[name + "_scale"]
        old = torch.where(inside > 0, scales[slot], 0.0)
        scale = torch.maximum(old, _power_scale(new.abs().amax(dim=1), int8))
        values = flat[rows].view(s[name].dtype).float() * old[:, None, None]
        values = torch.where(held[:, :, None], values, new[:, None, :])
        scales[slot] = scale
        flat[rows] = _codes(values, scale[:, None, None], int8)
    s["up"][row] = u.reshape(-1)
    s["lengths"] += 1
    return _appended(s)


def _appended(s):
    return {name: s[name] for name in ("k", "v", "k_scale", "v_scale", "up", "lengths")}


def _plain_decode(s):
    case = s["case"]
    n, G = s["lengths"].numel(), case["G"]
    seg, rows, used = _blocks(s["cap"], s["lengths"], s["rows"])
    k = s["k"].view(torch.int8)[rows].view(s["k"].dtype).float() * s["k_scale"][:, None, None]
    v = s["v"].view(torch.int8)[rows].view(s["v"].dtype).float() * s["v_scale"][:, None, None]
    q = s["q"].float().reshape(n, G, D)[seg].transpose(1, 2).contiguous()
    logits = torch.where(used[:, :, None], torch.bmm(k, q) * SCALE, -math.inf)           # [slots, 32, G]
    top = torch.full((n, G), -math.inf, device=_DEVICE).index_reduce_(0, seg, logits.amax(dim=1), "amax")
    ref = torch.where(top > -math.inf, top, 0.0)
    p = torch.exp(logits - ref[seg][:, None, :])
    den = torch.zeros((n, G), dtype=torch.float64, device=_DEVICE).index_add_(0, seg, p.sum(dim=1).double())
    part = torch.bmm(p.transpose(1, 2).contiguous(), v)                                   # [slots, G, 128]
    num = torch.zeros((n, G, D), dtype=torch.float64, device=_DEVICE).index_add_(0, seg, part.double())
    s["out"].copy_(torch.where(den[..., None] > 0, num / den[..., None], 0.0).reshape(s["out"].shape))
    s["lse"].copy_((ref.double() + torch.log(den)).reshape(s["lse"].shape))
    return {"out": s["out"], "lse": s["lse"]}


def _plain_reevict(s):
    case, new, total = s["case"], s["new"], s["total"]
    n, slack = s["lengths"].numel(), case["slack"]
    b = torch.as_tensor(s["budgets"], device=_DEVICE).long()
    cap, held = s["cap"].long(), s["lengths"].long()
    o = torch.cat((torch.zeros(1, dtype=torch.int64, device=_DEVICE), torch.cumsum(b, 0)))
    most = int(s["held"].max())
    at = torch.arange(most, device=_DEVICE)[None, :]
    inside = at < held[:, None]
    score = torch.where(inside, s["up"][(cap[:-1, None] + at).clamp(max=s["rows"] - 1)], -math.inf)
    order = torch.argsort(score, dim=1, descending=True, stable=True)                     # ties: the earlier row
    keep = torch.zeros((n, most), dtype=torch.bool, device=_DEVICE).scatter_(1, order, (at < b[:, None]).expand(n, most))
    place = torch.where(keep.reshape(-1), torch.cumsum(keep.reshape(-1), 0) - 1, total)
    src = torch.zeros(total + 1, dtype=torch.int64, device=_DEVICE).scatter_(0, place, (cap[:-1, None] + at).reshape(-1))[:total]
    seg = torch.searchsorted(o, torch.arange(total, device=_DEVICE), right=True) - 1
    dst = torch.arange(total, device=_DEVICE) + slack * seg
    new["cap"].copy_(o + slack * torch.arange(n + 1, device=_DEVICE))
    new["lengths"].copy_(b)
    slot = cap[seg] // BLOCK + seg + (src - cap[seg]) // BLOCK
    for name in ("k", "v"):
        x = torch.zeros(new[name].shape, dtype=torch.float32, device=_DEVICE)
        x[dst] = s[name].view(torch.int8)[src].view(s[name].dtype).float() * s[name + "_scale"][slot][:, None]
        _write_blocks(x, new["cap"], new["lengths"], new[name], new[name + "_scale"])
    new["up"][dst] = s["up"][src]
    return {**new, "total": total}


_PLAIN = {"rope": _plain_rope, "compact": _plain_compact, "append": _plain_append, "decode": _plain_decode,
          "reevict": _plain_reevict}


# ---- the framework's calls ------------------------------------------------------------------------


def _context(lkv):
    """The process's library context (a program makes one and keeps it)."""
    global _ctx
    if _ctx is None:
        _ctx = lkv.Context(0)
    return _ctx


def _own(s):
    from paper_2605_06676_amd import lkv

    ctx, case, op = _context(lkv), s["case"], s["op"]
    if op == "rope":
        rotary = lkv.Rotary(s["inv_freq"], pairs=case["pairs"], factor=s["factor"])
        lkv.lkv_rope(ctx, rotary, s["x"], s["y"], positions=s["positions"], backward=case["backward"])
        return s["y"]
    packed = lkv.QuantRows(s["k"], s["v"], s["k_scale"], s["v_scale"])
    if op == "compact":
        cache = lkv.Cache([k for k, _ in s["kv"]], [v for _, v in s["kv"]], case["H"])
        lkv.lkv_compact_quant(ctx, cache, s["idx"], s["offsets"], s["total"], packed, slack=case["slack"], scores=s.get("scores"),
                              up=s.get("up"), cap_offsets=s.get("cap"), lengths=s.get("lengths"))
        return _compacted(s)
    if op == "append":
        s["lengths"].copy_(s["lengths_before"])
        rotary = lkv.Rotary(s["inv_freq"], pairs=case["pairs"], factor=s["factor"])
        lkv.lkv_append_quant(ctx, case["n_seq"], case["L"], case["H"], D, s["k_new"], s["v_new"], packed, s["cap"], s["lengths"],
                             scorer=s["scorer"], up=s["up"], rotary=rotary, positions=s["positions"])
        return _appended(s)
    if op == "decode":
        if "ws" not in s:
            need = lkv.lkv_decode_quant_workspace_bytes(s["lengths"].numel(), s["rows"], case["H"] * case["G"], case["H"])
            s["ws"] = torch.empty(need, dtype=torch.uint8, device=_DEVICE)
        lkv.lkv_decode_attn_quant(ctx, case["n_seq"], case["L"], case["H"], case["H"] * case["G"], D, s["q"], packed, s["cap"],
                                  s["lengths"], s["rows"], SCALE, s["out"], s["lse"], s["ws"])
        return {"out": s["out"], "lse": s["lse"]}
    new = s["new"]
    fresh = lkv.QuantRows(new["k"], new["v"], new["k_scale"], new["v_scale"])
    total = lkv.lkv_reevict_quant(ctx, D, packed, s["up"], s["cap"], s["lengths"], s["held"], s["budgets"], case["slack"], s["idx"],
                                  s["offsets"], fresh, new["up"], new["cap"], new["lengths"])
    return {**new, "total": total}


def run(s):
    return _own(s) if own else _PLAIN[s["op"]](s)


def work(case):
    op = case["op"]
    if op == "rope":
        n = case["B"] * case["heads"] * case["T"]
        return {"bytes": n * D * (8 if case["f32"] else 4) + case["B"] * case["T"] * 4, "flops": 3 * n * case["rotary_dim"]}
    segments = case["n_seq"] * case["L"] * case["H"]
    block = 8 / BLOCK                                    # bytes of scales to a row
    if op == "compact":
        per_seq = case["L"] * case["H"]
        kept = sum(int(_skewed(per_seq, case["R"] * T, min(T, 8), T, 0).sum()) for T in _seq_lengths(case))
        return {"bytes": kept * (4 * D + 2 * D + block + 4 + (8 if case["slack"] else 0)), "flops": 4 * kept * D}
    if op == "append":
        weights = case["L"] * max(case["hidden"], 1) * 2 * D * 2
        return {"bytes": segments * (4 * D + 2 * D + 8 + 16) + weights, "flops": 4 * segments * D * max(case["hidden"], 1)}
    held = _skewed(segments, case["rows"], 1, 64 * case["rows"], 0)
    if op == "decode":
        rows = int(held.sum())
        return {"bytes": rows * (2 * D + block) + segments * case["G"] * D * 6, "flops": 4 * rows * case["G"] * D}
    kept = int(np.maximum(1, np.floor(held * case["keep"])).sum())
    return {"bytes": int(held.sum()) * 4 + kept * (4 * D + 2 * block + 8), "flops": 4 * kept * D}


# ---- the definitions in 64 bits -------------------------------------------------------------------


def _nearest(x, int8):
    """x rounded to the nearest whole number, or to the nearest e4m3 number (four significant bits, steps of 2^-9 below 2^-6)."""
    if int8:
        return torch.round(x)
    _, e = torch.frexp(x)
    step = (((e - 4).clamp(min=-9).long() + 1023) << 52).view(torch.float64)
    return torch.round(x / step) * step


def _scale_64(top, int8):
    most = 127.0 if int8 else 448.0
    if not top > 0:
        return 0.0
    k = max(-126, math.floor(math.log2(top / most)) - 1)
    while math.ldexp(most, k) < top:
        k += 1
    return math.ldexp(1.0, k)


def _quantised_64(blocks, int8):
    """A list of [n, 128] fp64 blocks: their codes and scales."""
    tops = torch.stack([b.abs().max() for b in blocks]).tolist()
    scales = [_scale_64(t, int8) for t in tops]
    return [_nearest(b / t, int8) if t else torch.zeros_like(b) for b, t in zip(blocks, scales)], scales


def _segment_blocks(x, number0, codes, scales, row0, int8):
    """Writes the quantised rows x of one segment behind row row0, scales from number0 on."""
    parts = list(x.split(BLOCK))
    if parts:
        q, t = _quantised_64(parts, int8)
        codes[row0:row0 + x.shape[0]] = torch.cat(q)
        scales[number0:number0 + len(t)] = torch.tensor(t, dtype=torch.float64, device=x.device)


def _exact_rope(s):
    case, r = s["case"], s["case"]["rotary_dim"]
    x = s["x"].double()
    y = x.clone()
    angle = s["positions"].double()[:, None, :] * 1.0
    for i in range(r // 2):
        a, b = (2 * i, 2 * i + 1) if case["pairs"] else (i, r // 2 + i)
        c, n = torch.cos(angle * s["inv_freq"][i]) * s["factor"], torch.sin(angle * s["inv_freq"][i]) * s["factor"]
        n = -n if case["backward"] else n
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * n, x[..., a] * n + x[..., b] * c
    return y


def _exact_compact(s):
    case, slack, int8 = s["case"], s["case"]["slack"], s["int8"]
    o, idx = s["offsets"].tolist(), s["idx"].long()
    f = dict(dtype=torch.float64, device=_DEVICE)
    got = {n: torch.zeros(s[n].shape, **f) for n in ("k", "v", "k_scale", "v_scale", *(["up"] if slack else []))}
    per_seq = case["L"] * case["H"]
    for g in range(len(o) - 1):
        kv, lh = s["kv"][g // per_seq], g % per_seq
        l, h, rows, row0 = lh // case["H"], lh % case["H"], idx[o[g]:o[g + 1]], o[g] + slack * g
        for i, n in enumerate(("k", "v")):
            _segment_blocks(kv[i][l, h][rows].double(), row0 // BLOCK + g, got[n], got[n + "_scale"], row0, int8)
        if slack:
            got["up"][row0:row0 + rows.numel()] = s["scores"][g // per_seq][l, h][rows].double()
    return got


def _exact_append(s):
    """The new row, the rows of its block and its score; what else there is in the cache stays."""
    case, int8 = s["case"], s["int8"]
    per_seq, H = case["L"] * case["H"], case["H"]
    cap, used = s["cap"].tolist(), s["lengths_before"].tolist()
    got = {n: s[n].to(torch.float64) for n in ("k", "v", "k_scale", "v_scale", "up")}
    x = {"x": s["k_new"].reshape(case["n_seq"], per_seq, 1, D), "positions": s["positions"][:, None], "inv_freq": s["inv_freq"],
         "factor": s["factor"], "case": {**case, "backward": False}}
    new = {"k": _exact_rope(x).to(torch.bfloat16).double().reshape(-1, D), "v": s["v_new"].double().reshape(-1, D)}
    tops = {n: new[n].abs().amax(dim=1).tolist() for n in new}
    sc = s["scorer"]
    for g in range(len(used)):
        row, first, number = cap[g] + used[g], cap[g] + used[g] // BLOCK * BLOCK, cap[g] // BLOCK + g + used[g] // BLOCK
        for n in ("k", "v"):
            t = _scale_64(tops[n][g], int8)
            if row > first:
                old = got[n + "_scale"][number].item()
                if old > t:
                    t = old
                elif old < t:
                    got[n][first:row] = _nearest(got[n][first:row] * (old / t), int8)
            got[n + "_scale"][number] = t
            got[n][row] = _nearest(new[n][g] / t, int8) if t else torch.zeros_like(new[n][g])
        l = g % per_seq // H
        z = sc["w1"][l, 0].double() @ torch.cat((new["k"][g], new["v"][g])) + sc["b1"][l, 0].double()
        got["up"][row] = z[0] if not case["hidden"] else (z / (1 + torch.exp(-z)) * sc["w2"][l, 0].double()).sum()
    return got


def _exact_decode(s):
    case, G = s["case"], s["case"]["G"]
    cap, used = s["cap"].tolist(), s["lengths"].tolist()
    q = s["q"].double().reshape(-1, G, D)
    out = torch.zeros((len(used), G, D), dtype=torch.float64, device=_DEVICE)
    lse = torch.full((len(used), G), -math.inf, dtype=torch.float64, device=_DEVICE)
    for g, n in enumerate(used):
        if n:
            number = cap[g] // BLOCK + g + torch.arange(n, device=_DEVICE) // BLOCK
            k, v = (s[m][cap[g]:cap[g] + n].double() * s[m + "_scale"][number].double()[:, None] for m in ("k", "v"))
            logits = q[g] @ k.T / math.sqrt(D)
            lse[g] = torch.logsumexp(logits, dim=1)
            out[g] = torch.exp(logits - lse[g][:, None]) @ v
    return {"out": out.reshape(s["out"].shape), "lse": lse.reshape(s["lse"].shape)}


def _exact_reevict(s):
    case, int8, slack = s["case"], s["int8"], s["case"]["slack"]
    cap, used, budgets = s["cap"].tolist(), s["held"].tolist(), s["budgets"].tolist()
    f = dict(dtype=torch.float64, device=_DEVICE)
    got = {n: torch.zeros(s["new"][n].shape, **f) for n in ("k", "v", "k_scale", "v_scale", "up")}
    row0 = 0
    for g, n in enumerate(used):
        u = s["up"][cap[g]:cap[g] + n]
        rows = torch.sort(torch.sort(u, descending=True, stable=True).indices[:budgets[g]]).values
        for m in ("k", "v"):
            x = s[m][cap[g]:cap[g] + n].double() * s[m + "_scale"].double()[cap[g] // BLOCK + g + torch.arange(n, device=_DEVICE) // BLOCK][:, None]
            _segment_blocks(x[rows], row0 // BLOCK + g, got[m], got[m + "_scale"], row0, int8)
        got["up"][row0:row0 + budgets[g]] = u[rows].double()
        row0 += budgets[g] + slack
    return got


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("compact", "append", "reevict") and case["n_seq"] * case["L"] * case["H"] > 2048:
        return None
    return {"rope": _exact_rope, "compact": _exact_compact, "append": _exact_append, "decode": _exact_decode,
            "reevict": _exact_reevict}[case["op"]](s)
