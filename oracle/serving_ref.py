"""Plain float64 definitions of rotary positions and of the 8-bit paged cache (append, attention, eviction), in numpy.
Slow and literal: one token, head or page at a time; used by tests only."""
from __future__ import annotations

import math

import numpy as np

TOP = {"e4m3": 448.0, "int8": 127.0}
MIN_SCALE = 2.0 ** -100


# ---------------------------------------------------------------------------------------------------------
# Rotary positions
# ---------------------------------------------------------------------------------------------------------
def rope_frequencies(rotary_dim, base, scaling="none", factor=1.0, original_length=0.0, low=0.0, high=0.0):
    """Radians per token of each pair, one at a time."""
    r, s, out = rotary_dim, factor, []
    low = low if low > 0 else 1.0
    high = high if high > 0 else (32.0 if scaling == "yarn" else 4.0)
    for i in range(r // 2):
        f = base ** (-2.0 * i / r)
        if scaling == "linear":
            f = f / s
        elif scaling == "ntk":
            f = (base * s ** (r / (r - 2.0))) ** (-2.0 * i / r)
        elif scaling == "yarn":
            dim = lambda n: r * math.log(original_length / (2 * math.pi * n)) / (2 * math.log(base))
            lo = min(max(math.floor(dim(high)), 0), r - 1)
            hi = min(max(math.ceil(dim(low)), 0), r - 1)
            t = min(max((i - lo) / max(hi - lo, 1e-3), 0.0), 1.0)
            f = f / s * t + f * (1 - t)
        elif scaling == "wavelength":
            u = min(max((original_length * f / (2 * math.pi) - low) / (high - low), 0.0), 1.0)
            f = f * u + f / s * (1 - u)
        out.append(f)
    return np.asarray(out)


def rope_magnitude(scaling="none", factor=1.0, magnitude=0.0):
    if magnitude > 0:
        return magnitude
    return 0.1 * math.log(factor) + 1.0 if scaling == "yarn" else 1.0


def rope(x, positions, freqs, rotary_dim, layout="half", magnitude=1.0, backward=False):
    """x [T][heads][D] -> turned copy in float64."""
    y = np.array(x, dtype=np.float64)
    angle = np.asarray(positions, dtype=np.float64)[:, None] * freqs[None]
    c, s = magnitude * np.cos(angle), magnitude * np.sin(angle) * (-1.0 if backward else 1.0)
    for i in range(rotary_dim // 2):
        a, b = (i, i + rotary_dim // 2) if layout == "half" else (2 * i, 2 * i + 1)
        u, v = np.array(x[..., a], dtype=np.float64), np.array(x[..., b], dtype=np.float64)
        y[..., a] = u * c[:, i, None] - v * s[:, i, None]
        y[..., b] = v * c[:, i, None] + u * s[:, i, None]
    return y


# ---------------------------------------------------------------------------------------------------------
# Codes
# ---------------------------------------------------------------------------------------------------------
def e4m3_values():
    """Value of each of the 256 codes."""
    v = np.zeros(256)
    for c in range(256):
        sign, e, m = -1.0 if c & 128 else 1.0, (c >> 3) & 15, c & 7
        v[c] = math.nan if (c & 127) == 127 else sign * (m / 8.0 * 2.0 ** -6 if e == 0 else (1 + m / 8.0) * 2.0 ** (e - 7))
    return v


def code_values(kind, codes):
    """Codes (uint8 bit patterns) -> what they stand for."""
    codes = np.asarray(codes, dtype=np.uint8)
    return e4m3_values()[codes] if kind == "e4m3" else codes.view(np.int8).astype(np.float64)


def nearest(kind, x):
    """Nearest code value (ties to even) of finite or infinite numbers, NaN kept for e4m3 and 0 for int8."""
    x = np.asarray(x, dtype=np.float64)
    if kind == "int8":
        return np.where(np.isnan(x), 0.0, np.clip(np.rint(np.nan_to_num(x, nan=0.0)), -127, 127))
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        a = np.minimum(np.abs(x), 448.0)
        e = np.maximum(np.floor(np.log2(np.maximum(a, 2.0 ** -30))), -6.0)
        step = 2.0 ** (e - 3)
        return np.where(np.isnan(x), np.nan, np.copysign(np.minimum(np.rint(a / step) * step, 448.0), x))


def fresh_scale(kind, x):
    """Smallest power of two that brings max |x| under the largest code."""
    x = np.asarray(x, dtype=np.float64)
    largest_bf16 = (2 - 2.0 ** -7) * 2.0 ** 127
    x = np.where(np.isnan(x), 0.0, np.minimum(np.abs(x), largest_bf16))
    a = float(x.max()) if x.size else 0.0
    s = MIN_SCALE
    while a / s > TOP[kind]:
        s *= 2
    return s


# ---------------------------------------------------------------------------------------------------------
# The cache.  state: dict(k, v: code values [pages][hkv][page][D]; k_scale, v_scale [pages][hkv]; weight or None)
# ---------------------------------------------------------------------------------------------------------
def append(kind, state, page_table, length, row_offset, k, v):
    """In place; k, v [rows][hkv][D]."""
    page_tokens = state["k"].shape[2]
    for b in range(len(length)):
        n = row_offset[b + 1] - row_offset[b]
        start = max(length[b] - n, 0)
        shift = row_offset[b] + n - length[b]                 # row of position p is p + shift
        p0 = start
        while n > 0 and p0 < length[b]:
            j = p0 // page_tokens
            p1 = min((j + 1) * page_tokens, length[b])
            page, held = page_table[b][j], p0 - j * page_tokens
            for h in range(state["k"].shape[1]):
                for name, x in (("k", k), ("v", v)):
                    rows = np.asarray(x[p0 + shift:p1 + shift, h], dtype=np.float64)
                    scale = fresh_scale(kind, rows)
                    codes = state[name][page, h]
                    if held:
                        old = state[name + "_scale"][page, h]
                        scale = max(scale, old)
                        codes[:held] = nearest(kind, codes[:held] * (old / scale))
                    state[name + "_scale"][page, h] = scale
                    codes[held:held + p1 - p0] = nearest(kind, rows / scale)
                if state.get("weight") is not None:
                    state["weight"][page, h, held:held + p1 - p0] = 0.0
            p0 = p1


def gather(state, name, pages, n, h):
    """Values [n][D] of the first n tokens on `pages`."""
    x = state[name][pages, h] * state[name + "_scale"][pages, h][:, None, None]
    return x.reshape(-1, x.shape[-1])[:n]


def attention(state, page_table, length, row_offset, q, scale=0.0):
    """q [rows][hq][D] -> dict(o, lse, weights = list per sequence of [hkv][length], spread = sum p |v|, size = max scale sum |q||k|)."""
    rows, hq, d = q.shape
    hkv, page_tokens = state["k"].shape[1], state["k"].shape[2]
    g, scale = hq // hkv, scale if scale > 0 else 1.0 / math.sqrt(d)
    o, lse = np.zeros((rows, hq, d)), np.full((rows, hq), -np.inf)
    spread, size, weights = np.zeros((rows, hq, d)), np.zeros((rows, hq)), []
    for b in range(len(length)):
        n, t = row_offset[b + 1] - row_offset[b], length[b]
        pages = np.asarray(page_table[b][:-(-t // page_tokens)], dtype=np.int64)
        w = np.zeros((hkv, t))
        for h in range(hkv):
            k, v = gather(state, "k", pages, t, h), gather(state, "v", pages, t, h)
            for j in range(n):
                seen = t - n + j + 1
                if seen <= 0:
                    continue
                for i in range(g):
                    row, head = row_offset[b] + j, h * g + i
                    s = k[:seen] @ np.asarray(q[row, head], dtype=np.float64) * scale
                    m = s.max()
                    e = np.exp(s - m)
                    p = e / e.sum()
                    o[row, head] = p @ v[:seen]
                    lse[row, head] = m + math.log(e.sum())
                    spread[row, head] = p @ np.abs(v[:seen])
                    size[row, head] = (np.abs(k[:seen]) @ np.abs(np.asarray(q[row, head], dtype=np.float64))).max() * scale
                    w[h, :seen] += p
        weights.append(w)
    return dict(o=o, lse=lse, weights=weights, spread=spread, size=size)


def choose(weight, n_sink, n_heavy, n_recent):
    """Positions of one head that stay, in order; equal weights: the earlier one, NaN last."""
    t = len(weight)
    if t <= n_sink + n_heavy + n_recent:
        return np.arange(t)
    middle = list(range(n_sink, t - n_recent))
    order = sorted(middle, key=lambda p: (math.isnan(weight[p]), 0.0 if math.isnan(weight[p]) else -weight[p], p))
    return np.asarray(sorted(list(range(n_sink)) + order[:n_heavy] + list(range(t - n_recent, t))), dtype=np.int64)


def evict(kind, state, page_table, length, n_sink, n_heavy, n_recent, dst_table):
    """In place; returns kept [B][hkv][keep] and new_length [B]."""
    keep, page_tokens, hkv = n_sink + n_heavy + n_recent, state["k"].shape[2], state["k"].shape[1]
    kept = np.full((len(length), hkv, keep), -1, np.int64)
    new_length = np.minimum(np.asarray(length), keep)
    for b in range(len(length)):
        for h in range(hkv):
            pages = np.asarray(page_table[b][:-(-length[b] // page_tokens)], dtype=np.int64)
            pos = choose(state["weight"][pages, h].reshape(-1)[:length[b]], n_sink, n_heavy, n_recent)
            kept[b, h, :len(pos)] = pos
            src = [(page_table[b][p // page_tokens], p % page_tokens) for p in pos]
            for j in range(0, len(pos), page_tokens):
                dst, part = dst_table[b][j // page_tokens], src[j:j + page_tokens]
                for name in ("k", "v"):
                    s = max(max(state[name + "_scale"][p, h] for p, _ in part), MIN_SCALE)
                    for i, (p, slot) in enumerate(part):
                        state[name][dst, h, i] = nearest(kind, state[name][p, h, slot] * (state[name + "_scale"][p, h] / s))
                    state[name + "_scale"][dst, h] = s
                for i, (p, slot) in enumerate(part):
                    state["weight"][dst, h, i] = state["weight"][p, h, slot]
    return kept, new_length
