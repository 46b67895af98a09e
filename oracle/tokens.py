"""Plain numpy statements of the 8-bit transformer operators -- test infrastructure only.

Codes and scales are decided in fp32, one rounding per operation, exactly as the C ABI
states; every sum is taken in integers or in double.
"""
from __future__ import annotations

import numpy as np

F = np.float32
INV127 = F(1.0) / F(127.0)
TINY = F(2.0 ** -126)  # the smallest normal number


def scale_of(x, axes):
    """Scale(s) of fp32 values along `axes` (kept): amax * fl(1/127), 0 below the smallest normal, NaN with a non-finite value."""
    x = np.asarray(x, F)
    a = np.abs(x)
    bad = ~np.isfinite(x).all(axes, keepdims=True) if x.size else np.zeros_like(a.sum(axes, keepdims=True), bool)
    with np.errstate(invalid="ignore", over="ignore"):
        s = (np.where(np.isfinite(a), a, 0).max(axes, keepdims=True, initial=0) * INV127).astype(F)
    s = np.where(s < TINY, F(0), s)
    return np.where(bad, F(np.nan), s).astype(F)


def codes_of(x, s):
    """clamp(rint(fl(x * fl(1/s))), -127, 127); 0 where s is 0 or NaN."""
    with np.errstate(divide="ignore", invalid="ignore", over="ignore"):
        inv = np.where(s > 0, F(1) / s, F(0)).astype(F)
        t = (np.asarray(x, F) * inv).astype(F)
        return np.where(s > 0, np.clip(np.rint(t), -127, 127), 0).astype(np.int8)


def quantize_tokens(x):
    """(codes [M, K] int8, scales [M] fp32) of x [M, K]."""
    s = scale_of(x, (1,))
    return codes_of(x, s), s[:, 0]


def linear(q, w):
    """int64 sums [M, N] of codes q [M, K] and w [N, K]."""
    return q.astype(np.int64) @ w.astype(np.int64).T


def linear_value(acc, s_x, s_w, bias=None):
    """The layer's output in double, without a rounding."""
    y = acc.astype(np.float64) * s_x.astype(np.float64)[:, None] * s_w.astype(np.float64)[None]
    return y if bias is None else y + bias.astype(np.float64)[None]


def append(codes, scales, table, start, x):
    """One side: the run x [n, H, D] of one sequence quantised into codes [pages, H, T, D] and scales [pages, H], in place."""
    T = codes.shape[2]
    n = x.shape[0]
    for block in range(start // T, -(-(start + n) // T)):
        lo, hi = max(start, block * T), min(start + n, block * T + T)
        page, old = table[block], lo - block * T
        new = np.asarray(x[lo - start:hi - start], F).transpose(1, 0, 2)  # [H, tokens, D]
        s = scale_of(new, (1, 2))[:, 0, 0]
        if old:
            was = scales[page].copy()
            with np.errstate(invalid="ignore"):
                s = np.where(np.isnan(s) | np.isnan(was), F(np.nan), np.maximum(s, was)).astype(F)
            for h in range(codes.shape[1]):
                if not s[h] == was[h]:
                    inv = F(1) / s[h] if s[h] > 0 else F(0)
                    ratio = F(was[h] * inv) if s[h] > 0 else F(0)
                    t = (codes[page, h, :old].astype(F) * ratio).astype(F)
                    codes[page, h, :old] = np.clip(np.rint(t), -127, 127).astype(np.int8)
        codes[page, :, old:old + hi - lo] = codes_of(new, s[:, None, None])
        scales[page] = s


def read(codes, scales, table, start, n):
    """fp32 values [n, H, D] of one side's tokens."""
    T = codes.shape[2]
    pos = np.arange(start, start + n)
    page, slot = np.asarray(table)[pos // T], pos % T
    return (codes[page, :, slot].astype(F) * scales[page][:, :, None]).astype(F)


def attention(q, k, v, scale, causal=True, window=0, seen=None):
    """One sequence: q [n, Hq, D], k and v [len, Hkv, D]; seen [n, len]: what each query sees, instead of the rest.  Returns (o, spread, top) in double: o [n, Hq, D], spread = sum
    softmax * |v| (what an error of the probabilities is multiplied with) and the largest |score| of each row [n, Hq, 1]."""
    n, Hq, D = q.shape
    length, H = k.shape[0], k.shape[1]
    o = np.zeros((n, Hq, D))
    spread = np.zeros((n, Hq, D))
    top = np.zeros((n, Hq, 1))
    if length == 0:
        return o, spread, top
    at = (length - n + np.arange(n))[:, None]
    j = np.arange(length)[None]
    if seen is not None:
        causal = False
    else:
        seen = np.ones((n, length), bool)
    if causal:
        seen = j <= at
        if window:
            seen &= j > at - window
    for hq in range(Hq):
        h = hq // (Hq // H)
        s = scale * (q[:, hq].astype(np.float64) @ k[:, h].astype(np.float64).T)
        s = np.where(seen, s, -np.inf)
        with np.errstate(invalid="ignore"):
            m = s.max(1, keepdims=True)
            m = np.where(np.isneginf(m), 0, m)
            p = np.where(seen, np.exp(s - m), 0.0)
            l = p.sum(1, keepdims=True)
            p = np.where(l == 0, 0, p / np.where(l == 0, 1, l))
        vh = v[:, h].astype(np.float64)
        for i in range(n):  # values that no probability reaches do not count, whatever they are
            on = seen[i]
            o[i, hq] = p[i, on] @ vh[on]
            spread[i, hq] = p[i, on] @ np.abs(vh[on])
        top[:, hq, 0] = np.where(seen, np.abs(np.where(seen, s, 0)), 0).max(1)
    return o, spread, top


def sees_sinks(n, length, window, sinks):
    """[n, length]: the tokens up to each of the last n ones, through a window (0: none) and with the first `sinks`."""
    at, j = (length - n + np.arange(n))[:, None], np.arange(length)[None]
    return (j <= at) & ((j > at - window) | (j < sinks) | (window == 0))


def sees_tree(n, length, bits):
    """[n, length]: everything before the last n tokens, and those of the last n whose bit is set in bits [n, words]."""
    out = np.zeros((n, length), bool)
    for i in range(n):
        for j in range(length):
            d = j - (length - n)
            out[i, j] = d < 0 or int(bits[i, d // 32]) >> (d % 32) & 1
    return out


def norm_rope(x, weight, eps, positions, frequencies, interleaved, norm=True):
    """Heads x [tokens, heads, D] normed and rotated, in double.  Returns (y, size): size [tokens, heads, D] the sum of the
    magnitudes that each output is made of."""
    x = np.asarray(x, np.float64)
    if norm:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * (1 if weight is None else np.asarray(weight, np.float64))
    y, size = x.copy(), np.abs(x)
    for j, f in enumerate(frequencies):
        a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + len(frequencies))
        angle = np.asarray(positions, np.float64) * f
        c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
        size[..., a] = size[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    return y, size


def w4_quantize(w, group, round_scale=None, smallest=TINY):
    """(codes [N, K] int8, scales [N, groups] fp32) of w [N, K]; round_scale: fp32 to the scales' type and back."""
    w = np.asarray(w, F)
    N, K = w.shape
    groups = -(-K // group)
    codes, scales = np.zeros((N, K), np.int8), np.zeros((N, groups), F)
    for g in range(groups):
        part = w[:, g * group:(g + 1) * group]
        a = np.abs(part)
        with np.errstate(all="ignore"):
            s = (np.where(np.isfinite(a), a, 0).max(1) * (F(1) / F(7))).astype(F)
            s = s if round_scale is None else round_scale(s)
            s = np.where(s < smallest, F(0), s).astype(F)
            s = np.where(np.isfinite(part).all(1) & np.isfinite(s), s, F(np.nan))
            inv = np.where(s > 0, F(1) / s, F(0)).astype(F)[:, None]
            c = np.clip(np.rint((part * inv).astype(F)), -7, 7)
        codes[:, g * group:(g + 1) * group] = np.where(inv > 0, c, 0).astype(np.int8)
        scales[:, g] = s
    return codes, scales


def linear_w4(x, codes, scales, group, bias=None):
    """(y, size) in double: y [M, N], size the sum of the products' magnitudes."""
    x, w = np.asarray(x, np.float64), codes.astype(np.float64) * np.repeat(np.asarray(scales, np.float64), group, 1)[:, : codes.shape[1]]
    y, size = x @ w.T, np.abs(x) @ np.abs(w).T
    return (y, size) if bias is None else (y + np.asarray(bias, np.float64), size + np.abs(bias))
