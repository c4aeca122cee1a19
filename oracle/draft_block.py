"""Drafted tokens on a key/value cache, in numpy and fp64: the plain definitions of cf_cache_* and cf_tree_attend
(include/cfdecode.h), written head by head and token by token.  Test infrastructure only.

The steps are those of the decode block (paper Eq. 1: rotation, append, softmax(q K^T / sqrt(d)) V) for several new tokens per
sequence; the 8-bit formats, the masks and the forms of the score are this library's own definitions.
"""
import math

import numpy as np

LARGEST = {"e4m3": 448.0, "int8": 127.0}


def rotate(x, position, base):
    """Pairs (i, i + d/2) of the last dimension turned by position * base^(-2i/d), fp64."""
    d = x.shape[-1]
    angle = position * np.array([math.pow(base, -2.0 * i / d) for i in range(d // 2)])
    c, s = np.cos(angle), np.sin(angle)
    lo, hi = x[..., :d // 2].astype(np.float64), x[..., d // 2:].astype(np.float64)
    return np.concatenate([lo * c - hi * s, hi * c + lo * s], -1)


def e4m3_codes():
    """The values of the 8-bit floats of format e4m3 by code: four exponent bits (bias 7), three of the mantissa, 0x7f NaN."""
    v = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        mag = math.nan if (c & 0x7f) == 0x7f else math.ldexp(m / 8.0, -6) if e == 0 else math.ldexp(1.0 + m / 8.0, e - 7)
        v[c] = -mag if c >> 7 else mag
    return v


E4M3 = e4m3_codes()


def encode(rows, fmt):
    """fp16 rows [..., d] -> (values of the codes as fp64, scales fp32): code = x Q / top, to the nearest, ties to even."""
    x = rows.astype(np.float64)
    top = np.abs(x).max(-1, keepdims=True)
    with np.errstate(invalid="ignore", divide="ignore"):
        y = np.where((top > 0) & np.isfinite(top), x * LARGEST[fmt] / top, 0.0)
    if fmt == "int8":
        code = np.rint(y)
    else:
        grid = E4M3[:127]                                      # ascending magnitudes, even codes have even mantissas
        at = np.clip(np.searchsorted(grid, np.abs(y), side="right") - 1, 0, 125)
        low, high = np.abs(y) - grid[at], grid[at + 1] - np.abs(y)
        pick = np.where((high < low) | ((high == low) & (at % 2 == 1)), at + 1, at)
        code = np.where(y == 0, 0.0, np.copysign(grid[pick], y))
    scale = np.where(np.isfinite(top), top.astype(np.float32) / np.float32(LARGEST[fmt]), np.float32("nan"))[..., 0]
    return code, scale.astype(np.float32)


def attend(q, keys, values, lens, counts, depth, mask, slopes=None, cap=0.0, window=0,
           value_scales=None):
    """q [B, T, nq, d], keys / values [B, nkv, rows, d] (fp64 values of the cache), lens / counts [B], depth [B, T],
    mask [B, T, T] (mask[b, t, u]: t sees the new token u).  Returns out [B, T, nq, d] (NaN for padding) and, of the same shape,
    sum_j p_j |v_j|, per (b, t, head) the largest sum_i |q_i k_i| / sqrt(d) of the seen keys, and, of out's shape, the largest
    p_j s_j times sum_j |v_j| / s_j, s_j the scales of the value rows ([B, nkv, rows], or 1)."""
    B, T, nq, d = q.shape
    group = nq // keys.shape[1]
    out, size, flat = np.full(q.shape, np.nan), np.zeros(q.shape), np.zeros(q.shape)
    reach = np.zeros((B, T, nq))
    for b in range(B):
        L, n = int(lens[b]), int(counts[b])
        key_pos = np.concatenate([np.arange(L), L + depth[b, :n]]).astype(np.float64)
        for t in range(n):
            seen = np.concatenate([np.ones(L, bool), mask[b, t, :n].astype(bool)])
            distance = L + depth[b, t] - key_pos
            if window > 0:
                seen &= distance < window
            idx = np.nonzero(seen)[0]
            for h in range(nq):
                if idx.size == 0:
                    out[b, t, h] = 0.0
                    continue
                k, v = keys[b, h // group, idx], values[b, h // group, idx]
                qq = q[b, t, h].astype(np.float64)
                s = k @ qq / math.sqrt(d)
                reach[b, t, h] = (np.abs(k) @ np.abs(qq)).max() / math.sqrt(d)
                if cap > 0:
                    s = cap * np.tanh(s / cap)
                if slopes is not None:
                    s = s - float(slopes[h]) * distance[idx]
                p = np.exp(s - s.max())
                p /= p.sum()
                out[b, t, h] = p @ v
                size[b, t, h] = p @ np.abs(v)
                unit = np.ones(idx.size) if value_scales is None else value_scales[b, h // group, idx].astype(np.float64)
                some = unit > 0
                if some.any():
                    flat[b, t, h] = (p * unit)[some].max() * (np.abs(v)[some] / unit[some, None]).sum(0)
    return out, size, reach, flat
