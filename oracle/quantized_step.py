"""A quantised step, in numpy and fp64: the plain definitions of cf_linear_*, of the 4-bit cache format and of the norms in
cf_cache_append_normed (include/cfdecode.h).  Test infrastructure only; these are the library's own definitions, the paper has none of them.
"""
import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])        # of the codes 0..7; 8..15 are their negatives


def encode4(rows):
    """fp16 rows [..., d] -> (codes [..., d] 0..15, scale bytes [..., d / 32])."""
    x = rows.astype(np.float64).reshape(rows.shape[:-1] + (-1, 32))
    top = np.abs(x).max(-1, keepdims=True)
    fine = np.isfinite(top)
    e = np.full(top.shape, -23)
    while True:                                                      # the smallest power of two, tried one after the other
        low = fine & (top > 6 * np.ldexp(1.0, e)) & (e < 13)
        if not low.any():
            break
        e = e + low
    y = np.where(fine, x, 0.0) / np.ldexp(1.0, e)
    gap = np.abs(np.abs(y)[..., None] - LEVELS)
    best = gap.min(-1, keepdims=True)
    first = (gap == best).argmax(-1)                                 # the lower of two that are as near
    tie = (gap == best).sum(-1) == 2
    code = first + (tie & (first % 2 == 1))
    code = np.where(fine, code + 8 * np.signbit(np.where(fine, x, 0.0)), 0)
    scale = np.where(fine, e + 127, 255)[..., 0]
    return code.reshape(rows.shape).astype(np.uint8), scale.astype(np.uint8)


def decode4(code, scale):
    """fp64 values of codes and scale bytes (104..140 or 255)."""
    unit = np.where(scale == 255, np.nan, np.ldexp(1.0, scale.astype(np.int32) - 127))
    value = np.where(code >= 8, -LEVELS[code & 7], LEVELS[code & 7])
    with np.errstate(invalid="ignore"):
        return value * np.repeat(unit, 32, -1)


def pack4(code):
    """Two codes to a byte, the first in the low half."""
    return (code[..., 0::2] | code[..., 1::2] << 4).astype(np.uint8)


def unpack4(packed):
    return np.stack([packed & 15, packed >> 4], -1).reshape(packed.shape[:-1] + (2 * packed.shape[-1],))


def head_norm(x, weight, eps):
    """x / sqrt(mean x^2 + eps) * weight over the last dimension, fp64."""
    x = x.astype(np.float64)
    with np.errstate(invalid="ignore", divide="ignore"):
        return x / np.sqrt((x * x).mean(-1, keepdims=True) + np.float64(np.float32(eps))) * weight.astype(np.float64)


def int8_product(x, x_scale, w, w_scale):
    """The sums as exact integers, and the result: (sum as fp32 * x_scale) * w_scale in fp32, as fp16."""
    total = x.astype(np.int64) @ w.astype(np.int64).T
    with np.errstate(over="ignore", invalid="ignore"):
        out = total.astype(np.float32) * x_scale[:, None].astype(np.float32) * w_scale[None].astype(np.float32)
        return total, out.astype(np.float16)
