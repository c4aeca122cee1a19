"""Inputs of the tests of cf_cache_* and cf_tree_* (seeded numpy), and what both files share."""
import numpy as np

from oracle import draft_block as orc

FORMATS = {"f16": 0, "e4m3": 1, "int8": 2}


def random_tree(rng, tokens, chain=False):
    """depth [T], mask [T, T] (bool) of a tree: every token continues an earlier one and sees its ancestors and itself."""
    depth, mask = np.zeros(tokens, np.int32), np.zeros((tokens, tokens), bool)
    for t in range(tokens):
        mask[t, t] = True
        if t:
            parent = t - 1 if chain else int(rng.integers(t))
            depth[t] = depth[parent] + 1
            mask[t] |= mask[parent]
    return depth, mask


def mask_words(mask):
    """[..., T, T] bool -> [..., T, (T + 63) / 64] uint64, bit u % 64 of word u / 64."""
    T = mask.shape[-1]
    words = np.zeros(mask.shape[:-1] + ((T + 63) // 64,), np.uint64)
    for u in range(T):
        words[..., u // 64] |= mask[..., u].astype(np.uint64) << np.uint64(u % 64)
    return words


def cache_values(rng, shape, fmt):
    """A cache of fp16 rows of different size: (stored tensor as numpy, scales or None, the fp64 values that it stands for)."""
    x = (rng.standard_normal(shape) * np.exp(0.5 * rng.standard_normal(shape[:-1] + (1,)))).astype(np.float16)
    if fmt == "f16":
        return x, None, x.astype(np.float64)
    code, scale = orc.encode(x, fmt)
    return code_bytes(code, fmt), scale, code * scale.astype(np.float64)[..., None]


def code_bytes(code, fmt):
    if fmt == "int8":
        return code.astype(np.int8).view(np.uint8)
    order = np.argsort(orc.E4M3[:127])
    at = order[np.searchsorted(orc.E4M3[:127], np.abs(code))]
    return (at + np.where(np.signbit(code), 128, 0)).astype(np.uint8)


def bytes_code(raw, fmt):
    return raw.view(np.int8).astype(np.float64) if fmt == "int8" else orc.E4M3[raw]


def bound(out, size, reach, flat, d, keys, slope_reach=0.0):
    """Largest error of an element of cf_tree_attend's result.  fp16 result: 2^-11 |out|, 2^-25 near zero.  Softmax weights
    rounded to fp16 for the second product: 2^-11 of each, so 2^-11 sum p |v|, and as much again for weights that enter the
    product times a scale.  Scores in fp32: d + 8 roundings of at most sum |q k| / sqrt(d) (and of the distance bias), which moves a weight, and the sum that divides
    it, by twice that.  Sums over the keys: one rounding per key, of both sums.
    Weights that are small beside the row's largest: fp16 numbers below 2^-14 lie 2^-24 apart, so that a weight w_j may be off by
    2^-25.  The largest w_j is at least 2^7 (where the reference was last moved to), w_j = p_j s_j L with s_j the scale of the value row
    (1 in fp16) and L the row's sum, so 1 / L <= 2^-7 max(p_j s_j), and the result is off by 2^-25 sum_j |v_j / s_j| / L at most."""
    half = 2.0 ** -11
    score = 2.0 * ((d + 8) * 2.0 ** -24 * reach + 4 * 2.0 ** -24 * slope_reach)
    return half * np.abs(out) + 2.0 ** -25 + 2.0 ** -32 * flat + size * (2 * half + score[..., None] + 2 * keys * 2.0 ** -24)
