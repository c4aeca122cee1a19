"""Pins of oracle/quantized_step.py and of the 4-bit format, all on the CPU."""
import math

import numpy as np
import pytest

from oracle import quantized_step as orc


def halves():
    """All finite fp16 numbers."""
    x = np.arange(65536, dtype=np.uint16).view(np.float16)
    return x[np.isfinite(x)]


def test_every_value_of_every_block_is_an_fp16_number():
    for byte in range(104, 141):
        v = orc.decode4(np.arange(16, dtype=np.uint8).repeat(2), np.array([byte], np.uint8))
        assert np.array_equal(v.astype(np.float16).astype(np.float64), v), byte
    assert np.isnan(orc.decode4(np.arange(32, dtype=np.uint8) % 16, np.array([255], np.uint8))).all()


def test_codes_by_hand():
    """One block with top 6: every border between two levels, and both sides of it."""
    x = np.zeros(32, np.float16)
    x[:16] = [6, 0.25, 0.26, 0.75, 0.74, 1.25, 1.26, 1.75, 1.74, 2.5, 2.51, 3.5, 3.49, 5, 5.01, -5]
    code, scale = orc.encode4(x)
    assert scale.tolist() == [127]
    assert code[:16].tolist() == [7, 0, 1, 2, 1, 2, 3, 4, 3, 4, 5, 6, 5, 6, 7, 14]
    assert orc.encode4(np.full(32, -0.0, np.float16))[0].tolist() == [8] * 32


@pytest.mark.parametrize("top,power", [(6.0, 0), (6.004, 1), (3.0, -1), (3.002, 0), (0.0, -23), (2.0 ** -24, -23), (65504.0, 13), (49152.0, 13), (49184.0, 13)])
def test_powers(top, power):
    x = np.zeros(64, np.float16)
    x[40] = top
    assert orc.encode4(x)[1].tolist() == [104, 127 + power]


def test_values_are_the_nearest_ones():
    """Of all fp16 numbers in blocks with tops of any size: no level of the block is nearer than the one that was taken."""
    rng = np.random.default_rng(0)
    x = rng.permutation(halves())
    x = x[:x.size // 32 * 32].reshape(-1, 32)
    x = np.concatenate([x, (x.astype(np.float64) * 2.0 ** rng.integers(-20, 0, (x.shape[0], 1))).astype(np.float16)])
    code, scale = orc.encode4(x)
    value = orc.decode4(code, scale)
    grid = np.concatenate([orc.LEVELS, -orc.LEVELS]) * np.ldexp(1.0, scale.astype(int) - 127)
    gap = np.abs(x.astype(np.float64)[..., None] - grid[:, None]).min(-1)
    assert np.array_equal(np.abs(x - value), gap)
    assert np.array_equal(np.signbit(value), np.signbit(x))


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_a_block_that_is_no_number(bad):
    x = np.ones(96, np.float16)
    x[50] = bad
    code, scale = orc.encode4(x)
    assert scale.tolist() == [125, 255, 125] and not code[32:64].any()       # 1 <= 6 / 4
    assert np.isnan(orc.decode4(code, scale)).tolist() == [False] * 32 + [True] * 32 + [False] * 32


def test_packing():
    code = np.arange(64, dtype=np.uint8) % 16
    assert orc.pack4(code)[:3].tolist() == [0x10, 0x32, 0x54] and np.array_equal(orc.unpack4(orc.pack4(code)), code)


def test_norm_of_heads():
    x = np.array([[3.0, 4.0]], np.float16)
    assert np.allclose(orc.head_norm(x, np.array([1, 2], np.float16), 0.0), [[3 / math.sqrt(12.5), 8 / math.sqrt(12.5)]], rtol=1e-15)
    y = orc.head_norm(np.random.default_rng(0).standard_normal((5, 64)).astype(np.float16), np.ones(64, np.float16), 0.0)
    assert np.allclose((y * y).mean(-1), 1.0, rtol=1e-12)


def test_integer_products():
    x, w = np.array([[127, -128, 3]], np.int8), np.array([[-128, -128, 5], [1, 0, 0]], np.int8)
    total, out = orc.int8_product(x, np.array([0.5], np.float32), w, np.array([0.25, 2], np.float32))
    assert total.tolist() == [[127 * -128 + 128 * 128 + 15, 127]] and out.tolist() == [[143 / 8, 127.0]]
