"""What a row of cf_tree_attend sees, and nothing else, decides its bits: the cases in which something else could.

The scores are set through the first dimension: queries 8 there, key j s_j, so that a score in units of log2 e is s_j * 8 / sqrt(d) *
log2 e, plus little from the other dimensions.  The 300 cached rows and the drafted ones behind them make steps of 32 keys, of which a
wavefront takes every one, every fourth, or every second; in every step the largest cached key has s = BASE."""
import numpy as np
import pytest

from draft_cases import bytes_code, code_bytes
from oracle import draft_block as orc
from test_gpu_tree import Case

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

L, BASE = 300, 2.0
SIZES = [8, 20, 40, 100, 160]      # rows of a KV head: every kernel and number of rows that a workgroup may have


def _shaped(fmt, T, window=0, mask=None, depth=None, d=64, nkv=2):
    """A case whose keys and values are set by put(): keys [rows] of the first dimension, values whose rows have one scale."""
    if mask is None:
        mask = np.zeros((T, T), bool)
    c = Case(fmt, nkv, nkv, d, [L], T, mask=mask[None], depth=(np.zeros(T, np.int32) if depth is None else depth)[None], window=window, seed=50)
    c.tree.set_splits(1)
    rng = np.random.default_rng(7)
    c.q[:] = 0.1 * rng.standard_normal(c.q.shape)
    c.q[..., 0] = np.sqrt(d)
    c.first = rng.uniform(BASE - 0.5, BASE, c.rows)
    c.first[np.arange(3, c.rows, 32)] = BASE
    c.rest = np.clip(0.1 * rng.standard_normal((1, nkv, c.rows, d)), -0.5, 0.5)
    v = np.clip(rng.standard_normal((1, nkv, c.rows, d)), -3, 3)
    v[..., 0] = 4.0
    c.v, c.vs, c.vv = _stored(v.astype(np.float16), fmt)
    return c


def _stored(x, fmt):
    if fmt == "f16":
        return x, None, x.astype(np.float64)
    code, scale = orc.encode(x, fmt)
    return code_bytes(code, fmt), scale, code * scale.astype(np.float64)[..., None]


def _put(c, at=None, value=0.0):
    """The keys, with key `at` set apart."""
    k = c.rest.copy()
    k[..., 0] = c.first
    if at is not None:
        k[:, :, at, 0] = value
    c.k, c.ks, c.kv = _stored(k.astype(np.float16), c.fmt)


BAND = 7.75 / 1.4426950408889634     # 2^(7 + 7.75): a weight between 2^14.5 and 2^15 where the largest so far has 2^7


@pytest.mark.parametrize("fmt", ["f16", "e4m3", "int8"])
@pytest.mark.parametrize("T", SIZES)
def test_a_drafted_key_that_others_see(fmt, T):
    """Drafted token 4 has a key just below where a row's reference moves, and all tokens see it; token 5, in the same step, has one far
    above, and every other token sees it."""
    mask = np.zeros((T, T), bool)
    mask[:, 4] = mask[1::2, 5] = True
    c = _shaped(fmt, T, mask=mask)
    c.first[L:] = 0
    c.first[L + 4] = BASE + BAND
    got = []
    for value in (0.0, 40.0):
        _put(c, L + 5, value)
        got.append(c.check())
    assert np.array_equal(got[0][:, 0::2], got[1][:, 0::2])
    assert not np.array_equal(got[0][:, 1::2], got[1][:, 1::2])


@pytest.mark.parametrize("fmt", ["f16", "e4m3", "int8"])
@pytest.mark.parametrize("T", SIZES)
def test_a_cached_key_outside_a_window(fmt, T):
    """The same with scores that have a window: key 141 is the last one inside the window of every other token, key 140 is outside."""
    depth = np.full(T, 10, np.int32)
    depth[1::2] = 2
    c = _shaped(fmt, T, window=L + 10 - 140, depth=depth)
    c.first[141] = BASE + BAND
    got = []
    for value in (0.0, 40.0):
        _put(c, 140, value)
        got.append(c.check())
    assert np.array_equal(got[0][:, 0::2], got[1][:, 0::2])
    assert not np.array_equal(got[0][:, 1::2], got[1][:, 1::2])


@pytest.mark.parametrize("fmt", ["f16", "e4m3", "int8"])
@pytest.mark.parametrize("T", SIZES)
def test_another_tokens_large_scores(fmt, T):
    """Scores of 10^6 and more of every other token, whose references then hold no fractions; the rest are small."""
    c = _shaped(fmt, T)
    rng = np.random.default_rng(8)
    k = (30 * rng.standard_normal(c.rest.shape)).astype(np.float16)
    c.k, c.ks, c.kv = _stored(k, fmt)
    c.q[:] = 0.05 * rng.standard_normal(c.q.shape)
    quiet = c.check()
    c.q[:, 1::2] = 60000.0 * np.sign(c.q[:, 1::2])
    assert np.abs(np.einsum("bthd,bhjd->bthj", c.q[:, 1::2].astype(np.float64), c.kv[:, :, :L])).max(-1).min() / 8 > 2 ** 20
    loud = c.run()
    assert np.array_equal(quiet[:, 0::2], loud[:, 0::2])


# ---- infinities and NaN among the values ---------------------------------------------------------------------------------

def _unfit(fmt):
    """What to put among the values: (as stored, as seen in the result)."""
    if fmt == "f16":
        return [(np.float16(x), x) for x in (np.inf, -np.inf, np.nan)]
    return [(0x7f, np.nan), (0xff, np.nan)]


@pytest.mark.parametrize("fmt", ["f16", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T", SIZES)
@pytest.mark.parametrize("window", [0, 10000])
def test_infinite_values_with_small_weights(fmt, d, T, window):
    """A seen value that is infinite or NaN shows in the result, whatever its weight: e^-21 and e^-250 of the largest (less than fp16 and
    less than fp32 hold), before and behind the key that has the largest, in steps that all tokens see and in steps that they do not,
    in a part with the largest and in another one.  The other dimensions, and the tokens that do not see it, keep their bits."""
    mask = np.zeros((T, T), bool)
    mask[::2, 2] = True
    c = _shaped(fmt, T, mask=mask, window=window, d=d)
    for gap in (21.0, 250.0):
        c.first = np.random.default_rng(9).uniform(-0.25, 0.25, c.rows)
        c.first[200] = gap
        _put(c)
        for splits in (1, 3):
            c.tree.set_splits(splits)
            clean = c.run()
            for at, sees in ((10, slice(None)), (250, slice(None)), (L - 1, slice(None)), (L + 2, slice(0, None, 2))):
                for stored, seen in _unfit(fmt):
                    before = c.v[0, :, at, 5].copy()
                    c.v[0, :, at, 5] = stored
                    want = clean.copy()
                    want[:, sees, :, 5] = seen
                    got = c.run()
                    assert np.array_equal(got, want, equal_nan=True), (gap, splits, at, seen)
                    c.v[0, :, at, 5] = before


@pytest.mark.parametrize("T", SIZES)
def test_infinities_of_both_signs(T):
    """Seen together they are NaN; the token that sees one of them gets that one."""
    mask = np.zeros((T, T), bool)
    mask[::2, 2] = True
    c = _shaped("f16", T, mask=mask)
    c.first[200] = 250.0
    _put(c)
    c.v[0, :, 10, 5], c.v[0, :, L + 2, 5] = np.inf, -np.inf
    got = c.run()
    assert np.isnan(got[:, ::2, :, 5]).all() and (got[:, 1::2, :, 5] == np.inf).all()
    keep = [i for i in range(64) if i != 5]
    assert np.isfinite(got[..., keep]).all()


@pytest.mark.parametrize("T", SIZES)
@pytest.mark.parametrize("d", [64, 128])
def test_unseen_rows_may_hold_nan_codes(T, d):
    """e4m3 codes that are NaN, in keys and values of a drafted token, and in cached rows outside a window."""
    mask = np.zeros((T, T), bool)
    mask[:, 4] = mask[1::2, 5] = True
    c = _shaped("e4m3", T, mask=mask, d=d)
    _put(c)
    clean = c.check()
    c.k[0, :, L + 5], c.v[0, :, L + 5] = 0x7f, 0xff
    got = c.run()
    assert np.array_equal(got[:, 0::2], clean[:, 0::2]) and np.isnan(got[:, 1::2]).all()
    depth = np.full(T, 10, np.int32)
    depth[1::2] = 2
    c = _shaped("e4m3", T, window=L + 10 - 140, depth=depth, d=d)
    _put(c)
    clean = c.check()
    c.k[0, :, 140], c.v[0, :, 140] = 0xff, 0x7f
    got = c.run()
    assert np.array_equal(got[:, 0::2], clean[:, 0::2]) and np.isnan(got[:, 1::2]).all()
    c.k[0, :, :140], c.v[0, :, :140] = 0x7f, 0x7f                   # what no token sees
    assert np.array_equal(c.run()[:, 0::2], clean[:, 0::2])


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("T", SIZES)
def test_a_nan_scale_with_a_small_weight(fmt, T):
    """A seen row of values with scale NaN is NaN in every dimension, however small its weight."""
    c = _shaped(fmt, T)
    c.first[200] = 250.0
    _put(c)
    for at in (10, 250, L - 1):
        before = c.vs[0, :, at].copy()
        c.vs[0, :, at] = np.nan
        assert np.isnan(c.run()).all(), at
        c.vs[0, :, at] = before


@pytest.mark.parametrize("T", SIZES)
def test_a_nan_score_beside_an_infinite_value(T):
    """Every dimension of a token that sees a key of NaN is NaN, that of the infinity too; the others get the infinity."""
    mask = np.zeros((T, T), bool)
    mask[::2, 2] = True
    c = _shaped("f16", T, mask=mask)
    _put(c)
    for splits in (1, 3):
        c.tree.set_splits(splits)
        clean = c.run()
        keep = c.v[0, :, 10, 5].copy(), c.k[0, :, L + 2].copy()
        c.v[0, :, 10, 5], c.k[0, :, L + 2] = np.inf, np.nan
        got = c.run()
        clean[..., 5] = np.inf
        assert np.isnan(got[:, ::2]).all() and np.array_equal(got[:, 1::2], clean[:, 1::2])
        c.v[0, :, 10, 5], c.k[0, :, L + 2] = keep
