"""Pins of oracle/draft_block.py, and the refusals of the cache entry points that need no GPU (arguments are checked on the host)."""
import math

import numpy as np
import pytest

from draft_cases import bytes_code, code_bytes, mask_words, random_tree
from oracle import draft_block as orc

torch = pytest.importorskip("torch")


def test_rotation_is_the_decode_blocks():
    from oracle import decode_block
    rng = np.random.default_rng(0)
    x = rng.standard_normal((3, 64))
    want = np.stack([decode_block.rope(x[i], 17, 10000.0) for i in range(3)])
    assert np.allclose(orc.rotate(x, 17, 10000.0), want, rtol=0, atol=1e-12)
    assert np.array_equal(orc.rotate(x, 0, 10000.0), x)
    assert np.allclose(np.linalg.norm(orc.rotate(x, 1234, 500000.0), axis=1), np.linalg.norm(x, axis=1))


def test_e4m3_table_is_torchs():
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(np.nan_to_num(t, nan=-1e9), np.nan_to_num(orc.E4M3, nan=-1e9))


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_codes_are_the_nearest(fmt):
    """Every code is a nearest one (the tie goes to the even one), the largest value gets the largest code, and scale * code
    is within half a step of the value."""
    rng = np.random.default_rng(1)
    x = (rng.standard_normal((200, 64)) * np.exp(3 * rng.standard_normal((200, 1)))).astype(np.float16)
    x[0] = np.arange(64) - 32                                   # top 32: 127/32 k has many ties in int8
    x[1] = 0
    code, scale = orc.encode(x, fmt)
    q = orc.LARGEST[fmt]
    grid = np.arange(-127, 128.0) if fmt == "int8" else np.unique(orc.E4M3[np.isfinite(orc.E4M3)])
    top = np.abs(x.astype(np.float64)).max(-1, keepdims=True)
    y = x.astype(np.float64) * q / np.where(top > 0, top, 1)
    best = np.abs(y[..., None] - grid).min(-1)
    assert np.array_equal(np.abs(y - code), best)
    assert np.array_equal(code[1], np.zeros(64)) and scale[1] == 0
    assert np.array_equal(np.abs(code).max(-1)[2:], np.full(198, q))
    raw = code_bytes(code, fmt)
    assert np.array_equal(bytes_code(raw, fmt), code)
    tie = np.sort(np.abs(y[..., None] - grid), -1)
    even = (raw.astype(int) & 1) == 0
    border = (tie[..., 0] == tie[..., 1]) & (y != 0)
    assert border.any() and even[border].all()


def test_rows_that_are_not_finite_have_scale_nan():
    x = np.ones((3, 64), np.float16)
    x[0, 5], x[1, 6] = np.inf, np.nan
    code, scale = orc.encode(x, "int8")
    assert np.isnan(scale[:2]).all() and scale[2] == np.float32(1) / np.float32(127) and not code[:2].any()


def test_attend_of_a_chain_is_causal_attention():
    rng = np.random.default_rng(2)
    L, T, d = 5, 4, 64
    q, k, v = rng.standard_normal((1, T, 2, d)), rng.standard_normal((1, 1, L + T, d)), rng.standard_normal((1, 1, L + T, d))
    depth, mask = random_tree(rng, T, chain=True)
    out, _, _, _ = orc.attend(q, k, v, [L], [T], depth[None], mask[None])
    for t in range(T):
        s = k[0, 0, :L + t + 1] @ q[0, t, 1] / 8.0
        p = np.exp(s) / np.exp(s).sum()
        assert np.allclose(out[0, t, 1], p @ v[0, 0, :L + t + 1])


def test_attend_masks_window_cap_and_empty_rows():
    rng = np.random.default_rng(3)
    q, k, v = rng.standard_normal((1, 2, 1, 64)), rng.standard_normal((1, 1, 6, 64)), rng.standard_normal((1, 1, 6, 64))
    none = np.zeros((1, 2, 2), bool)
    out, _, _, _ = orc.attend(q, k, v, [0], [2], np.zeros((1, 2), np.int32), none)
    assert not out.any()                                        # sees nothing
    own = none.copy()
    own[0, 1, 1] = True
    out, _, _, _ = orc.attend(q, k, v, [4], [2], np.array([[0, 1]], np.int32), own, window=1)
    assert np.allclose(out[0, 1, 0], v[0, 0, 5]) and not out[0, 0].any()
    # a bias that outweighs everything leaves the nearest key; a cap of nearly nothing leaves the mean
    out, _, _, _ = orc.attend(q, k, v, [4], [2], np.array([[0, 1]], np.int32), own, slopes=[1e6])
    assert np.allclose(out[0, 1, 0], v[0, 0, 5])
    out, _, _, _ = orc.attend(q, k, v, [4], [2], np.array([[0, 1]], np.int32), own, cap=1e-9)
    assert np.allclose(out[0, 0, 0], v[0, 0, :4].mean(0))


def test_mask_words():
    mask = np.zeros((70, 70), bool)
    mask[3, 69] = mask[3, 0] = mask[69, 63] = True
    w = mask_words(mask)
    assert w.shape == (70, 2) and w[3, 0] == 1 and w[3, 1] == 1 << 5 and w[69, 0] == np.uint64(1) << np.uint64(63)


# ---- refusals: nothing is launched, so the addresses need not be real --------------------------------------------------

EINVAL, EUNSUPPORTED = -1, -2
P = 1 << 20


def _kv(**over):
    import paper_2508_18850_amd as lib
    cfg = dict(n_q_heads=8, n_kv_heads=4, head_dim=64, max_batch=4, max_seq=100, format=1, rope_base=10000.0)
    cfg.update(over)
    return lib.KvCache(*cfg.values())


def _pointers(**over):
    import paper_2508_18850_amd as lib
    return lib.cache_pointers(**{**dict(k=P, v=2 * P, k_scale=3 * P, v_scale=4 * P), **over})


def _draft(**over):
    import paper_2508_18850_amd as lib
    return lib.draft(**{**dict(tokens=4, max_len=50), **over})


BAD_CONFIG = [(dict(n_q_heads=0), EINVAL), (dict(n_q_heads=9), EINVAL), (dict(n_kv_heads=0), EINVAL), (dict(head_dim=96), EUNSUPPORTED),
              (dict(max_batch=0), EINVAL), (dict(max_seq=0), EINVAL), (dict(format=3), EINVAL), (dict(format=-1), EINVAL),
              (dict(rope_base=1.0), EINVAL), (dict(rope_base=math.nan), EINVAL), (dict(rope_base=math.inf), EINVAL),
              (dict(max_seq=1 << 24), EUNSUPPORTED), (dict(n_q_heads=1 << 17, n_kv_heads=1 << 17), EUNSUPPORTED)]
BAD_CACHE = [(dict(k=0), EINVAL), (dict(v=0), EINVAL), (dict(k=P + 8), EINVAL), (dict(v=P + 8), EINVAL), (dict(k_scale=0), EINVAL),
             (dict(v_scale=0), EINVAL), (dict(k_scale=P + 2), EINVAL), (dict(v_scale=P + 1), EINVAL)]
BAD_DRAFT = [(dict(tokens=0), EINVAL), (dict(tokens=-1), EINVAL), (dict(max_len=-1), EINVAL), (dict(max_len=97), EINVAL),
             (dict(tokens=2 ** 31 - 1), EINVAL), (dict(row_len=P + 2), EINVAL), (dict(row_tokens=P + 1), EINVAL),
             (dict(depth=P + 2), EINVAL), (dict(tree=P + 4), EINVAL)]


@pytest.mark.parametrize("over,code", BAD_CONFIG, ids=str)
def test_bad_config_is_refused(over, code):
    import ctypes
    import paper_2508_18850_amd as lib
    kv = _kv(**over)
    assert kv.append_rc(1, P, _pointers(), _draft(), 2 * P) == code
    assert kv.read_rc(1, _pointers(), 0, 1, P, P) == code
    assert kv.keep_rc(1, _pointers(), _draft(), P, P) == code
    h = ctypes.c_void_p()
    assert lib.load_library().cf_tree_create(ctypes.byref(lib.TreeConfig(kv.cfg, 4, 0.0, 0)), ctypes.byref(h)) == code and not h


@pytest.mark.parametrize("over,code", BAD_CACHE, ids=str)
def test_bad_cache_is_refused(over, code):
    kv = _kv()
    assert kv.append_rc(1, P, _pointers(**over), _draft(), 2 * P) == code
    assert kv.read_rc(1, _pointers(**over), 0, 1, P, P) == code
    assert kv.keep_rc(1, _pointers(**over), _draft(), P, P) == code


@pytest.mark.parametrize("over,code", BAD_DRAFT, ids=str)
def test_bad_draft_is_refused(over, code):
    kv = _kv()
    assert kv.append_rc(1, P, _pointers(), _draft(**over), 2 * P) == code
    assert kv.keep_rc(1, _pointers(), _draft(**over), P, P) == code


def test_other_refusals():
    import ctypes
    import paper_2508_18850_amd as lib
    kv, c, d = _kv(), _pointers(), _draft()
    for batch in (0, -1, 5):
        assert kv.append_rc(batch, P, c, d, 2 * P) == EINVAL
        assert kv.read_rc(batch, c, 0, 1, P, P) == EINVAL
        assert kv.keep_rc(batch, c, d, P, P) == EINVAL
    for qkv, q_out in ((0, P), (P, 0), (P + 8, P), (P, P + 2)):
        assert kv.append_rc(1, qkv, c, d, q_out) == EINVAL
    assert kv.append_rc(1, P, c, d, P) == EINVAL and kv.append_rc(1, P, c, d, P + 4 * 16 * 64 * 2 - 16) == EINVAL      # q_out on qkv
    for first, rows in ((-1, 1), (0, -1), (100, 1), (0, 101), (2 ** 31 - 1, 2 ** 31 - 1)):
        assert kv.read_rc(1, c, first, rows, P, P) == EINVAL
    for k_out, v_out in ((0, P), (P, 0), (P + 8, P), (P, P + 4)):
        assert kv.read_rc(1, c, 0, 1, k_out, v_out) == EINVAL
    for kept, n_kept, new_len in ((0, P, 0), (P, 0, 0), (P + 2, P, 0), (P, P + 1, 0), (P, 2 * P, 3 * P + 2), (P, 2 * P, P), (P, 2 * P, 2 * P)):
        assert kv.keep_rc(1, c, d, kept, n_kept, new_len) == EINVAL
    assert kv.keep_rc(1, c, _draft(row_len=3 * P), P, 2 * P, 3 * P) == EINVAL
    big = _kv(max_seq=1000)
    assert big.keep_rc(1, c, _draft(tokens=257), P, 2 * P) == EUNSUPPORTED
    many = _kv(n_q_heads=1024, n_kv_heads=1024, max_batch=64)
    assert many.append_rc(64, P, c, d, 2 * P) == EUNSUPPORTED
    raw = lib.load_library()
    assert raw.cf_cache_append(None, 1, P, c, d, P, 0) == EINVAL and raw.cf_cache_append(kv.cfg, 1, P, None, d, P, 0) == EINVAL
    assert raw.cf_cache_append(kv.cfg, 1, P, c, None, P, 0) == EINVAL
    assert raw.cf_tree_create(None, None) == EINVAL and raw.cf_tree_destroy(None) == EINVAL and raw.cf_tree_set_splits(None, 0) == EINVAL
    assert raw.cf_tree_attend(None, 1, P, c, d, None, P, 0) == EINVAL and raw.cf_tree_algorithmic_bytes(None, 1, 1, 1) == 0
    h = ctypes.c_void_p()
    for tokens, cap, window in ((0, 0.0, 0), (257, 0.0, 0), (4, -1.0, 0), (4, math.nan, 0), (4, math.inf, 0), (4, 0.0, -1)):
        assert raw.cf_tree_create(ctypes.byref(lib.TreeConfig(kv.cfg, tokens, cap, window)), ctypes.byref(h)) == EINVAL and not h


def test_algorithmic_bytes():
    import ctypes
    import paper_2508_18850_amd as lib
    raw = lib.load_library()
    cfg = lib.TreeConfig(_kv(format=0).cfg, 8, 0.0, 0)
    assert raw.cf_tree_algorithmic_bytes(ctypes.byref(cfg), 2, 3, 40) == 2 * (2 * 4 * 128 * 43 + 4 * 3 * 8 * 64)
    cfg = lib.TreeConfig(_kv(format=2).cfg, 8, 0.0, 10)
    assert raw.cf_tree_algorithmic_bytes(ctypes.byref(cfg), 1, 3, 40) == 2 * 4 * 68 * 13 + 4 * 3 * 8 * 64


def test_buffers_that_overlap_are_refused():
    import ctypes
    import paper_2508_18850_amd as lib
    kv, c, d = _kv(), _pointers(), _draft()                         # of a batch of 1: 25600 bytes of keys, 1600 of their scales
    end, far = P + 25600, 8 * P
    for where in (P, end - 16, 2 * P, 3 * P, 3 * P + 1600 - 16, 4 * P):
        assert kv.append_rc(1, where, c, d, far) == EINVAL and kv.append_rc(1, far, c, d, where) == EINVAL
        assert kv.read_rc(1, c, 0, 1, where, far) == EINVAL and kv.read_rc(1, c, 0, 1, far, where) == EINVAL
        assert kv.keep_rc(1, c, d, far, far + 64, where) == EINVAL
    assert kv.read_rc(1, c, 0, 2, far, far + 1008) == EINVAL        # 4 heads x 2 rows x 64 fp16 values: 1024 bytes
    for over in (dict(v=end - 16), dict(k_scale=end - 16), dict(v_scale=2 * P), dict(v_scale=3 * P + 1596)):
        assert kv.append_rc(1, far, _pointers(**over), d, 9 * P) == EINVAL
        assert kv.keep_rc(1, _pointers(**over), d, far, far + 64) == EINVAL
    two = _draft(row_len=far + 256)
    for new_len in (far + 252, far + 260, far + 28, far + 68):      # of a batch of 2: on row_len, on kept [2][4], on n_kept
        assert kv.keep_rc(2, c, two, far, far + 64, new_len) == EINVAL
    h = ctypes.c_void_p()
    for cap in (1e-19, 1.2e18):
        cfg = lib.TreeConfig(kv.cfg, 4, cap, 0)
        assert lib.load_library().cf_tree_create(ctypes.byref(cfg), ctypes.byref(h)) == EUNSUPPORTED and not h
