"""The refusals of cf_cache_append, cf_cache_read and cf_cache_keep, each in a call that differs from an accepted one in what is refused.

All buffers lie apart, so that no other check refuses the call.  Nothing is launched by a refused call, so the addresses need not be
real; where there is no GPU the accepted call comes as far as its launch (CF_EHIP).  That the same calls run on a GPU is tested in
test_gpu_tree_calls.py."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

EINVAL, EUNSUPPORTED, EHIP = -1, -2, -3
M = 1 << 20                                                          # buffers are below 1 MiB, and at multiples of it


def config(**over):
    return {**dict(n_q_heads=8, n_kv_heads=4, head_dim=64, max_batch=4, max_seq=100, format=1, rope_base=10000.0), **over}


@pytest.mark.parametrize("fmt", [0, 1, 2])
@pytest.mark.parametrize("head_dim", [64, 128])
def test_slices_end_below_2_to_the_30_values(fmt, head_dim):
    """In every format.  (With a batch of 0 an accepted configuration is refused for the batch.)"""
    import paper_2508_18850_amd as lib
    for max_seq, code in (((1 << 30) // head_dim - 1, EINVAL), ((1 << 30) // head_dim, EUNSUPPORTED)):
        kv = lib.KvCache(**config(format=fmt, head_dim=head_dim, max_seq=max_seq))
        cache, draft = lib.cache_pointers(M, 2 * M, 3 * M, 4 * M), lib.draft(1, 10)
        assert kv.append_rc(0, 5 * M, cache, draft, 6 * M) == code
        assert kv.read_rc(0, cache, 0, 1, 5 * M, 6 * M) == code
        assert kv.keep_rc(0, cache, draft, 5 * M, 6 * M) == code
    for heads, code in ((65535, EINVAL), (65536, EUNSUPPORTED)):
        kv = lib.KvCache(**config(format=fmt, head_dim=head_dim, n_q_heads=heads, n_kv_heads=1))
        assert kv.append_rc(0, 5 * M, cache, lib.draft(1, 10), 6 * M) == code


POINTERS = dict(k=M, v=2 * M, k_scale=3 * M, v_scale=4 * M)
DRAFT = dict(tokens=4, max_len=50, row_len=7 * M, row_tokens=8 * M, depth=9 * M, tree=10 * M, per_row=True)
CALLS = {"append": dict(batch=2, qkv=5 * M, q_out=6 * M), "read": dict(batch=2, first=3, rows=7, k_out=14 * M, v_out=15 * M),
         "keep": dict(batch=2, kept=11 * M, n_kept=12 * M, new_len=13 * M)}


def call(name, cfg=None, cache=None, draft=None, **over):
    import paper_2508_18850_amd as lib
    kv = lib.KvCache(**config(**(cfg or {})))
    c, d = lib.cache_pointers(**{**POINTERS, **(cache or {})}), lib.draft(**{**DRAFT, **(draft or {})})
    a = {**CALLS[name], **over}
    if name == "append":
        return kv.append_rc(a["batch"], a["qkv"], c, d, a["q_out"])
    if name == "read":
        return kv.read_rc(a["batch"], c, a["first"], a["rows"], a["k_out"], a["v_out"])
    return kv.keep_rc(a["batch"], c, d, a["kept"], a["n_kept"], a["new_len"])


@pytest.mark.skipif(torch.cuda.is_available(), reason="these addresses are not to be launched on")
@pytest.mark.parametrize("fmt", [0, 1, 2])
@pytest.mark.parametrize("name", CALLS)
def test_the_calls_that_the_refused_ones_differ_from(name, fmt):
    """Accepted, as are their limits: what follows is refused for the one thing in which it differs."""
    cfg = dict(format=fmt)
    if fmt == 0:
        assert call(name, cfg, cache=dict(k_scale=0, v_scale=0)) == EHIP
    assert call(name, cfg) == EHIP and call(name, cfg, batch=4) == EHIP and call(name, cfg, batch=1) == EHIP
    none = dict(row_len=0, row_tokens=0, depth=0, tree=0, per_row=False)
    if name == "read":
        assert call(name, cfg, first=0, rows=100) == EHIP and call(name, cfg, first=99, rows=1) == EHIP
    else:
        assert call(name, cfg, draft=none) == EHIP and call(name, cfg, draft=dict(max_len=96)) == EHIP and call(name, cfg, draft=dict(max_len=0)) == EHIP
        assert call(name, cfg, draft=dict(tokens=1)) == EHIP and call(name, cfg, draft=dict(tokens=50)) == EHIP
    if name == "keep":
        assert call(name, cfg, new_len=0) == EHIP and call(name, dict(max_seq=1000), draft=dict(tokens=256)) == EHIP


def test_a_read_of_no_rows_is_accepted_without_a_launch():
    assert call("read", rows=0) == 0 and call("read", rows=0, first=100) == 0


@pytest.mark.parametrize("over,code", [
    (dict(n_q_heads=0), EINVAL), (dict(n_q_heads=-8), EINVAL), (dict(n_q_heads=9), EINVAL), (dict(n_kv_heads=0), EINVAL), (dict(n_kv_heads=3), EINVAL),
    (dict(n_kv_heads=-4), EINVAL), (dict(head_dim=96), EUNSUPPORTED), (dict(head_dim=0), EUNSUPPORTED), (dict(head_dim=256), EUNSUPPORTED), (dict(max_batch=0), EINVAL),
    (dict(max_seq=0), EINVAL), (dict(max_seq=-1), EINVAL), (dict(format=3), EINVAL), (dict(format=-1), EINVAL), (dict(rope_base=1.0), EINVAL),
    (dict(rope_base=-5.0), EINVAL), (dict(rope_base=float("nan")), EINVAL), (dict(rope_base=float("inf")), EINVAL)], ids=str)
def test_configurations(over, code):
    """By a read of no rows, which nothing else refuses (but for max_batch 0, which leaves no batch to read), and by all calls."""
    import paper_2508_18850_amd as lib
    assert call("read", over, first=0, rows=0) == code
    for name in CALLS:
        assert call(name, over) == code
    h = ctypes.c_void_p()
    tree = lib.TreeConfig(lib.CacheConfig(*config(**over).values()), 4, 0.0, 0)
    assert lib.load_library().cf_tree_create(ctypes.byref(tree), ctypes.byref(h)) == code and not h


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("over", [dict(k=0), dict(v=0), dict(k_scale=0), dict(v_scale=0), dict(k=M + 8), dict(v=2 * M + 8), dict(k=M + 1),
                                  dict(k_scale=3 * M + 2), dict(v_scale=4 * M + 1)], ids=str)
def test_pointers_of_a_cache(name, over):
    assert call(name, cache=over) == EINVAL


@pytest.mark.parametrize("name", ["append", "keep"])
@pytest.mark.parametrize("over", [dict(tokens=0), dict(tokens=-1), dict(max_len=-1), dict(max_len=97), dict(tokens=51), dict(tokens=2 ** 31 - 1),
                                  dict(tokens=2 ** 31 - 1, max_len=2 ** 31 - 1), dict(row_len=7 * M + 2), dict(row_tokens=8 * M + 1),
                                  dict(depth=9 * M + 2), dict(tree=10 * M + 4)], ids=str)
def test_drafts(name, over):
    assert call(name, draft=over) == EINVAL


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("batch", [0, -1, 5])
def test_batches(name, batch):
    assert call(name, batch=batch) == EINVAL


def test_heads_of_a_call():
    cfg = dict(n_q_heads=1024, n_kv_heads=1024, max_batch=64, max_seq=54)
    apart = dict(k=M << 10, v=M << 11, k_scale=M << 12, v_scale=M << 13)
    for name in CALLS:
        assert call(name, cfg, cache=apart, batch=64) == EUNSUPPORTED


@pytest.mark.parametrize("name,over", [
    ("append", dict(qkv=0)), ("append", dict(q_out=0)), ("append", dict(qkv=5 * M + 8)), ("append", dict(q_out=6 * M + 2)),
    ("read", dict(k_out=0)), ("read", dict(v_out=0)), ("read", dict(k_out=14 * M + 8)), ("read", dict(v_out=15 * M + 4)),
    ("read", dict(first=-1)), ("read", dict(rows=-1)), ("read", dict(first=94)), ("read", dict(first=100, rows=1)), ("read", dict(first=0, rows=101)),
    ("read", dict(first=2 ** 31 - 1, rows=2 ** 31 - 1)),
    ("keep", dict(kept=0)), ("keep", dict(n_kept=0)), ("keep", dict(kept=11 * M + 2)), ("keep", dict(n_kept=12 * M + 1)), ("keep", dict(new_len=13 * M + 2))], ids=str)
def test_arguments(name, over):
    assert call(name, **over) == EINVAL


def test_most_tokens_of_a_keep():
    assert call("keep", dict(max_seq=1000), draft=dict(tokens=257)) == EUNSUPPORTED


# What a call of `name` reads and writes besides the cache, in bytes, with the configuration and the calls above.
EXTENT = {"append": dict(qkv=2 * 4 * 16 * 64 * 2, q_out=2 * 4 * 8 * 64 * 2), "read": dict(k_out=2 * 4 * 7 * 64 * 2, v_out=2 * 4 * 7 * 64 * 2)}
CACHE = dict(k=2 * 4 * 100 * 64, v=2 * 4 * 100 * 64, k_scale=2 * 4 * 100 * 4, v_scale=2 * 4 * 100 * 4)


@pytest.mark.parametrize("name", ["append", "read"])
def test_buffers_on_the_cache_or_on_each_other(name):
    """From the first byte to the last: one step further it is accepted (where there is no GPU, as far as the launch)."""
    free = [] if torch.cuda.is_available() else [EHIP]
    for arg, size in EXTENT[name].items():
        for part, held in CACHE.items():
            at = POINTERS[part]
            step = 16
            for where, apart in ((at, False), (at + (held - 1) // step * step, False), (at - size + step, False), (at + (held + step - 1) // step * step, True), (at - size, True)):
                if not apart:
                    assert call(name, **{arg: where}) == EINVAL, (arg, part, where - at)
                elif free:
                    assert call(name, **{arg: where}) == EHIP, (arg, part, where - at)
    (one, one_size), (two, _) = EXTENT[name].items()
    start = CALLS[name][one]
    assert call(name, **{two: start}) == EINVAL and call(name, **{two: start + one_size - 16}) == EINVAL
    if free:
        assert call(name, **{two: start + one_size}) == EHIP


@pytest.mark.parametrize("name", ["append", "keep"])
def test_a_cache_whose_buffers_overlap(name):
    for part, at in POINTERS.items():
        for other in POINTERS:
            if other != part:
                assert call(name, cache={other: at}) == EINVAL, (part, other)
                last = (CACHE[part] - 1) // 16 * 16
                assert call(name, cache={other: at + last}) == EINVAL, (part, other)
                if not torch.cuda.is_available():
                    assert call(name, cache={other: at + (CACHE[part] + 15) // 16 * 16}) == EHIP, (part, other)


def test_new_lengths_on_another_array():
    for array, held in ((7 * M, 8), (8 * M, 8), (11 * M, 2 * 4 * 4), (12 * M, 8), *((POINTERS[n], CACHE[n]) for n in CACHE)):
        for where in (array, array + held - 4, array - 4):
            assert call("keep", new_len=where) == EINVAL, (array // M, where - array)
        if not torch.cuda.is_available():
            assert call("keep", new_len=array + held) == EHIP and call("keep", new_len=array - 8) == EHIP


def test_missing_structs():
    import paper_2508_18850_amd as lib
    raw, kv = lib.load_library(), lib.KvCache(**config())
    c, d = lib.cache_pointers(**POINTERS), lib.draft(**DRAFT)
    assert raw.cf_cache_append(None, 1, 5 * M, c, d, 6 * M, 0) == EINVAL and raw.cf_cache_append(kv.cfg, 1, 5 * M, None, d, 6 * M, 0) == EINVAL
    assert raw.cf_cache_append(kv.cfg, 1, 5 * M, c, None, 6 * M, 0) == EINVAL
    assert raw.cf_cache_read(None, 1, c, 0, 1, 14 * M, 15 * M, 0) == EINVAL and raw.cf_cache_read(kv.cfg, 1, None, 0, 1, 14 * M, 15 * M, 0) == EINVAL
    assert raw.cf_cache_keep(None, 1, c, d, 11 * M, 12 * M, 0, 0) == EINVAL and raw.cf_cache_keep(kv.cfg, 1, None, d, 11 * M, 12 * M, 0, 0) == EINVAL
    assert raw.cf_cache_keep(kv.cfg, 1, c, None, 11 * M, 12 * M, 0, 0) == EINVAL
