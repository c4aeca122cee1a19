"""The refusals of cf_cache_append_normed, of the cache calls in 4 bits and of cf_linear_*, each in a call that differs from an accepted one in
what is refused.  Nothing is launched by a refused call, so the addresses need not be real; where there is no GPU the accepted call
comes as far as its launch (CF_EHIP)."""
import ctypes

import pytest

torch = pytest.importorskip("torch")
no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="these addresses are not to be launched on")

EINVAL, EUNSUPPORTED, EHIP = -1, -2, -3
M = 1 << 20                                                          # buffers are below 1 MiB, and at multiples of it
CONFIG = dict(n_q_heads=8, n_kv_heads=4, head_dim=64, max_batch=4, max_seq=100, format=4, rope_base=10000.0)
POINTERS = dict(k=M, v=2 * M, k_scale=3 * M, v_scale=4 * M)
DRAFT = dict(tokens=4, max_len=50, row_len=7 * M, row_tokens=8 * M, depth=9 * M, tree=10 * M, per_row=True)
CALLS = {"append": dict(batch=2, qkv=5 * M, q_out=6 * M), "read": dict(batch=2, first=3, rows=7, k_out=14 * M, v_out=15 * M),
         "keep": dict(batch=2, kept=11 * M, n_kept=12 * M, new_len=13 * M),
         "append_normed": dict(batch=2, qkv=5 * M, q_out=6 * M, q_weight=16 * M, k_weight=17 * M, eps=1e-6)}


def call(name, cfg=None, cache=None, draft=None, **over):
    import paper_2508_18850_amd as lib
    kv = lib.KvCache(**{**CONFIG, **(cfg or {})})
    c, d = lib.cache_pointers(**{**POINTERS, **(cache or {})}), lib.draft(**{**DRAFT, **(draft or {})})
    a = {**CALLS[name], **over}
    if name == "append":
        return kv.append_rc(a["batch"], a["qkv"], c, d, a["q_out"])
    if name == "append_normed":
        return kv.append_normed_rc(a["batch"], a["qkv"], a["q_weight"], a["k_weight"], a["eps"], c, d, a["q_out"])
    if name == "read":
        return kv.read_rc(a["batch"], c, a["first"], a["rows"], a["k_out"], a["v_out"])
    return kv.keep_rc(a["batch"], c, d, a["kept"], a["n_kept"], a["new_len"])


@no_gpu
@pytest.mark.parametrize("fmt", [0, 1, 2, 4])
@pytest.mark.parametrize("name", CALLS)
def test_the_calls_that_the_refused_ones_differ_from(name, fmt):
    cfg = dict(format=fmt)
    if fmt == 0:
        assert call(name, cfg, cache=dict(k_scale=0, v_scale=0)) == EHIP
    assert call(name, cfg) == EHIP and call(name, cfg, batch=4) == EHIP and call(name, dict(format=fmt, head_dim=128, max_seq=55)) == EHIP
    if name == "append_normed":
        assert call(name, cfg, eps=0.0) == EHIP and call(name, cfg, k_weight=16 * M) == EHIP


@pytest.mark.parametrize("fmt", [3, 5, 8, -4])
@pytest.mark.parametrize("name", CALLS)
def test_formats(name, fmt):
    assert call(name, dict(format=fmt)) == EINVAL


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("head_dim", [64, 128])
def test_slices_end_below_2_to_the_30_values(name, head_dim):
    """(With a batch of 0 an accepted configuration is refused for the batch.)"""
    for max_seq, code in (((1 << 30) // head_dim - 1, EINVAL), ((1 << 30) // head_dim, EUNSUPPORTED)):
        assert call(name, dict(head_dim=head_dim, max_seq=max_seq), batch=0) == code


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("over", [dict(k=0), dict(v=0), dict(k_scale=0), dict(v_scale=0), dict(k=M + 8), dict(v=2 * M + 8), dict(k_scale=3 * M + 2),
                                  dict(v_scale=4 * M + 1)], ids=str)
def test_pointers_of_a_cache(name, over):
    assert call(name, cache=over) == EINVAL


@pytest.mark.parametrize("over", [dict(qkv=0), dict(q_out=0), dict(q_weight=0), dict(k_weight=0), dict(q_weight=16 * M + 8), dict(k_weight=17 * M + 2), dict(eps=-1e-9),
                                  dict(eps=float("nan")), dict(eps=float("inf")), dict(batch=0), dict(batch=5), dict(qkv=5 * M + 8), dict(q_out=6 * M + 4),
                                  dict(draft=dict(tokens=0)), dict(draft=dict(max_len=97)), dict(draft=dict(depth=9 * M + 2))], ids=str)
def test_arguments_of_an_append_with_norms(over):
    assert call("append_normed", **over) == EINVAL


# of a cache of 2 rows, 4 heads, 100 cached tokens of 64 values; in 4 bits and in fp16
def held(fmt):
    return dict(k=800 * {4: 32, 0: 128, 1: 64}[fmt], v=800 * {4: 32, 0: 128, 1: 64}[fmt], **({} if fmt == 0 else {n: 800 * {4: 2, 1: 4}[fmt] for n in ("k_scale", "v_scale")}))


@pytest.mark.parametrize("fmt", [0, 1, 4])
@pytest.mark.parametrize("name,sizes", [("append_normed", dict(qkv=2 * 4 * 16 * 64 * 2, q_out=2 * 4 * 8 * 64 * 2, q_weight=128, k_weight=128)),
                                        ("append", dict(qkv=2 * 4 * 16 * 64 * 2, q_out=2 * 4 * 8 * 64 * 2)),
                                        ("read", dict(k_out=2 * 4 * 7 * 64 * 2, v_out=2 * 4 * 7 * 64 * 2))])
def test_buffers_on_the_cache(name, sizes, fmt):
    """From the first byte to the last: one step further it is accepted (where there is no GPU, as far as the launch)."""
    for arg, size in sizes.items():
        for part, n in held(fmt).items():
            at = POINTERS[part]
            for where, apart in ((at, False), (at + (n - 1) // 16 * 16, False), (at - size + 16, False), (at + (n + 15) // 16 * 16, True), (at - size, True)):
                if not apart:
                    assert call(name, dict(format=fmt), **{arg: where}) == EINVAL, (arg, part, where - at)
                elif not torch.cuda.is_available():
                    assert call(name, dict(format=fmt), **{arg: where}) == EHIP, (arg, part, where - at)


def test_weights_on_the_queries():
    for w in ("q_weight", "k_weight"):
        for where, apart in ((6 * M, False), (6 * M + 8192 - 16, False), (6 * M - 112, False), (6 * M + 8192, True), (6 * M - 128, True)):
            if not apart:
                assert call("append_normed", **{w: where}) == EINVAL
            elif not torch.cuda.is_available():
                assert call("append_normed", **{w: where}) == EHIP


@pytest.mark.parametrize("name", ["append", "append_normed", "keep"])
def test_a_cache_whose_buffers_overlap(name):
    for part, n in held(4).items():
        for other in POINTERS:
            if other != part:
                at = POINTERS[part]
                assert call(name, cache={other: at}) == EINVAL and call(name, cache={other: at + (n - 1) // 16 * 16}) == EINVAL, (part, other)
                if not torch.cuda.is_available():
                    assert call(name, cache={other: at + (n + 15) // 16 * 16}) == EHIP, (part, other)


def test_missing_structs():
    import paper_2508_18850_amd as lib
    raw, kv = lib.load_library(), lib.KvCache(**CONFIG)
    c, d = lib.cache_pointers(**POINTERS), lib.draft(**DRAFT)
    args = (5 * M, 16 * M, 17 * M, 1e-6)
    assert raw.cf_cache_append_normed(None, 1, *args, c, d, 6 * M, 0) == EINVAL and raw.cf_cache_append_normed(kv.cfg, 1, *args, None, d, 6 * M, 0) == EINVAL
    assert raw.cf_cache_append_normed(kv.cfg, 1, *args, c, None, 6 * M, 0) == EINVAL


def test_bytes_of_an_attention_in_4_bits():
    """Two heads of 128 values: 64 + 4 bytes for a key and as much for its value; queries and results fp16."""
    import paper_2508_18850_amd as lib
    cfg = lib.TreeConfig(lib.CacheConfig(4, 2, 128, 1, 1000, 4, 10000.0), 8, 0.0, 0)
    assert lib.load_library().cf_tree_algorithmic_bytes(ctypes.byref(cfg), 1, 3, 500) == 2 * 2 * 68 * 503 + 4 * 3 * 4 * 128


# ---- integer products -----------------------------------------------------------------------------------------------------------

def quantize(**over):
    import paper_2508_18850_amd as lib
    a = {**dict(rows=3, n=64, x=M, codes=2 * M, scale=3 * M), **over}
    return lib.quantize_rows_rc(a["rows"], a["n"], a["x"], a["codes"], a["scale"])


@no_gpu
def test_accepted_rows():
    assert quantize() == EHIP and quantize(n=16, rows=1) == EHIP and quantize(n=5008) == EHIP and quantize(rows=0) == 0


@pytest.mark.parametrize("over,code", [(dict(rows=-1), EINVAL), (dict(n=0), EINVAL), (dict(n=-16), EINVAL), (dict(n=24), EINVAL), (dict(x=0), EINVAL), (dict(codes=0), EINVAL),
                                       (dict(scale=0), EINVAL), (dict(x=M + 8), EINVAL), (dict(codes=2 * M + 8), EINVAL), (dict(scale=3 * M + 2), EINVAL),
                                       (dict(rows=(1 << 23) + 1, n=16, codes=1 << 40, scale=1 << 42), EUNSUPPORTED), (dict(rows=0, n=8), EINVAL), (dict(rows=0, x=0), EINVAL),
                                       (dict(codes=M), EINVAL), (dict(codes=M + 368), EINVAL), (dict(codes=M - 176), EINVAL), (dict(scale=M + 380), EINVAL), (dict(scale=M - 8), EINVAL),
                                       (dict(scale=2 * M), EINVAL), (dict(scale=2 * M + 188), EINVAL), (dict(scale=2 * M - 8), EINVAL)], ids=str)
def test_refused_rows(over, code):
    assert quantize(**over) == code


@no_gpu
def test_rows_side_by_side():
    assert quantize(codes=M + 384) == EHIP and quantize(codes=M - 192) == EHIP and quantize(scale=M + 384) == EHIP and quantize(scale=2 * M + 192) == EHIP
    assert quantize(scale=2 * M - 12) == EHIP


@pytest.mark.parametrize("sizes,code", [((0, 64, 1), EINVAL), ((8, 64, 1), EINVAL), ((-16, 64, 1), EINVAL), ((72, 64, 1), EINVAL), ((64, 0, 1), EINVAL), ((64, 12, 1), EINVAL),
                                        ((64, -8, 1), EINVAL), ((64, 64, 0), EINVAL), ((64, 64, -1), EINVAL), ((131072, 64, 1), EUNSUPPORTED), ((65536, 32768, 1), EUNSUPPORTED),
                                        ((64, 64, (1 << 23) + 1), EUNSUPPORTED)], ids=str)
def test_refused_handles(sizes, code):
    import paper_2508_18850_amd as lib
    h = ctypes.c_void_p()
    cfg = lib.LinearConfig(*sizes)
    assert lib.load_library().cf_linear_create(ctypes.byref(cfg), ctypes.byref(h)) == code and not h


def test_missing_handles():
    import paper_2508_18850_amd as lib
    raw, h = lib.load_library(), ctypes.c_void_p()
    cfg = lib.LinearConfig(64, 64, 1)
    assert raw.cf_linear_create(None, ctypes.byref(h)) == EINVAL and raw.cf_linear_create(ctypes.byref(cfg), None) == EINVAL
    assert raw.cf_linear_destroy(None) == EINVAL and raw.cf_linear_forward(None, 1, M, 2 * M, 3 * M, 4 * M, 5 * M, 0) == EINVAL
    assert raw.cf_linear_algorithmic_bytes(ctypes.byref(cfg), 3) == 3 * 64 + 64 * 64 + 4 * 67 + 2 * 3 * 64 and raw.cf_linear_algorithmic_bytes(None, 3) == 0
