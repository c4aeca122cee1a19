"""Handles and refusals of cf_tree_attend, and the calls that the cache's refusals are compared with."""
import numpy as np
import pytest

from test_gpu_tree import Case

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def test_small_handles_have_small_workspaces():
    """One token of one head of 64 dimensions over up to 200 rows: two parts of 16 rows of partial results, some kilobytes."""
    import paper_2508_18850_amd as lib
    torch.cuda.synchronize()
    lib.TreeAttention(1, 1, 64, 1, 200, 0, 10000.0, 1).close()
    before = torch.cuda.mem_get_info()[0]
    handles = [lib.TreeAttention(1, 1, 64, 1, 200, 0, 10000.0, 1) for _ in range(8)]
    held = before - torch.cuda.mem_get_info()[0]
    for h in handles:
        h.close()
    assert held <= 8 * (2 << 20), held                              # (memory is handed out in pieces of 2 MiB)


@pytest.mark.parametrize("fmt", ["f16", "e4m3", "int8"])
@pytest.mark.parametrize("nq,nkv,B,rows,T", [(1, 1, 1, 200, 1), (8, 1, 1, 1000, 40), (4, 2, 3, 400, 17), (64, 8, 1, 5000, 4), (2, 1, 1, 3000, 130)], ids=str)
def test_workspaces_hold_every_division(fmt, nq, nkv, B, rows, T):
    """Handles as small as their largest call, at every limit on the parts, with and without forms of the score."""
    for window in (0, rows):
        c = Case(fmt, nq, nkv, 64, [rows - T] * B, T, window=window, seed=60, extra=0)
        for splits in (0, 64, 2):
            c.tree.set_splits(splits)
            c.check()


# ---- refusals: each call differs from one that runs in what is refused ------------------------------------------------------

M = 1 << 20
EINVAL, EUNSUPPORTED = -1, -2


class Calls:
    """Buffers apart from each other at multiples of 1 MiB, all zero but for the counts, and a handle."""

    def __init__(self, fmt=1, batch=2, **cfg):
        import paper_2508_18850_amd as lib
        self.lib, self.batch = lib, batch
        self.cfg = {**dict(n_q_heads=8, n_kv_heads=4, head_dim=64, max_batch=4, max_seq=100, format=fmt, rope_base=10000.0), **cfg}
        self.mem = torch.zeros(17 * M, dtype=torch.uint8, device="cuda")
        self.base = (self.mem.data_ptr() + M - 1) // M * M - M       # buffer n is at base + n M
        self.tree = lib.TreeAttention(**self.cfg, max_tokens=8)
        self.kv = lib.KvCache(**self.cfg)
        at = 8 * M + self.base - self.mem.data_ptr()
        self.mem[at:at + 16].view(torch.int32).fill_(4)

    def at(self, n):
        return self.base + n if n else 0

    def cache(self, **over):
        return self.lib.cache_pointers(**{k: self.at(n) for k, n in {**dict(k=M, v=2 * M, k_scale=3 * M, v_scale=4 * M), **over}.items()})

    def draft(self, tokens=4, max_len=50, per_row=True, **over):
        return self.lib.draft(tokens, max_len, per_row=per_row, **{k: self.at(n) for k, n in {**dict(row_len=7 * M, row_tokens=8 * M, depth=9 * M, tree=10 * M), **over}.items()})

    def attend(self, batch=2, q=5 * M, out=6 * M, slopes=14 * M, cache=None, draft=None):
        rc = self.tree.attend_rc(batch, self.at(q), self.cache(**(cache or {})), self.draft(**(draft or {})), self.at(slopes), self.at(out),
                                 torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        return rc


@pytest.mark.parametrize("fmt", [0, 1, 2])
def test_accepted_calls_of_attend(fmt):
    c = Calls(fmt)
    assert c.attend() == 0 and c.attend(batch=1) == 0 and c.attend(batch=4) == 0 and c.attend(slopes=0) == 0
    assert c.attend(draft=dict(row_len=0, row_tokens=0, depth=0, tree=0, per_row=False)) == 0
    assert c.attend(draft=dict(tokens=8)) == 0 and c.attend(draft=dict(tokens=1)) == 0 and c.attend(draft=dict(max_len=96)) == 0 and c.attend(draft=dict(max_len=0)) == 0
    if fmt == 0:
        assert c.attend(cache=dict(k_scale=0, v_scale=0)) == 0
    c.tree.close()


@pytest.mark.parametrize("over", [
    dict(batch=0), dict(batch=-1), dict(batch=5), dict(q=0), dict(out=0), dict(q=5 * M + 8), dict(out=6 * M + 2), dict(slopes=14 * M + 2),
    *(dict(cache=x) for x in (dict(k=0), dict(v=0), dict(k_scale=0), dict(v_scale=0), dict(k=M + 8), dict(v=2 * M + 4), dict(k_scale=3 * M + 1), dict(v_scale=4 * M + 2))),
    *(dict(draft=x) for x in (dict(tokens=0), dict(tokens=9), dict(tokens=-1), dict(max_len=-1), dict(max_len=97), dict(row_len=7 * M + 1), dict(row_tokens=8 * M + 2),
                              dict(depth=9 * M + 2), dict(tree=10 * M + 4)))], ids=str)
def test_refused_calls_of_attend(over):
    c = Calls()
    assert c.attend() == 0 and c.attend(**over) == EINVAL
    c.tree.close()


def test_results_on_other_buffers_are_refused():
    """out on q or on a part of the cache, from the first byte to the last, and accepted one step further."""
    c = Calls()
    size = 2 * 4 * 8 * 64 * 2
    for start, held in ((5 * M, size), (M, 2 * 4 * 100 * 64), (2 * M, 2 * 4 * 100 * 64), (3 * M, 3200), (4 * M, 3200)):
        assert c.attend(out=start) == EINVAL and c.attend(out=start + held - 16) == EINVAL
        assert c.attend(out=start + held) == 0
        if start > M:                                               # (in front of buffer 1 there is none)
            assert c.attend(out=start - size + 16) == EINVAL and c.attend(out=start - size) == 0
    c.tree.close()


def test_heads_and_handles():
    import ctypes
    c = Calls()
    for n in (-1, 65):
        with pytest.raises(c.lib.CfError):
            c.tree.set_splits(n)
    for n in (64, 1, 0):
        c.tree.set_splits(n)
    h = ctypes.c_void_p()
    create = lambda tokens, cap, window: c.lib.load_library().cf_tree_create(  # noqa: E731
        ctypes.byref(c.lib.TreeConfig(c.lib.CacheConfig(*c.cfg.values()), tokens, cap, window)), ctypes.byref(h))
    for args in ((1, 0.0, 0), (256, 0.0, 0), (4, 2.0 ** -60, 0), (4, 2.0 ** 60, 2 ** 31 - 1)):
        assert create(*args) == 0 and c.lib.load_library().cf_tree_destroy(h) == 0
    for args, code in (((0, 0.0, 0), EINVAL), ((257, 0.0, 0), EINVAL), ((4, -1.0, 0), EINVAL), ((4, float("nan"), 0), EINVAL), ((4, float("inf"), 0), EINVAL),
                       ((4, 0.0, -1), EINVAL), ((4, 2.0 ** -61, 0), EUNSUPPORTED), ((4, 2.0 ** 61, 0), EUNSUPPORTED)):
        assert create(*args) == code and not h
    many = c.lib.TreeAttention(1024, 1024, 64, 64, 100, 1, 10000.0, 8)
    assert many.attend_rc(64, c.at(5 * M), c.cache(), c.draft(), 0, c.at(6 * M)) == EUNSUPPORTED
    many.close()
    c.tree.close()


@pytest.mark.parametrize("fmt", [0, 1, 2])
def test_accepted_calls_on_a_cache(fmt):
    """The calls from which those of test_draft_refusals.py differ, and those of its limits that fit these buffers, run."""
    c = Calls(fmt)
    s = torch.cuda.current_stream().cuda_stream
    none = dict(row_len=0, row_tokens=0, depth=0, tree=0, per_row=False)
    for batch, draft in ((2, {}), (4, {}), (1, {}), (2, none), (2, dict(max_len=96)), (2, dict(max_len=0)), (2, dict(tokens=1)), (2, dict(tokens=50))):
        assert c.kv.append_rc(batch, c.at(5 * M), c.cache(), c.draft(**draft), c.at(6 * M), s) == 0
        assert c.kv.keep_rc(batch, c.cache(), c.draft(**draft), c.at(11 * M), c.at(12 * M), c.at(13 * M), s) == 0
        torch.cuda.synchronize()
    assert c.kv.keep_rc(2, c.cache(), c.draft(), c.at(11 * M), c.at(12 * M), 0, s) == 0
    for first, rows in ((3, 7), (0, 100), (99, 1), (100, 0)):
        assert c.kv.read_rc(2, c.cache(), first, rows, c.at(14 * M), c.at(15 * M), s) == 0
        torch.cuda.synchronize()
    if fmt == 0:
        plain = c.cache(k_scale=0, v_scale=0)
        assert c.kv.append_rc(2, c.at(5 * M), plain, c.draft(), c.at(6 * M), s) == 0 and c.kv.read_rc(2, plain, 3, 7, c.at(14 * M), c.at(15 * M), s) == 0
        assert c.kv.keep_rc(2, plain, c.draft(), c.at(11 * M), c.at(12 * M), 0, s) == 0
    torch.cuda.synchronize()
    c.tree.close()
