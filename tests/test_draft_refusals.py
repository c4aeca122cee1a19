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
