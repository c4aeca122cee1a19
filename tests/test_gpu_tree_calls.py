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
