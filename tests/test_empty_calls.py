"""Calls for no rows: they do nothing, and their pointers are checked as in any other call (an empty tensor's address may be null)."""
import pytest

import paper_2508_18850_amd as lib

EINVAL, M = -1, 1 << 20                                              # nothing is launched, so the addresses need not be real


@pytest.mark.parametrize("missing", [None, "x", "codes", "scale"])
def test_no_rows_to_quantise(missing):
    at = {n: 0 if n == missing else (i + 1) * M for i, n in enumerate(("x", "codes", "scale"))}
    assert lib.quantize_rows_rc(0, 64, at["x"], at["codes"], at["scale"]) == (EINVAL if missing else 0)


@pytest.mark.parametrize("missing", [None, "k_out", "v_out"])
@pytest.mark.parametrize("fmt", [0, 1, 2, 4])
def test_no_rows_to_read(missing, fmt):
    at = {n: 0 if n == missing else (i + 5) * M for i, n in enumerate(("k_out", "v_out"))}
    kv = lib.KvCache(4, 2, 64, 2, 100, fmt, 10000.0)
    assert kv.read_rc(2, lib.cache_pointers(M, 2 * M, 3 * M, 4 * M), 100, 0, at["k_out"], at["v_out"]) == (EINVAL if missing else 0)
