"""What the compiler made of the kernels of a quantised step: the metadata of the code objects in the built library."""
import pytest

pytest.importorskip("msgpack")

from test_kernel_resources import kernels  # noqa: E402

# name in the symbol -> instances: ways of the product, rows to codes by one wavefront or four, {64, 128} dimensions x forms of the score or 16 / 32 rows
COUNTS = {"linear_stream": None, "linear_tiles": None, "quantize_rows": 2, "tree_fours": 6, "cache_append": 16, "cache_read": 8, "cache_keep": 1}


@pytest.mark.parametrize("name", COUNTS)
def test_no_scratch(name):
    """All of them keep what is in flight in registers; a copy to memory would wait for it."""
    mine = {k: v for k, v in kernels().items() if name in k}
    assert mine and (COUNTS[name] is None or len(mine) == COUNTS[name])
    for symbol, kernel in mine.items():
        assert kernel[".private_segment_fixed_size"] == 0 and kernel[".vgpr_spill_count"] == 0, symbol


def test_room_on_a_compute_unit():
    """Two workgroups of the 4-bit attention share a compute unit (160 KB of LDS, 512 registers to a lane's four wavefronts on a SIMD): its loads are
    hidden by the other one.  The product's workgroups have one to themselves at most."""
    for symbol, kernel in kernels().items():
        if "tree_fours" in symbol:
            assert 2 * kernel[".group_segment_fixed_size"] <= 160 * 1024 and kernel[".vgpr_count"] <= 256, symbol
        if "linear_" in symbol:
            assert kernel[".group_segment_fixed_size"] <= 160 * 1024, symbol
