"""How the integer products are dealt to workgroups, on the host (cf_linear_plan.h)."""
import collections

import pytest

import linear_plan

BLOCKS = [(1, 1), (1, 7), (1, 8), (1, 112), (1, 257), (3, 1), (16, 1), (16, 2), (64, 2), (128, 1), (128, 3), (19, 5), (64, 9), (5, 13), (4, 96), (16, 17), (2, 768), (7, 1023)]


@pytest.mark.parametrize("row_blocks,col_blocks", BLOCKS)
def test_every_block_once_and_the_dies_alike(row_blocks, col_blocks):
    """Workgroup i runs on die i mod 8: the fullest die has an eighth of the blocks, rounded up."""
    dealt = linear_plan.stream_blocks(row_blocks, col_blocks)
    mine = [(i % 8, m, n) for i, (m, n) in enumerate(dealt) if n < col_blocks]
    assert sorted((m, n) for _, m, n in mine) == [(m, n) for m in range(row_blocks) for n in range(col_blocks)]
    assert all(m >= 0 and n >= 0 for m, n in dealt)
    assert max(collections.Counter(die for die, _, _ in mine).values()) == -(-row_blocks * col_blocks // 8)
    assert len(dealt) < row_blocks * col_blocks + 8


@pytest.mark.parametrize("row_blocks,col_blocks", BLOCKS)
def test_the_row_blocks_of_an_output_follow_each_other(row_blocks, col_blocks):
    """On a die: the weights of a block of outputs are read while they are in its cache."""
    dealt = linear_plan.stream_blocks(row_blocks, col_blocks)
    for die in range(8):
        mine = [b for b in dealt[die::8] if b[1] < col_blocks]
        for (m, n), (m1, n1) in zip(mine, mine[1:]):
            assert (m1, n1) == (m + 1, n) or (m + 1 == row_blocks and n1 > n)


@pytest.mark.parametrize("rows,n_in,n_out,way", linear_plan.NARROW, ids=str)
def test_ways_of_few_outputs(rows, n_in, n_out, way):
    """What the products of test_gpu_linear_ways.py are divided into, on 256 compute units."""
    assert linear_plan.way_of(rows, n_out) == way and -(-n_out // way.cols) % 8 and rows % way.rows and n_out % way.cols and n_in % 128


@pytest.mark.parametrize("rows,n_in,n_out,way", linear_plan.TILED, ids=str)
def test_ways_of_tiles(rows, n_in, n_out, way):
    """The same, and more steps than a tile has requested at a time, the short one not the last of all dies (each starts at a step of its own)."""
    assert linear_plan.way_of(rows, n_out) == way and rows % way.rows and n_out % way.cols and n_in % 128 and -(-n_in // 128) > 8


def test_every_way_is_tested():
    assert {w for *_, w in linear_plan.NARROW + linear_plan.TILED} == set(linear_plan.ways())
