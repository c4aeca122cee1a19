"""Every way to divide an integer product, at sizes that the rule gives to it (tests/test_linear_plan.py): sums, rows and outputs that end inside a block.
Sums are whole numbers and the roundings in a fixed order, so that nothing has a tolerance."""
import pytest

import linear_plan
from test_gpu_linear import Product

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,n_in,n_out,way", linear_plan.NARROW, ids=str)
def test_many_rows_and_few_outputs(rows, n_in, n_out, way):
    Product(rows, n_in, n_out, full=True).check()


@pytest.mark.parametrize("rows,n_in,n_out,way", linear_plan.TILED, ids=str)
def test_tiles(rows, n_in, n_out, way):
    Product(rows, n_in, n_out, full=True).check()


TILES = linear_plan.TILED[:4]                                       # one for each kind


@pytest.mark.parametrize("n_in", [16, 112, 128, 144, 272, 400])
@pytest.mark.parametrize("rows,_,n_out,way", TILES, ids=str)
def test_short_sums_in_tiles(rows, _, n_out, way, n_in):
    """Fewer steps than a tile requests ahead, and one or two more."""
    Product(rows, n_in, n_out, full=True).check()


@pytest.mark.parametrize("rows,_,n_out,way", TILES, ids=str)
def test_largest_sums_in_tiles(rows, _, n_out, way):
    """-128 times -128 as often as there may be inputs, and beside them the most negative sums."""
    c = Product(rows, 131056, n_out)
    c.x.fill_(-128)
    c.w.fill_(-128)
    c.w[n_out - 3] = 127
    c.xs.fill_(2.0 ** -9)
    c.ws.fill_(2.0 ** -9)
    c.check()


@pytest.mark.parametrize("rows,n_in,n_out,way", TILES, ids=str)
def test_special_scales_in_tiles(rows, n_in, n_out, way):
    """NaN rows and outputs stay apart, in the first blocks and in the last ones; zeros, infinities and results beyond fp16."""
    c = Product(rows, n_in, n_out)
    c.xs[0], c.xs[1], c.xs[rows - 1] = float("nan"), 0.0, float("nan")
    c.ws[5], c.ws[6], c.ws[n_out - 1] = float("inf"), 1e30, float("nan")
    c.call()
    torch.cuda.synchronize()
    want, got = c.want(), c.out[:rows]
    assert torch.equal(torch.nan_to_num(got, 3.0, 4.0, 5.0), torch.nan_to_num(want, 3.0, 4.0, 5.0)) and torch.equal(got.isnan(), want.isnan())
    assert got[0].isnan().all() and got[rows - 1].isnan().all() and got[:, n_out - 1].isnan().all() and got[2:rows - 1, 7:n_out - 1].isfinite().all()
    assert (c.out[rows:] == 7.0).all()


@pytest.mark.parametrize("rows,n_in,n_out,way", TILES, ids=str)
def test_tiles_captured_and_replayed(rows, n_in, n_out, way):
    """Three replays with eager calls and changed inputs between them."""
    c = Product(rows, n_in, n_out)
    want = c.check()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=torch.cuda.Stream()):
        c.call(torch.cuda.current_stream().cuda_stream)
    for replay in range(3):
        c.out.fill_(7.0)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.out[:rows], want), replay
        c.x.neg_()
        want = -want
        c.check()


@pytest.mark.parametrize("rows,n_in,n_out,way", TILES + linear_plan.NARROW[:7], ids=str)
def test_the_same_bits_in_another_call(rows, n_in, n_out, way):
    """A few of the rows by themselves, which are divided in another way."""
    c = Product(rows, n_in, n_out, max_rows=rows)
    all_rows = c.check()
    for first, n in ((0, 1), (3, 17), (rows - 40, 40)):
        out = torch.full((n + 1, n_out), 7.0, dtype=torch.float16, device="cuda")
        c.linear.forward(n, c.x[first:].data_ptr(), c.xs[first:].data_ptr(), c.w.data_ptr(), c.ws.data_ptr(), out.data_ptr(), torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert torch.equal(out[:n], all_rows[first:first + n]) and (out[n:] == 7.0).all()
