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
