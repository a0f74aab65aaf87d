"""Joins inside the sweep's launch at every remainder of rows times shares by four: the sums of its parts lie in LDS behind a factor
a (row, share), at multiples of sixteen bytes."""
import pytest

from test_gpu_attend import run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [1, 2, 3, 5])
@pytest.mark.parametrize("shares", [2, 3, 5, 7])
def test_rows_and_shares_of_any_number(rows, shares):
    run(rows + 8 * shares, 1, [128 * shares - 3], rows, 1, 1, weigh=True)
    run(rows + 8 * shares, 1, [128 * shares], 2 * rows, 2, 1)
