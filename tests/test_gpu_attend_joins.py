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


@pytest.mark.parametrize("rows,shares", [(1, 20), (1, 21), (3, 20), (4, 16), (4, 17), (8, 8), (8, 9), (9, 2), (16, 3), (20, 2), (32, 3)])
def test_both_sides_of_what_the_last_workgroup_joins(rows, shares):
    run(100 + rows + shares, 1, [128 * shares - 5], 2 * rows, 2, 1, weigh=True)
    run(200 + rows + shares, 1, [128 * shares - 5], 2 * rows, 2, 1)


@pytest.mark.parametrize("rows,weigh", [(1, True), (4, True), (4, False), (20, True), (50, False)])
def test_more_shares_than_a_wave_has_lanes(rows, weigh):
    run(300 + rows, 1, [128 * 150 + 77], rows, 1, 1, weigh=weigh)
