"""How products of ee_linear and ee_linear_grad are split (host arithmetic, no GPU): the sizes of the tests of every tile reach every tile."""
import ctypes

import pytest

import paper_2505_21594_amd as ee

FORWARD, DX, DW = 0, 1, 2
# rows, inputs and outputs of a layer, and the ways that this case is there for: (product, rows and columns of a tile, whether the sum is taken in parts).  Sizes that are no multiples
# of a tile, a step or eight; sums of at least two turns through a tile's buffers.
CASES = [
    ((415, 415, 133), [(FORWARD, 64, 64, False)]),
    ((415, 2500, 262), [(FORWARD, 64, 64, True)]),
    ((8003, 262, 450), [(FORWARD, 128, 128, False)]),
    ((1541, 6003, 1030), [(FORWARD, 128, 128, True)]),
    ((5001, 262, 1030), [(FORWARD, 192, 128, False)]),
    ((1290, 6003, 4099), [(FORWARD, 192, 128, True)]),
    ((415, 133, 415), [(DX, 64, 64, False)]),
    ((415, 262, 2500), [(DX, 64, 64, True)]),
    ((8003, 450, 262), [(DX, 128, 128, False)]),
    ((1541, 1030, 6003), [(DX, 128, 128, True)]),
    ((5001, 1030, 262), [(DX, 192, 128, False)]),
    ((1290, 4099, 6003), [(DX, 192, 128, True)]),
    ((415, 133, 133), [(DW, 64, 64, False)]),
    ((1541, 415, 450), [(DW, 64, 64, True)]),
    ((415, 2050, 2500), [(DW, 128, 128, False)]),
    ((4101, 450, 2500), [(DW, 128, 128, True)]),
    ((415, 2050, 6003), [(DW, 256, 128, False)]),
    ((6007, 2050, 2500), [(DW, 256, 128, True)]),
]


def step_of(rows):
    """Of the sum, for a tile of so many rows, and the buffers that its steps go through."""
    return {64: (64, 3), 128: (64, 2), 192: (64, 2), 256: (32, 3)}[rows]


@pytest.mark.parametrize("sizes,ways", CASES)
def test_cases_reach_the_ways_they_are_there_for(sizes, ways):
    rows, n_in, n_out = sizes
    for product, ti, tj, parts in ways:
        plan = ee.ee_debug_linear_plan(rows, n_in, n_out, product)
        assert (plan[:2], plan[2] > 1) == ((ti, tj), parts), f"product {product}: {plan}"
        step, buffers = step_of(ti)
        length = {FORWARD: n_in, DX: n_out, DW: rows}[product]
        assert min(plan[3], length) >= 2 * buffers * step, "too few steps for the buffers to come round"
        assert (length - (plan[2] - 1) * plan[3]) % step, "no part that ends inside a step"
        across = {FORWARD: (rows, n_out), DX: (rows, n_in), DW: (n_out, n_in)}[product]
        assert all(n % 8 and n % 64 for n in across), "no row or column that ends inside a piece"


def test_every_tile_of_every_product_is_reached():
    reached = {way for _, ways in CASES for way in ways}
    assert reached == {(p, t, 64 if t == 64 else 128, parts) for p, tiles in ((FORWARD, (64, 128, 192)), (DX, (64, 128, 192)), (DW, (64, 128, 256))) for t in tiles for parts in (False, True)}


def test_plans_are_whole():
    """Parts cover the sum, and none is empty."""
    for rows in (0, 1, 16, 17, 32, 33, 63, 300, 2041, 5000, 40000):
        for n_in in (1, 7, 64, 384, 1000, 4096, 32000):
            for n_out in (1, 33, 256, 688, 4096, 11008):
                for product, length in ((FORWARD, n_in), (DX, n_out), (DW, rows)):
                    ti, tj, parts, per = ee.ee_debug_linear_plan(rows, n_in, n_out, product)
                    assert per % 64 == 0 and parts * per >= length and (parts == 1 or (parts - 1) * per < length)
                    assert product == FORWARD or ti >= 64


def test_plan_is_checked():
    lib, plan = ee.load_library(), (ctypes.c_int32 * 4)()
    for bad in ((-1, 64, 64, 0), (5, 0, 64, 0), (5, 64, (1 << 22) + 1, 1), (5, 64, 64, 3), (5, 64, 64, -1)):
        assert lib.ee_debug_linear_plan(*bad, plan) == ee.EE_EINVAL
    assert lib.ee_debug_linear_plan(5, 64, 64, 0, None) == ee.EE_EINVAL
