"""Every kernel of the 8-bit products in every way that it ends a tile and a contraction (i8_shapes.py), on guarded memory, against 64 bits."""
import pytest

import i8_checks as c
import i8_shapes as shapes
from test_gpu_i8_bounds import check_gated, check_linear, check_linear_backward

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    c.binding.load_library()
    return torch


def cases(groups, gated):
    return [pytest.param(d, s, id="%dx%d_tile%d_T%d_%dx%d" % (d, 8, t, *s)) for (g, d, t), some in groups.items() if g == gated for s in some]


# Elements by which inputs and outputs start behind 64 aligned bytes: results in the middle of a word are stored in another way, addends there do not come
# through the ring.
PLAIN, GATED = (0, 1, 4), (0, 4, (0, 1), (1, 0))


@pytest.mark.parametrize("digits,shape", cases(shapes.TILES, False) + cases(shapes.SHARED, False))
def test_plain_tiles(torch, digits, shape):
    T, cols, n = shape
    check_linear(torch, T, cols, n, digits, PLAIN)
    check_linear_backward(torch, T, n, cols, digits, PLAIN[:2])


@pytest.mark.parametrize("digits,shape", cases(shapes.TILES, True) + cases(shapes.SHARED, True))
def test_gated_tiles(torch, digits, shape):
    check_gated(torch, *shape, digits, GATED, ((True, True), (False, False)))


@pytest.mark.parametrize("digits,tile", list(shapes.AHEAD))
def test_addends_through_the_ring(torch, digits, tile):
    for shape in shapes.AHEAD[digits, tile]:
        check_gated(torch, *shape, digits, GATED, ((True, True), (True, False)))


@pytest.mark.parametrize("digits", [1, 2])
def test_streamed_results(torch, digits):
    check_gated(torch, *shapes.STREAMED[digits], digits, (0,), ((True, True), (True, False), (False, True), (False, False)))


@pytest.mark.parametrize("gated,way", list(shapes.OWN_ROWS))
def test_rows_made_by_the_product(torch, gated, way):
    for shape in shapes.OWN_ROWS[gated, way]:
        if gated:
            check_gated(torch, *shape, 1, (0, 1, 8))
        else:
            check_linear(torch, *shape, 1, (0, 1, 8))
