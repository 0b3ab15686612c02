"""Every kernel that a size can take is one that a GPU test's size takes, with a list of rows and without, where the rule knows of the list."""
import pytest

import layer_rules as rules
import test_layer_gpu as base
import test_layer_kernels_gpu as many


def test_rows_to_8_bits():
    met = {rules.row_shape(rows, H) for rows, H in [*((37, H) for H in base.WIDTHS), *(m[:2] for m in many.MANY_ROWS)]}
    can = {rules.row_shape(rows, H) for rows in (1, 2048, 2049, 1 << 30) for H in [1, *range(64, 16385, 64)]}
    assert met == can and len(can) == 9


@pytest.mark.parametrize("listed", [False, True])
def test_activations(listed):
    sizes = [*base.SHAPES, *(m[:3] for m in many.MANY_TILES)]
    met = {rules.product_tile(*size, listed) for size in sizes}
    assert met == {(16, 16), (64, 64), (128, 64), (128, 128), (256, 256)}


def test_the_weights_gradient():
    met = {rules.gradient_tile(*m[:3])[0] for m in many.MANY_SLABS}
    assert met == {32, 64, 128}


@pytest.mark.parametrize("rows, H, A, listed, tile", [
    # what a rule was measured at, and the sizes at its borders
    (1, 2048, 6000, False, (16, 16)), (16, 2048, 6000, False, (16, 16)), (16, 2048, 6400, False, (16, 16)), (1, 2048, 6401, False, (64, 64)),
    (32, 2048, 6000, False, (64, 64)), (300, 2048, 6000, False, (64, 64)), (27200, 2048, 60, False, (128, 64)), (48000, 2048, 29, True, (128, 64)),
    (5000, 2048, 60, False, (64, 64)), (25600, 2048, 64, False, (64, 64)), (25601, 2048, 64, False, (128, 64)), (25601, 2048, 65, False, (128, 128)),
    (3000, 512, 6000, False, (128, 128)), (19200, 2048, 6000, False, (256, 256)), (32000, 2048, 6000, True, (256, 256)), (8991, 1111, 4733, True, (256, 256))])
def test_tiles_of_activations(rows, H, A, listed, tile):
    assert rules.product_tile(rows, H, A, listed) == tile
