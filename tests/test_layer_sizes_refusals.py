"""Sizes that a C int does not hold, and numbers that are no sizes, are refused by the size functions as by the calls, and not cut to fit."""
import numpy as np
import pytest

from paper_1512_02595_amd import layer

ASK = {
    "row_pitch": (layer.row_pitch, 1),
    "rms_norm_workspace_size": (layer.rms_norm_workspace_size, 2),
    "weight_gradient_workspace_size": (layer.weight_gradient_workspace_size, 3),
}


@pytest.mark.parametrize("what, at", [(n, i) for n, (_, k) in ASK.items() for i in range(k)])
def test_sizes_out_of_range(what, at):
    ask, count = ASK[what]
    for bad, error in ((2 ** 32 + 5, OverflowError), (-2 ** 31 - 1, OverflowError), (2 ** 31, OverflowError), (10.5, TypeError), ("5", TypeError), (None, TypeError)):
        sizes = [100] * count
        sizes[at] = bad
        with pytest.raises(error):
            ask(*sizes)


def test_sizes_of_numpys():
    assert layer.row_pitch(np.int64(129)) == 256
    assert layer.weight_gradient_workspace_size(np.int32(500), np.int64(100), 29) == layer.weight_gradient_workspace_size(500, 100, 29)
