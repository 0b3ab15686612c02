"""An error that the caller met before is none of the output layer's calls'."""
import pytest
import torch

import test_layer_gpu as base
from paper_1512_02595_amd import layer

pytestmark = pytest.mark.gpu


def test_an_error_from_before_is_not_reported():
    """hipSetDevice of a device that is not there: refused on the host, and remembered as the thread's last error."""
    lib = layer.load()
    step = base.Step(51, 6, 4, 200, 300, base.F32)
    step.run(base.stream())
    want, before = step.results(), layer.last_hip_error()
    step.clear()
    assert lib.hipSetDevice(1000) != 0
    try:
        step.run(base.stream())                          # (each call raises what it reports)
    finally:
        lib.hipGetLastError()                            # (torch would take it for its own)
    assert all(torch.equal(a, b) for a, b in zip(step.results(), want))
    assert layer.last_hip_error() == before
