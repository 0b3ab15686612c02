"""What harness.RecurrentBlock and harness.StreamingBlock refuse before anything is enqueued.  No GPU is touched: the blocks' buffers are the host's, the
tensors they are given have another device and no memory, or another shape or type."""
import pytest
import torch

from paper_1512_02595_amd import ctc, harness

T, B, H = 5, 3, 100
CPU = torch.device("cpu")


def given(*shape, dtype=torch.float32, device="meta"):
    return torch.empty(shape, dtype=dtype, device=device)


def here(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype)


TRAINING = {
    "set_lengths": lambda b, t: b.set_lengths(t(B, dtype=torch.int32), stream=0),
    "projections": lambda b, t: b.forward(t(T, B, 3 * H), stream=0),
    "residual": lambda b, t: b.forward(here(T, B, 3 * H), t(T, B, H), stream=0),
    "initial": lambda b, t: b.forward(here(T, B, 3 * H), None, t(B, H), stream=0),
    "dnormed": lambda b, t: b.backward(here(T, B, 3 * H), t(T, B, H), stream=0),
    "dsum": lambda b, t: b.backward(here(T, B, 3 * H), here(T, B, H), t(T, B, H), stream=0),
    "dfinal": lambda b, t: b.backward(here(T, B, 3 * H), here(T, B, H), None, None, t(B, H), stream=0),
}
STREAMING = {
    "set_lengths": lambda b, t: b.set_lengths(t(B, dtype=torch.int32), stream=0),
    "residual": lambda b, t: b.forward(t(T, B, H), stream=0),
    "weight": lambda b, t: b.set_weights(t(3 * H, H), stream=0),
}


@pytest.mark.parametrize("call", TRAINING)
def test_training(call):
    for kind in ("another device", "another type", "another shape", "a strided one"):
        made = harness.RecurrentBlock(T, B, H, device=CPU)
        with pytest.raises(AssertionError):
            TRAINING[call](made, wrong(kind))


@pytest.mark.parametrize("call", STREAMING)
def test_streaming(call):
    for kind in ("another device", "another type", "another shape", "a strided one"):
        made = harness.StreamingBlock(B, H, T, device=CPU)
        with pytest.raises(AssertionError):
            STREAMING[call](made, wrong(kind))


def wrong(kind):
    def make(*shape, dtype=torch.float32):
        if kind == "another device":
            return given(*shape, dtype=dtype)
        if kind == "another type":
            return here(*shape, dtype=torch.float64)
        if kind == "another shape":
            return here(*shape[:-1], shape[-1] + 1, dtype=dtype)
        return here(*shape, 2, dtype=dtype)[..., 0]
    return make


def test_gradients_in_the_blocks_own_places():
    made = harness.RecurrentBlock(T, B, H, device=CPU)
    for own in (made.dresidual, made.dstates):
        with pytest.raises(AssertionError):
            made.backward(here(T, B, 3 * H), own, stream=0)


def test_sizes():
    with pytest.raises(ctc.CTCError):
        harness.RecurrentBlock(T, B, 16385, device=CPU)
    with pytest.raises(ctc.CTCError):
        harness.StreamingBlock(B, H, T, group=100, device=CPU)
