"""What harness.OutputLayer refuses before anything is enqueued.  No GPU is touched: the layer's buffers are the host's, the tensors it is given
have another device and no memory (their address is null)."""
import pytest
import torch

from paper_1512_02595_amd import ctc, harness

T, B, H, A = 5, 3, 100, 29


def given(*shape, dtype=torch.float32):
    return torch.empty(shape, dtype=dtype, device="meta")


CALLS = {
    "set_weights": lambda out: out.set_weights(given(A, H), stream=0),
    "set_lengths": lambda out: out.set_lengths(given(B, dtype=torch.int32), stream=0),
    "forward": lambda out: out.forward(given(T, B, H), stream=0),
    "residual": lambda out: out.forward(torch.zeros(T, B, H), given(T, B, H), stream=0),
    "weight_gradient": lambda out: out.weight_gradient(given(T, B, A), stream=0),
    "norm_backward": lambda out: out.norm_backward(given(T, B, H), stream=0),
    "dresidual": lambda out: out.norm_backward(torch.zeros(T, B, H), given(T, B, H), stream=0),
}


@pytest.mark.parametrize("call", CALLS)
def test_tensors_of_another_device(call):
    out = harness.OutputLayer(T, B, H, A, device=torch.device("cpu"))
    with pytest.raises(AssertionError):
        CALLS[call](out)


def test_activations_of_another_device():
    with pytest.raises(AssertionError):
        harness.OutputLayer(T, B, H, A, logits=given(T, B, A), device=torch.device("cpu"))


def test_a_width_without_a_pitch():
    with pytest.raises(ctc.CTCError):
        harness.OutputLayer(T, B, 16385, A, device=torch.device("cpu"))
