"""harness.OutputLayer where its calls meet: streams of the caller's, minibatches one after another, buffers of its own."""
import numpy as np
import pytest
import torch

import layer_reference as ref
from paper_1512_02595_amd import ctc, harness

pytestmark = pytest.mark.gpu
F32, BF16 = ctc.DTYPE_F32, ctc.DTYPE_BF16


def random(rng, *shape, dtype=torch.float32):
    return torch.from_numpy(rng.standard_normal(shape)).to(dtype).cuda()


def lengths(*values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def busy(product):
    """Some tens of milliseconds of work on the current stream."""
    for _ in range(30):
        product = torch.mm(product, product).clamp_(-1.0, 1.0)


@pytest.mark.parametrize("handle", ["a stream of torch's", "the default stream"])
def test_weights_are_set_on_the_stream_that_is_given(handle):
    """The current stream is behind: what the call copies does not wait for it, and the next call on the same stream has it."""
    rng = np.random.default_rng(1)
    T, B, H, A = 6, 3, 200, 29
    x, weight, bias, norm = random(rng, T, B, H), random(rng, A, H), random(rng, A), random(rng, H)
    layers = [harness.OutputLayer(T, B, H, A) for _ in range(2)]
    for out in layers:
        out.set_lengths(lengths(6, 4, 1))
    layers[0].set_weights(weight, bias, norm)
    want = layers[0].forward(x).clone()
    large = random(rng, 8192, 8192)
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    current, given = (torch.cuda.current_stream(), other) if handle == "a stream of torch's" else (other, torch.cuda.default_stream())
    with torch.cuda.stream(current):
        busy(large)
        layers[1].set_weights(weight, bias, norm, stream=given.cuda_stream)
        layers[1].forward(x, stream=given.cuda_stream)
    given.synchronize()
    with torch.cuda.stream(given):
        got = layers[1].logits.clone()
    torch.cuda.synchronize()
    assert torch.equal(got, want) and want.any()
    assert torch.equal(layers[1].bias, bias) and torch.equal(layers[1].norm_weight, norm)
