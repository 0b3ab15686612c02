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


def test_gradients_on_two_streams():
    """The weights' and the norm's gradient need nothing of each other: neither writes where the other does."""
    rng = np.random.default_rng(2)
    T, B, H, A = 300, 30, 700, 29
    out = harness.OutputLayer(T, B, H, A, BF16)
    out.set_lengths(torch.from_numpy(rng.integers(100, T + 1, B).astype(np.int32)).cuda())
    out.set_weights(random(rng, A, H))
    out.forward(random(rng, T, B, H, dtype=torch.bfloat16))
    grads, dy = random(rng, T, B, A, dtype=torch.bfloat16), random(rng, T, B, H, dtype=torch.bfloat16)
    want = [t.clone() for t in (*out.weight_gradient(grads), *out.norm_backward(dy))]
    (a, b), (n, m) = out.ws_ptr, out.ws_bytes
    assert a + n <= b or b + m <= a
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        out.dweight.zero_(), out.dbias.zero_(), out.dnorm_weight.zero_()
        torch.cuda.synchronize()
        for _ in range(3):
            out.weight_gradient(grads, stream=streams[0].cuda_stream)
            out.norm_backward(dy, stream=streams[1].cuda_stream)
        torch.cuda.synchronize()
        assert all(torch.equal(g, w) for g, w in zip((out.dweight, out.dbias, out.dsum, out.dnorm_weight), want))
