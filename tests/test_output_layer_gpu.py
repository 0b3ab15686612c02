"""harness.OutputLayer where its calls meet: streams of the caller's, minibatches one after another, buffers of its own."""
import numpy as np
import pytest
import torch

import layer_reference as ref
from paper_1512_02595_amd import ctc, harness, layer

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


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("given_twice", [None, "dy", "dresidual"])
def test_gradients_behind_an_utterances_end_are_zeros_in_every_minibatch(given_twice, dtype):
    """Utterances get shorter: what the minibatch before left behind their new ends is gone.  So with an input in the result's place."""
    rng = np.random.default_rng(3)
    T, B, H, A, t = 9, 4, 130, 29, ref.torch_type(dtype)
    out = harness.OutputLayer(T, B, H, A, dtype)
    norm = random(rng, H)
    out.set_weights(random(rng, A, H), norm_weight=norm)
    for ends in ((9, 9, 7, 8), (3, 0, 7, 1), (9, 1, 0, 4)):
        x, dy, dresidual = (random(rng, T, B, H, dtype=t) for _ in range(3))
        out.set_lengths(lengths(*ends))
        out.forward(x)
        keep = torch.arange(T)[:, None] < torch.tensor(ends)[None, :]
        want, dweight, bound, terms = ref.norm_backward(dy.cpu()[keep].double(), x.cpu()[keep].double(), norm.cpu().double(),
                                                        float(np.float32(out.eps)), dresidual.cpu()[keep].double())
        if given_twice:
            out.dsum.copy_(dy if given_twice == "dy" else dresidual)
        dsum, dnorm = out.norm_backward(out.dsum if given_twice == "dy" else dy, out.dsum if given_twice == "dresidual" else dresidual)
        got = dsum.cpu()
        assert not got[~keep].any()
        assert ((got[keep].double() - want).abs() <= 1.001 * bound + ref.half_step(dtype) * (want.abs() + bound) + 1e-40).all()
        assert ((dnorm.cpu().double() - dweight).abs() <= ref.HALF * (int(keep.sum()) + 8) * terms + 1e-40).all()


def test_a_captured_norms_gradient_clears_what_the_replay_before_left():
    rng = np.random.default_rng(4)
    T, B, H, A = 12, 5, 300, 29
    out = harness.OutputLayer(T, B, H, A)
    out.set_weights(random(rng, A, H))
    x, dy, ends = torch.zeros((T, B, H), device="cuda"), torch.zeros((T, B, H), device="cuda"), lengths(*[T] * B)

    def step():
        out.set_lengths(ends)
        out.forward(x)
        out.norm_backward(dy)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for _ in range(4):
        x.copy_(random(rng, T, B, H)), dy.copy_(random(rng, T, B, H))
        ends.copy_(torch.from_numpy(rng.integers(0, T + 1, B).astype(np.int32)))
        step()
        torch.cuda.synchronize()
        want = out.dsum.clone(), out.dnorm_weight.clone()
        out.dsum.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.dsum, want[0]) and torch.equal(out.dnorm_weight, want[1]) and want[0].any()
        assert not out.dsum[torch.arange(T, device="cuda")[:, None] >= ends[None, :]].any()


def test_all_frames_count_until_lengths_are_set():
    rng = np.random.default_rng(5)
    T, B, H, A = 7, 3, 140, 29
    weight, x, grads, dy = random(rng, A, H), random(rng, T, B, H), random(rng, T, B, A), random(rng, T, B, H)
    results = []
    for said in (True, False):
        out = harness.OutputLayer(T, B, H, A)
        out.set_weights(weight)
        if said:
            out.set_lengths(lengths(*[T] * B))
        results.append([t.clone() for t in (out.forward(x), *out.weight_gradient(grads), *out.norm_backward(dy))])
    assert all(torch.equal(a, b) and a.any() for a, b in zip(*results))


def test_a_workspace_of_the_largest_minibatch_serves_a_smaller_one():
    """32768 rows take wide tiles and six times the workspace of 32800 rows, which take narrow ones."""
    rng = np.random.default_rng(6)
    most, rows, H, A = 32800, 32768, 2048, 172
    size = layer.weight_gradient_workspace_size(most, H, A)
    grads, scales = random(rng, rows, A), random(rng, rows)
    q = torch.from_numpy(rng.integers(-127, 128, (rows, H)).astype(np.int8)).cuda()
    results = []
    for n in (size, layer.weight_gradient_workspace_size(rows, H, A)):
        work, dweight, dbias = ref.Guarded((n,), torch.uint8), torch.zeros((A, H), device="cuda"), torch.zeros(A, device="cuda")
        assert work.t.data_ptr() % 256 == 0
        layer.weight_gradient_i8(grads.data_ptr(), q.data_ptr(), scales.data_ptr(), None, rows, H, A, F32, dweight.data_ptr(), dbias.data_ptr(),
                                 work.t.data_ptr(), n, ref.stream())
        torch.cuda.synchronize()
        assert work.intact()
        results.append((dweight, dbias))
    assert all(torch.equal(a, b) and a.any() for a, b in zip(*results))
