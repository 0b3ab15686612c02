"""The output layer's calls at the ends of what they take: the largest alphabet, the widest state, tensors of more than 2^31 elements without a list,
and calls from several threads at once."""
import threading

import numpy as np
import pytest
import torch

import layer_reference as ref
import layer_rules as rules
import test_layer_gpu as base
from layer_reference import frame_list
from paper_1512_02595_amd import ctc, layer

pytestmark = pytest.mark.gpu
F32, BF16 = ctc.DTYPE_F32, ctc.DTYPE_BF16


@pytest.mark.parametrize("kind", ["all", "some"])
@pytest.mark.parametrize("rows, H, dtype", [(3, 64, F32), (40, 100, BF16)])
def test_the_largest_alphabet(rows, H, dtype, kind):
    print("largest alphabet", rows, H, dtype, kind, flush=True)
    rng = np.random.default_rng(rows)
    A = 1 << 20
    q, s = base.levels(rng, rows, H)
    wq, ws = base.levels(rng, A, H)
    bias = torch.from_numpy(rng.standard_normal(A)).float()
    frames, names = frame_list(kind, rows, rng)
    base.check_linear(base.linear(q, s, wq, ws, bias, dtype, frames), q, s, wq, ws, bias, dtype, names)
    grads = torch.from_numpy(rng.standard_normal((rows, A))).float().to(ref.torch_type(dtype)).float()
    base.check_gradient(*base.weight_gradient(grads, q, s, dtype, frames, names=names), grads, q, s, names)


@pytest.mark.parametrize("kind", ["all", "odd entries"])
@pytest.mark.parametrize("rows, A, symbols", [(2000, 129, 64), (6000, 300, 128)])
def test_the_widest_state(rows, A, symbols, kind):
    print("widest state", rows, A, kind, flush=True)
    H = 16384
    assert rules.gradient_tile(rows, H, A)[0] == symbols
    rng = np.random.default_rng(rows)
    q, s = base.levels(rng, rows, H)
    frames, names = frame_list(kind, rows, rng)
    grads = base.gradients(rng, rows, A, BF16)
    base.check_gradient(*base.weight_gradient(grads, q, s, BF16, frames, names=names), grads, q, s, names)
    wq, ws = base.levels(rng, A, H)
    base.check_linear(base.linear(q, s, wq, ws, None, BF16, frames), q, s, wq, ws, None, BF16, names)


def test_more_than_2_to_the_31_activations():
    """All rows of a tensor of 2.2e9 activations, written and read: the last ones, and some in between."""
    rows, H, A = 70001, 130, 31999
    pitch = layer.row_pitch(H)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    q, wq = (torch.randint(-127, 128, (n, pitch), dtype=torch.int8, device="cuda", generator=gen) for n in (rows, A))
    q[:, H:], wq[:, H:] = 0, 0
    s, ws = (torch.rand(n, device="cuda", generator=gen) * 0.01 for n in (rows, A))
    out = torch.empty((rows, A), dtype=torch.bfloat16, device="cuda")
    layer.linear_i8(q.data_ptr(), s.data_ptr(), wq.data_ptr(), ws.data_ptr(), None, None, rows, H, A, BF16, out.data_ptr(), ref.stream())
    look = torch.cat((torch.arange(0, rows, 997), torch.arange(rows - 40, rows)))
    total = q[look].cpu()[:, :H].double() @ wq.cpu()[:, :H].double().t()
    want = total * s[look].cpu().double()[:, None] * ws.cpu().double()[None, :]
    assert ((out[look].cpu().double() - want).abs() <= 2.0 ** -8 * 1.001 * want.abs() + 1e-30).all()
    # and its gradients: ones in a few rows, the last among them
    out.zero_()
    some = torch.tensor([0, rows // 2, rows - 2, rows - 1])
    out[some] = 1.0
    size = layer.weight_gradient_workspace_size(rows, H, A)
    work, dweight, dbias = torch.empty(size, dtype=torch.uint8, device="cuda"), torch.empty((A, H), device="cuda"), torch.empty(A, device="cuda")
    layer.weight_gradient_i8(out.data_ptr(), q.data_ptr(), s.data_ptr(), None, rows, H, A, BF16, dweight.data_ptr(), dbias.data_ptr(), work.data_ptr(),
                             size, ref.stream())
    torch.cuda.synchronize()
    y = q[some].cpu()[:, :H].double() * s[some].cpu().double()[:, None]
    assert ((dweight.cpu().double() - y.sum(0)).abs() <= ref.HALF * 24 * y.abs().sum(0)).all() and (dbias == 4.0).all()


def test_calls_from_several_threads():
    """Each thread with buffers and a stream of its own; the results are those of one after another."""
    steps = [base.Step(60 + i, 20 + i, 9, 200 + 77 * i, (29, 300, 64, 1000)[i], (F32, BF16)[i % 2]) for i in range(4)]
    want = []
    for step in steps:
        step.run(ref.stream())
        want.append(step.results())
        step.clear()
    torch.cuda.synchronize()
    streams, failed = [torch.cuda.Stream() for _ in steps], []

    def work(step, on):
        try:
            for _ in range(20):
                step.run(on.cuda_stream)
        except BaseException as e:
            failed.append(e)

    threads = [threading.Thread(target=work, args=pair) for pair in zip(steps, streams)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed
    for step, w in zip(steps, want):
        assert all(torch.equal(a, b) for a, b in zip(step.results(), w))
