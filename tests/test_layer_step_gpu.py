"""The output layer and CTC together, as a training step and an alignment use them: states to activations to costs and gradients to the
weights' gradient, against the same chain in 64 bits on the CPU, for a minibatch of unlike lengths."""
import numpy as np
import pytest
import torch

import layer_reference as ref
from oracle import ctc_oracle as orc
from paper_1512_02595_amd import ctc, harness
from paper_1512_02595_amd import workloads as wl

pytestmark = pytest.mark.gpu


def chain(T, B, H, A, max_label, dtype, seed):
    rng = np.random.default_rng(seed)
    t = ref.torch_type(dtype)
    batch = wl.make_random(seed, T=T, B=B, A=A, max_label=max_label, min_input=min(T, max(2, T // 3)))
    db = harness.DeviceBatch(batch, dtype)
    out = harness.OutputLayer(T, B, H, A, dtype, logits=db.x)
    x = torch.from_numpy(rng.standard_normal((T, B, H))).to(t).cuda()
    residual = torch.from_numpy(rng.standard_normal((T, B, H))).to(t).cuda()
    weight = torch.from_numpy(rng.standard_normal((A, H)) * 3 / np.sqrt(H)).float().cuda()
    bias, norm_weight = torch.from_numpy(rng.standard_normal(A)).float(), torch.from_numpy(1 + 0.3 * rng.standard_normal(H)).float()
    out.set_weights(weight, bias.cuda(), norm_weight.cuda())
    out.set_lengths(torch.from_numpy(batch.input_lengths.astype(np.int32)).cuda())
    return batch, db, out, x, residual, weight, bias, norm_weight


@pytest.mark.parametrize("dtype", [ctc.DTYPE_F32, ctc.DTYPE_BF16])
@pytest.mark.parametrize("T, B, H, A, max_label", [(60, 9, 200, 29, 15), (40, 17, 333, 500, 9), (1, 3, 64, 29, 1)])
def test_a_training_step(T, B, H, A, max_label, dtype):
    print("step", T, B, H, A, dtype, flush=True)
    batch, db, out, x, residual, weight, bias, norm_weight = chain(T, B, H, A, max_label, dtype, 41 + T)
    t = ref.torch_type(dtype)
    db.x.fill_(7.0)                                      # (padding holds whatever it held)
    out.forward(x, residual)
    db.run()
    dweight, dbias = out.weight_gradient(db.grads)
    dy = torch.matmul(db.grads.float(), weight).to(t).contiguous()
    dsum, dnorm = out.norm_backward(dy)
    costs, grads = db.results()

    valid = torch.from_numpy(np.arange(T)[:, None] < batch.input_lengths[None, :])
    z = (x.cpu().float() + residual.cpu().float()).to(t)[valid]
    u = z.float() * norm_weight
    q, s = ref.to_levels(u)
    eps = float(np.float32(out.eps))
    y = q * (s * ref.rms(z.double(), eps))[:, None]
    wq, ws = ref.to_levels(weight.cpu())
    logits = y @ (wq * ws[:, None]).t() + bias.double()
    got = db.x.cpu()[valid].double()
    # the row's scale and a weight's, their product, its product with the sum, the sum with the bias: half a step each
    assert ((got - logits).abs() <= 6 * ref.HALF * ((logits - bias.double()).abs() + logits.abs()) + ref.half_step(dtype) * 1.01 * logits.abs()).all()
    assert (db.x.cpu()[~valid] == 7.0).all()

    # CTC on the activations that it was given
    rows = np.zeros((T, B, A), dtype=np.float32)
    rows[valid.numpy()] = db.x.float().cpu().numpy()[valid.numpy()]
    want_c, want_g = orc.ctc_loss_and_grad(rows, batch.flat_labels, batch.label_lengths, batch.input_lengths, batch.blank)
    inf = np.isinf(want_c)
    assert np.array_equal(np.isinf(costs), inf)
    assert (np.abs(costs[~inf] - want_c[~inf]) <= 1e-4 * np.maximum(np.abs(want_c[~inf]), 1e-2)).all()
    assert np.abs(grads - want_g).max() <= (1e-4 if dtype == ctc.DTYPE_F32 else 1e-2)

    # the weights' gradient, of the gradient that CTC gave and the rows as they are held
    g = db.grads.cpu()[valid].double()
    held = out.q.cpu()[:, :H].double().view(T, B, H)[valid] * out.scales.cpu().double().view(T, B)[valid][:, None]
    want, terms = g.t().contiguous() @ held, g.abs().t().contiguous() @ held.abs()
    assert ((dweight.cpu().double() - want).abs() <= ref.HALF * (3 * len(g) + 8) * terms + 1e-38).all()
    assert ((dbias.cpu().double() - g.sum(0)).abs() <= ref.HALF * (len(g) + 8) * g.abs().sum(0) + 1e-38).all()
    # and of the padded sum: CTC writes zeros for padding, so the whole tensor gives the same
    whole = db.grads.cpu().double().view(-1, A).t().contiguous() @ (out.q.cpu()[:, :H].double() * out.scales.cpu().double()[:, None])
    assert ((whole - want).abs() <= 1e-12 * (terms + 1e-30)).all()

    dz, dw, bound, sizes = ref.norm_backward(dy.cpu()[valid].double(), z.double(), norm_weight.double(), eps, None)
    got = dsum.cpu()[valid].double()
    assert ((got - dz).abs() <= 1.001 * bound + ref.half_step(dtype) * (dz.abs() + bound) + 1e-40).all()
    assert ((dnorm.cpu().double() - dw).abs() <= ref.HALF * (len(z) + 8) * sizes + 1e-40).all()
    assert not dsum.cpu()[~valid].any()


def test_alignments_of_activations_from_8_bits():
    batch, db, out, x, residual, *_ = chain(80, 12, 256, 29, 20, ctc.DTYPE_F32, 77)
    out.forward(x, residual)
    db.run_best_path()
    scores, states = db.best_path_results()
    rows = np.zeros((80, 12, 29), dtype=np.float32)
    valid = np.arange(80)[:, None] < batch.input_lengths[None, :]
    rows[valid] = db.x.cpu().numpy()[valid]
    want_s, want_a = orc.ctc_best_path(rows, batch.flat_labels, batch.label_lengths, batch.input_lengths, batch.blank)
    inf = np.isinf(want_s)
    assert np.array_equal(np.isinf(scores), inf)
    assert (np.abs(scores[~inf] - want_s[~inf]) <= 1e-4 * np.maximum(np.abs(want_s[~inf]), 1e-2)).all()
    assert np.array_equal(states, want_a)


def test_a_step_whose_lengths_stay_on_the_gpu_is_captured_whole():
    """Lengths, labels and states change between replays; every replay gives what the calls give."""
    T, B, H, A, max_label = 50, 8, 192, 29, 12
    dm = harness.DeviceMetaBatch(T, B, A, max_label)
    out = harness.OutputLayer(T, B, H, A, logits=dm.x)
    rng = np.random.default_rng(5)
    x, residual = torch.zeros((T, B, H), device="cuda"), torch.zeros((T, B, H), device="cuda")
    weight = torch.zeros((A, H), device="cuda")

    def fill(seed):
        batch = wl.make_random(seed, T=T, B=B, A=A, max_label=max_label, min_input=20)
        dm.load(batch)
        for buf in (x, residual, weight):
            buf.copy_(torch.from_numpy(rng.standard_normal(tuple(buf.shape)) * 0.5))

    def step():
        out.set_lengths(dm.input_lengths)
        out.set_weights(weight)
        out.forward(x, residual)
        dm.run()
        out.weight_gradient(dm.grads)

    def results():
        torch.cuda.synchronize()
        return [t.clone() for t in (dm.costs, dm.grads, out.dweight, out.dbias, dm.status)]

    fill(1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for seed in (2, 3, 4):
        fill(seed)
        step()
        want = results()
        dm.grads.fill_(1.0)
        out.dweight.fill_(1.0)
        graph.replay()
        got = results()
        assert int(got[4]) == ctc.STATUS_SUCCESS
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and got[2].any()
