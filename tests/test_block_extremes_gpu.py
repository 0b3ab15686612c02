"""The norms around a block and the products with weights in 4 bits where numbers are huge, tiny or not finite, rows many, and calls captured or at once."""
import threading

import numpy as np
import pytest
import torch

import block_reference as ref
from layer_reference import Guarded, HALF, half_step, library_rows, put, stream, torch_type
from paper_1512_02595_amd import block, ctc, layer
from test_block_norm_gpu import EPS, Call, at, backward, forward

pytestmark = pytest.mark.gpu
F32, BF16 = ctc.DTYPE_F32, ctc.DTYPE_BF16
TYPES = [F32, BF16]


def say(*a):
    print(*a, flush=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scale", [1e-36, 1e-30, 1e-20, 1e-12, 1e12, 1e20, 1e30])
@pytest.mark.parametrize("H", [70, 500, 1300, 8200])
def test_rows_of_every_size(H, scale, dtype):
    """Squares that fp32 does not hold: the row's sums are formed in fp64."""
    say("sizes", H, scale, dtype)
    c = Call(9, H, dtype, "all", H, 3)
    for name in ("x", "z", "residual"):
        setattr(c, name, (getattr(c, name).double() * scale).float().to(c.tt).float())
    c.x[2], c.z[2], c.residual[2] = 0.0, 0.0, 0.0
    c.x[3], c.dy[4], c.dz[4] = 0.0, 0.0, 0.0
    if scale > 1:
        c.w[0] = c.w[0] * 1e-3                          # (what is added to a residual of this size may be of its size)
        c.ones[0], c.w_dev[0] = c.w[0], put(c.w[0], torch.float32)
    forward(c)
    backward(c)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H", [70, 500, 1300, 8200])
def test_rows_that_are_not_finite(H, dtype):
    """An infinity or a NaN in a row is that row's own affair, and its columns' in the weights' gradients."""
    say("not finite", H, dtype)
    rows = 12
    c = Call(rows, H, dtype, "all", H, 4)
    clean, dirty = run(c), None
    c.x[1, 3], c.gate[2, 5], c.residual[3, 7], c.dy[4, 9], c.z[5, 2] = float("inf"), float("nan"), float("-inf"), float("nan"), float("inf")
    dirty = run(c)
    fine = [r for r in range(rows) if r not in (1, 2, 3, 4, 5)]
    for name in ("sum", "normed", "dx", "dgate", "dresidual"):
        assert torch.equal(clean[name][fine], dirty[name][fine]), name
    assert bool(torch.isnan(dirty["normed"][1]).any()) and bool(torch.isnan(dirty["sum"][2, 5])) and bool(torch.isnan(dirty["normed"][3]).any())
    assert torch.equal(clean["sum"][2, :5], dirty["sum"][2, :5])
    assert bool(torch.isnan(dirty["dx"][4]).any()) and bool(torch.isnan(dirty["dweight_before"]).any())


def buffers(c):
    size = block.block_norm_workspace_size(c.rows, c.H)
    ws = torch.empty(size + 256, dtype=torch.uint8, device="cuda")
    b = {"x": c.dev(c.x), "gate": c.gate_dev(), "residual": c.dev(c.residual), "z": c.dev(c.z), "dy": c.dev(c.dy), "dz": c.dev(c.dz)}
    out = {k: torch.zeros(c.rows, c.pitch if k == "dgate" else c.H, dtype=c.tt, device="cuda") for k in ("sum", "normed", "dx", "dgate", "dresidual")}
    out.update({k: torch.zeros(c.H, device="cuda") for k in ("dweight_after", "dscale", "dweight_before")})
    return b, out, (ws, (ws.data_ptr() + 255) // 256 * 256, size)


def enqueue(c, b, out, ws, s):
    frames = None if c.frames is None else c.frames.data_ptr()
    block.block_norm(at(b["x"]), at(b["gate"]), c.pitch, at(b["residual"]), *map(at, c.w_dev), EPS, frames, c.rows, c.H, c.dtype,
                     out["sum"].data_ptr(), out["normed"].data_ptr(), s)
    block.block_norm_backward(at(b["dy"]), at(b["dz"]), at(b["x"]), at(b["gate"]), c.pitch, at(b["z"]), *map(at, c.w_dev), EPS, frames, c.rows,
                              c.H, c.dtype, *(out[k].data_ptr() for k in ("dx", "dgate", "dresidual", "dweight_after", "dscale", "dweight_before")),
                              ws[1], ws[2], s)


def run(c):
    b, out, ws = buffers(c)
    enqueue(c, b, out, ws, stream())
    torch.cuda.synchronize()
    return out


@pytest.mark.parametrize("rows, H", [(1, 300), (40, 64), (300, 1100), (50, 9000)])
def test_replays_of_captured_norms(rows, H):
    """A replay reads the list and the inputs afresh; two graphs share a workspace on one stream."""
    say("graphs", rows, H)
    calls = [Call(rows, H, F32, "some", H, s) for s in (5, 6)]
    made = [buffers(c) for c in calls]
    ws = made[0][2]
    for c, (b, out, _) in zip(calls, made):
        enqueue(c, b, out, ws, stream())
    torch.cuda.synchronize()
    want = [{k: v.clone() for k, v in out.items()} for _, out, _ in made]
    side, graphs = torch.cuda.Stream(), []
    for c, (b, out, _) in zip(calls, made):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            enqueue(c, b, out, ws, torch.cuda.current_stream().cuda_stream)
        graphs.append(g)
    for _ in range(4):
        for g, (_, out, _), w in zip(graphs, made, want):
            for v in out.values():
                v.zero_()
            run(Call(20, H, BF16, "all", H, 8))          # (the program's own work in between)
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(out[k], w[k]) for k in w)
    calls[0].frames[0] = 0                               # no row counts: weights' gradients are zeros, rows stay
    before = {k: v.clone() for k, v in made[0][1].items()}
    graphs[0].replay()
    torch.cuda.synchronize()
    for k, v in made[0][1].items():
        assert not v.any() if k in ("dweight_after", "dscale", "dweight_before") else torch.equal(v, before[k])


def test_norms_at_once():
    say("two streams")
    calls = [Call(400, 700, F32, "some", 700, s) for s in (7, 8)]
    want = [run(c) for c in calls]
    results = [None, None]

    def work(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            b, out, ws = buffers(calls[i])
            for _ in range(30):
                enqueue(calls[i], b, out, ws, torch.cuda.current_stream().cuda_stream)
            torch.cuda.current_stream().synchronize()
            results[i] = out

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for got, w in zip(results, want):
        assert all(torch.equal(got[k], w[k]) for k in w)


def test_rows_listed_twice():
    """Row-wise outputs are those of one listing, sums count it twice."""
    say("twice")
    c = Call(30, 200, F32, "all", 200, 9)
    once = run(c)
    entries = list(range(30)) + [4, 4]
    c.frames = torch.tensor([30] + entries[:30], dtype=torch.int32, device="cuda")
    c.frames[1:31] = torch.tensor([4 if i in (10, 11) else i for i in range(30)], dtype=torch.int32)
    got = run(c)
    rest = [i for i in range(30) if i not in (10, 11)]
    for k in ("sum", "normed", "dx", "dgate", "dresidual"):
        assert torch.equal(got[k][rest], once[k][rest]) and not got[k][[10, 11]].any()
    part = c.dy.double() * c.z.double() / torch.sqrt((c.z.double() ** 2).mean(1, keepdim=True) + float(np.float32(EPS)))
    want = part[rest].sum(0) + 2 * part[4]
    assert torch.allclose(got["dweight_before"].cpu().double(), want, rtol=1e-5, atol=1e-5 * float(part.abs().sum(0).max()))


def test_norms_of_more_than_2_31_elements():
    rows, H = 2_200_000, 1000
    say("beyond 2^31", rows * H)
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, z = (torch.empty(rows, H, dtype=torch.bfloat16, device="cuda").normal_(generator=gen) for _ in range(2))
    total, normed = torch.empty_like(x), torch.empty_like(x)
    block.block_norm(x.data_ptr(), x.data_ptr(), H, z.data_ptr(), None, None, None, EPS, None, rows, H, BF16, total.data_ptr(), normed.data_ptr(), stream())
    size = block.block_norm_workspace_size(rows, H)
    ws = torch.empty(size + 256, dtype=torch.uint8, device="cuda")
    dx, dgate, dres, dw = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x), torch.empty(3, H, device="cuda")
    block.block_norm_backward(z.data_ptr(), None, x.data_ptr(), x.data_ptr(), H, total.data_ptr(), None, None, None, EPS, None, rows, H, BF16, dx.data_ptr(),
                              dgate.data_ptr(), dres.data_ptr(), dw[0].data_ptr(), dw[1].data_ptr(), dw[2].data_ptr(),
                              (ws.data_ptr() + 255) // 256 * 256, size, stream())
    torch.cuda.synchronize()
    for part in (slice(0, 5), slice(rows - 5, rows)):
        xs, zs = x[part].contiguous(), z[part].contiguous()
        out = [torch.empty_like(xs) for _ in range(5)]
        block.block_norm(xs.data_ptr(), xs.data_ptr(), H, zs.data_ptr(), None, None, None, EPS, None, 5, H, BF16, out[0].data_ptr(), out[1].data_ptr(), stream())
        block.block_norm_backward(zs.data_ptr(), None, xs.data_ptr(), xs.data_ptr(), H, out[0].data_ptr(), None, None, None, EPS, None, 5, H, BF16,
                                  out[2].data_ptr(), out[3].data_ptr(), out[4].data_ptr(), None, None, None, None, 0, stream())
        torch.cuda.synchronize()
        for whole, few in zip((total, normed, dx, dgate, dres), out):
            assert torch.equal(whole[part], few)


# ---- weights in 4 bits ------------------------------------------------------------------------------------------

def product_of(rows, A, H, group, dtype, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    w = torch.randn(A, H, device="cuda", generator=gen)
    nw, ns = block.weights_i4_sizes(A, H, group)
    wq, ws = torch.empty(nw, dtype=torch.uint8, device="cuda"), torch.empty(ns // 4, device="cuda")
    block.quantize_weights_i4(w.data_ptr(), A, H, group, F32, wq.data_ptr(), ws.data_ptr(), stream())
    q = torch.zeros(rows, layer.row_pitch(H), dtype=torch.int8, device="cuda")
    q[:, :H] = torch.randint(-127, 128, (rows, H), device="cuda", generator=gen, dtype=torch.int8)
    return w, wq, ws, q, torch.rand(rows, device="cuda", generator=gen)


@pytest.mark.parametrize("rows", [3, 30, 60, 400])
def test_replays_of_captured_products(rows):
    say("graphs", rows)
    A, H, group = 300, 700, 64
    w, wq, ws, q, scales = product_of(rows, A, H, group, F32)
    frames = torch.cat((torch.tensor([rows], dtype=torch.int32), torch.arange(rows, dtype=torch.int32))).cuda()
    out = torch.zeros(rows, A, device="cuda")

    def call(s):
        block.quantize_weights_i4(w.data_ptr(), A, H, group, F32, wq.data_ptr(), ws.data_ptr(), s)
        block.linear_i4(q.data_ptr(), scales.data_ptr(), wq.data_ptr(), ws.data_ptr(), group, None, frames.data_ptr(), rows, H, A, F32, out.data_ptr(), s)

    call(stream())
    torch.cuda.synchronize()
    side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        call(torch.cuda.current_stream().cuda_stream)
    for turn in range(4):
        w.mul_(0.5)                                      # (exactly half of everything)
        want = out * 0.5
        out.zero_()
        if turn == 2:
            frames[0] = rows // 2
            want[rows // 2:] = 0.0
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_sums_at_their_largest():
    """The widest state, all of it at the ends of both ranges: 64 columns' sums, 16 times, stay far inside 32 bits."""
    say("largest sums")
    for group in (64, 128, 16384):
        for rows in (1, 40, 130):
            A, H = 20, 16384
            w = torch.full((A, H), 7.0, device="cuda")
            w[1] = -7.0
            nw, ns = block.weights_i4_sizes(A, H, group)
            wq, ws = torch.empty(nw, dtype=torch.uint8, device="cuda"), torch.empty(ns // 4, device="cuda")
            block.quantize_weights_i4(w.data_ptr(), A, H, group, F32, wq.data_ptr(), ws.data_ptr(), stream())
            q, scales = torch.full((rows, H), 127, dtype=torch.int8, device="cuda"), torch.ones(rows, device="cuda")
            out = torch.empty(rows, A, device="cuda")
            block.linear_i4(q.data_ptr(), scales.data_ptr(), wq.data_ptr(), ws.data_ptr(), group, None, None, rows, H, A, F32, out.data_ptr(), stream())
            torch.cuda.synchronize()
            assert bool((out[:, 0] == 127.0 * 7 * H).all()) and bool((out[:, 1] == -127.0 * 7 * H).all())


def test_scales_that_are_not_finite():
    """A row's or a group's NaN scale makes what it enters NaNs, and nothing else."""
    say("scales")
    for rows in (2, 20, 50, 300):
        A, H, group = 40, 300, 64
        w, wq, ws, q, scales = product_of(rows, A, H, group, F32, 1)
        w[3, 70] = float("inf")
        block.quantize_weights_i4(w.data_ptr(), A, H, group, F32, wq.data_ptr(), ws.data_ptr(), stream())
        scales[1] = float("nan")
        out = torch.empty(rows, A, device="cuda")
        block.linear_i4(q.data_ptr(), scales.data_ptr(), wq.data_ptr(), ws.data_ptr(), group, None, None, rows, H, A, F32, out.data_ptr(), stream())
        torch.cuda.synchronize()
        bad = torch.isnan(out)
        assert bool(bad[1].all()) and bool(bad[:, 3].all())
        bad[1], bad[:, 3] = False, False
        assert not bad.any()


def test_products_of_more_than_2_31_activations():
    rows, A, H = 180_000, 12_000, 64
    say("beyond 2^31", rows * A)
    w, wq, ws, q, scales = product_of(rows, A, H, 64, BF16, 2)
    out = torch.empty(rows, A, dtype=torch.bfloat16, device="cuda")
    block.linear_i4(q.data_ptr(), scales.data_ptr(), wq.data_ptr(), ws.data_ptr(), 64, None, None, rows, H, A, BF16, out.data_ptr(), stream())
    few = torch.empty(7, A, dtype=torch.bfloat16, device="cuda")
    last = q[-7:].contiguous()
    block.linear_i4(last.data_ptr(), scales[-7:].data_ptr(), wq.data_ptr(), ws.data_ptr(), 64, None, None, 7, H, A, BF16, few.data_ptr(), stream())
    torch.cuda.synchronize()
    assert torch.equal(out[-7:], few)                    # (one group: no sum of several)


def test_an_error_from_before_is_not_reported():
    """hipSetDevice of a device that is not there: refused on the host, and remembered as the thread's last error; none of these calls' own."""
    lib, before = block.load(), layer.last_hip_error()
    c = Call(20, 300, F32, "all", 300, 11)
    w, wq, ws, q, scales = product_of(20, 30, 300, 64, F32)
    inputs, states, out = torch.zeros(40, 1, 600, device="cuda"), torch.zeros(40, 1, 300, device="cuda"), torch.zeros(20, 30, device="cuda")
    b, outs, norm_ws = buffers(c)
    torch.cuda.synchronize()
    assert lib.hipSetDevice(1000) != 0
    try:                                                 # (each call raises what it reports)
        enqueue(c, b, outs, norm_ws, stream())
        block.recurrence(inputs.data_ptr(), 600, None, None, 32, 1, 300, 300, F32, states.data_ptr(), None, None, 0, stream())
        block.recurrence_backward(states.data_ptr(), None, inputs.data_ptr(), 600, states.data_ptr(), None, None, 32, 1, 300, 300, F32,
                                  torch.empty_like(inputs).data_ptr(), None, None, 0, stream())
        block.quantize_weights_i4(w.data_ptr(), 30, 300, 64, F32, wq.data_ptr(), ws.data_ptr(), stream())
        block.linear_i4(q.data_ptr(), scales.data_ptr(), wq.data_ptr(), ws.data_ptr(), 64, None, None, 20, 300, 30, F32, out.data_ptr(), stream())
        block.dequantize_weights_i4(wq.data_ptr(), ws.data_ptr(), 30, 300, 64, F32, w.data_ptr(), stream())
    finally:
        lib.hipGetLastError()                            # (torch would take it for its own)
    torch.cuda.synchronize()
    assert layer.last_hip_error() == before
