"""Weights in 4 bits against their definition: the whole numbers exactly, the products within what fp32 sums may add."""
import numpy as np
import pytest
import torch

import block_reference as ref
from layer_reference import Guarded, HALF, frame_list, half_step, library_rows, others, pointer, put, stream, torch_type
from paper_1512_02595_amd import block, ctc

pytestmark = pytest.mark.gpu
F32, BF16 = ctc.DTYPE_F32, ctc.DTYPE_BF16
TYPES = [F32, BF16]
NAN = float("nan")


def say(*a):
    print(*a, flush=True)


def weights(A, H, dtype, seed=0):
    rng = np.random.default_rng([A, H, dtype, seed])
    w = rng.standard_normal((A, H)) * np.exp(rng.standard_normal((A, 1)))
    w[rng.random((A, H)) < 0.05] = 0.0
    return torch.from_numpy(w).float().to(torch_type(dtype)).float()


def packed(w, dtype, group, shift=0):
    A, H = w.shape
    nw, ns = block.weights_i4_sizes(A, H, group)
    q, s = Guarded((nw,), torch.uint8), Guarded((ns // 4,), torch.float32)
    dev = put(w, torch_type(dtype), shift)
    block.quantize_weights_i4(dev.t.data_ptr(), A, H, group, dtype, q.t.data_ptr(), s.t.data_ptr(), stream())
    torch.cuda.synchronize()
    assert q.intact() and s.intact()
    return q, s


def check_packed(q, s, w, group):
    A, H = w.shape
    got_q, got_s = ref.unpack_i4(q.t.cpu().numpy(), s.t.cpu().numpy(), A, H, group)
    want_q, want_s = ref.to_i4(w, group)
    assert np.array_equal(got_q.astype(np.float64), want_q.numpy())
    assert np.array_equal(np.isnan(got_s), np.isnan(want_s.numpy()))
    off = np.abs(got_s - want_s.numpy()) <= 1.0001 * HALF * want_s.numpy() + 2.0 ** -150
    assert (off | np.isnan(got_s)).all()
    return got_q, got_s


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("group", [64, 128, 256, 1024, 16384])
@pytest.mark.parametrize("A, H", [(1, 1), (16, 128), (15, 63), (17, 64), (29, 65), (33, 127), (5, 129), (40, 300), (3, 1999), (300, 200), (2, 16384), (20, 4100)])
def test_weights(A, H, group, dtype):
    say("weights", A, H, group, dtype)
    w = weights(A, H, dtype)
    q, s = packed(w, dtype, group, shift=4)
    got_q, got_s = check_packed(q, s, w, group)
    out = Guarded((A, H), torch_type(dtype))
    block.dequantize_weights_i4(q.t.data_ptr(), s.t.data_ptr(), A, H, group, dtype, out.t.data_ptr(), stream())
    torch.cuda.synchronize()
    spread = np.repeat(got_s, group, 1)[:, :H]
    want = torch.from_numpy(got_q.astype(np.float32) * spread).to(torch_type(dtype))
    assert torch.equal(out.t.cpu(), want) and out.intact()


def test_weights_at_middles_and_extremes():
    """Odd multiples of half a step and their neighbours, for tiny and huge groups; zeros; infinities and NaNs."""
    say("weights at middles")
    rng = np.random.default_rng(5)
    A, H, group = 200, 512, 128
    m = np.abs(rng.standard_normal((A, 1))).astype(np.float32) * np.float32(10.0) ** rng.integers(-44, 37, (A, 1)).astype(np.float32)
    w = ((2 * rng.integers(0, 7, (A, H)) + 1) / 14.0 * m.astype(np.float64)).astype(np.float32)
    w = np.where(rng.random((A, H)) < 0.6, np.nextafter(w, np.where(rng.random((A, H)) < 0.5, np.float32(-1e38), np.float32(3e38))), w)
    w *= np.where(rng.random((A, H)) < 0.5, np.float32(-1), np.float32(1))
    w[:, ::group] = m
    w[:20] = np.float32(14.0) * rng.integers(-14, 15, (20, H)) / np.float32(14.0)          # exact middles
    w[:20, ::group] = 14.0
    w[30, :group], w[31, 5], w[32, 200], w[33, 300] = 0.0, np.inf, -np.inf, np.nan
    w = torch.from_numpy(w)
    q, s = packed(w, F32, group)
    check_packed(q, s, w, group)


def rows_of(rows, H, seed=0):
    rng = np.random.default_rng([rows, H, seed])
    q = torch.from_numpy(rng.integers(-127, 128, (rows, H)))
    return q, torch.from_numpy(np.exp(rng.standard_normal(rows))).float()


def product(rows, A, H, group, dtype, kind, bias=True, seed=0):
    say("product", rows, A, H, group, dtype, kind)
    rng = np.random.default_rng([rows, A, H, seed])
    w = weights(A, H, F32, seed)
    wq, ws = packed(w, F32, group)
    got_q, got_s = ref.unpack_i4(wq.t.cpu().numpy(), ws.t.cpu().numpy(), A, H, group)
    q, scales = rows_of(rows, H, seed)
    frames, names = frame_list(kind, rows, rng)
    poisoned = torch.full_like(scales, NAN)
    poisoned[names] = scales[names]
    q_dev, s_dev = library_rows(q, poisoned, H)
    b = torch.from_numpy(rng.standard_normal(A)).float()
    b_dev = put(b, torch.float32)
    out = Guarded((rows, A), torch_type(dtype))
    block.linear_i4(q_dev.t.data_ptr(), s_dev.t.data_ptr(), wq.t.data_ptr(), ws.t.data_ptr(), group, b_dev.t.data_ptr() if bias else None,
                    pointer(frames), rows, H, A, dtype, out.t.data_ptr(), stream())
    torch.cuda.synchronize()
    total, size = torch.zeros(len(names), A, dtype=torch.float64), torch.zeros(len(names), A, dtype=torch.float64)
    wide, spread = torch.from_numpy(got_q).double(), torch.from_numpy(np.repeat(got_s, group, 1)[:, :H]).double()
    step = 64 if group == 64 else 128
    steps = 0
    for k in range(0, H, step):
        part = (q[names][:, k:k + step].double() @ wide[:, k:k + step].t().contiguous()) * spread[:, k]
        total += part
        size += part.abs()
        steps += 1
    by = scales[names].double()[:, None]
    want = total * by + (b.double() if bias else 0.0)
    # each step's share is rounded when it is added, with all that follow; four wavefronts' sums, the row's scale, the bias
    bound = (2 * steps + 8) * HALF * size * by.abs()
    tolerance = bound + (HALF + half_step(dtype)) * (want.abs() + bound) + 2.0 ** -140
    off = (out.t.cpu()[names].double() - want).abs() / tolerance
    worst = float(off.max()) if off.numel() else 0.0
    say("   %.3f of what is allowed" % worst)
    assert worst <= 1 and out.untouched(others(rows, names)) and out.intact()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("group", [64, 128, 384])
@pytest.mark.parametrize("rows", [1, 2, 15, 16, 17, 33, 64, 65, 130])
@pytest.mark.parametrize("A, H", [(1, 1), (29, 200), (16, 128), (70, 1000), (300, 129)])
def test_product(rows, A, H, group, dtype):
    product(rows, A, H, group, dtype, "all")


@pytest.mark.parametrize("kind", ["some", "none", "odd entries"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [5, 16, 40, 70, 200])
def test_product_of_listed_rows(rows, dtype, kind):
    for group in (64, 128):
        product(rows, 77, 500, group, dtype, kind, bias=rows != 40)


@pytest.mark.parametrize("kind", ["some", "none", "odd entries"])
@pytest.mark.parametrize("dtype", TYPES)
def test_product_of_many_listed_rows(dtype, kind):
    product(6300, 450, 200, 64, dtype, kind)
    product(3200, 900, 300, 128, dtype, kind, bias=False)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, A, H, group", [(1, 6000, 2048, 128), (1, 29, 16384, 64), (3, 6000, 700, 64), (64, 2100, 1024, 128), (500, 29, 640, 64),
                                               (257, 1025, 1999, 128), (1000, 4000, 130, 64), (2, 70000, 64, 64), (6300, 500, 130, 64), (2000, 1600, 1000, 128), (1600, 2000, 333, 384),
                                               (65, 25000, 64, 64), (12, 5000, 300, 64), (1, 4500, 4200, 128), (500, 2000, 640, 64)])
def test_product_of_many(rows, A, H, group, dtype):
    product(rows, A, H, group, dtype, "all")
