"""The output layer's calls against their definitions in 64 bits: odd sizes, lists of rows of every kind, both types,
alignments, values that are not finite, and what may be done with the calls (graphs, streams, buffers given twice)."""
import numpy as np
import pytest
import torch

import layer_reference as ref
from layer_reference import HALF, Guarded, frame_list, half_step, others, pointer, poisoned, put, stream, torch_type
from paper_1512_02595_amd import ctc, layer

pytestmark = pytest.mark.gpu
F32, BF16 = ctc.DTYPE_F32, ctc.DTYPE_BF16
TYPES = [F32, BF16]
LISTS = ["all", "some", "none", "odd entries"]


def states(rng, rows, H, dtype):
    """Values of unlike size, some zero, held exactly by `dtype`."""
    x = rng.standard_normal((rows, H)) * np.exp(rng.standard_normal((rows, 1)) * 3 + 0.5 * rng.standard_normal((1, H)))
    x[rng.random((rows, H)) < 0.05] = 0.0
    return torch.from_numpy(x).float().to(torch_type(dtype)).float()


def say(*a):
    print(*a, flush=True)


# ---- the list of frames -----------------------------------------------------------------------------------------

@pytest.mark.parametrize("T, B", [(1, 1), (1, 300), (7, 5), (50, 4), (33, 64), (20, 65), (5, 129), (750, 64), (3, 4097)])
def test_pack_frames(T, B):
    say("pack", T, B)
    rng = np.random.default_rng(T * 1000 + B)
    lengths = rng.integers(0, T + 1, B).astype(np.int32)
    lengths[rng.random(B) < 0.1] = 0
    if B > 3:
        lengths[0], lengths[1], lengths[2], lengths[3] = T, -3, T + 9, 2 ** 31 - 1
    frames = Guarded((1 + T * B,), torch.int32)
    dev = torch.from_numpy(lengths).cuda()
    layer.pack_frames(dev.data_ptr(), T, B, frames.t.data_ptr(), stream())
    torch.cuda.synchronize()
    got = frames.t.cpu().numpy()
    want = [t * B + b for t in range(T) for b in range(B) if t < min(lengths[b], T)]
    assert got[0] == len(want)
    assert np.array_equal(np.sort(got[1:1 + len(want)]), want)
    assert (got[1 + len(want):] == np.frombuffer(bytes([ref.PATTERN] * 4), np.int32)[0]).all() and frames.intact()


# ---- 8 bits and back --------------------------------------------------------------------------------------------

def check_rows(q, scales, u, names, rows, H, factor=None, scale_bound=HALF):
    """Whole numbers exactly; a scale is rounded once."""
    want_q, want_s = ref.to_levels(u)
    if factor is not None:
        want_s = want_s * factor
    got_q, got_s = q.t.cpu()[names], scales.t.cpu()[names].double()
    assert torch.equal(got_q[:, :H].double(), want_q)
    assert not got_q[:, H:].any()
    assert torch.equal(torch.isnan(got_s), torch.isnan(want_s))
    fine = ~torch.isnan(want_s)
    # (an fp32 below 2^-126 has an absolute step of 2^-149)
    assert ((got_s - want_s).abs()[fine] <= 1.0001 * scale_bound * want_s[fine] + 2.0 ** -150).all()
    rest = others(rows, names)
    assert q.untouched(rest) and scales.untouched(rest) and q.intact() and scales.intact()


WIDTHS = [1, 3, 64, 100, 128, 511, 513, 1000, 1999, 2049, 4096, 4100, 9000, 16384]


@pytest.mark.parametrize("kind", LISTS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H", WIDTHS)
def test_quantize_rows(H, dtype, kind):
    say("quantize", H, dtype, kind)
    rng = np.random.default_rng(H)
    rows = 37
    x = states(rng, rows, H, dtype)
    x[5] = 0.0
    frames, names = frame_list(kind, rows, rng)
    dev = put(poisoned(x, names), torch_type(dtype))
    q, scales = Guarded((rows, layer.row_pitch(H)), torch.int8), Guarded((rows,), torch.float32)
    layer.quantize_rows(dev.t.data_ptr(), pointer(frames), rows, H, dtype, q.t.data_ptr(), scales.t.data_ptr(), stream())
    torch.cuda.synchronize()
    check_rows(q, scales, x[names], names, rows, H)
    # ... and back: one rounding of the product, one more to bf16
    out = Guarded((rows, H), torch_type(dtype))
    layer.dequantize_rows(q.t.data_ptr(), scales.t.data_ptr(), pointer(frames), rows, H, dtype, out.t.data_ptr(), stream())
    torch.cuda.synchronize()
    want = (q.t.cpu()[names][:, :H].float() * scales.t.cpu()[names][:, None]).to(torch_type(dtype))
    assert torch.equal(out.t.cpu()[names], want)
    assert out.untouched(others(rows, names)) and out.intact()


def test_ties_and_their_neighbours():
    """m = 254: every odd multiple of 1 is halfway between two whole numbers; its neighbours in fp32 are not."""
    odd = np.arange(1, 254, 2, dtype=np.float32)
    rows = np.stack([odd, np.nextafter(odd, np.float32(0)), np.nextafter(odd, np.float32(999)), -odd,
                     odd * np.float32(2.0 ** -140), odd * np.float32(2.0 ** 119)])
    rows = np.concatenate([rows, np.float32(254) * np.array([[1], [1], [1], [1], [2.0 ** -140], [2.0 ** 119]], np.float32)], 1)
    n, H = rows.shape
    dev = put(torch.from_numpy(rows), torch.float32)
    q, scales = Guarded((n, layer.row_pitch(H)), torch.int8), Guarded((n,), torch.float32)
    layer.quantize_rows(dev.t.data_ptr(), None, n, H, F32, q.t.data_ptr(), scales.t.data_ptr(), stream())
    torch.cuda.synchronize()
    got = q.t.cpu().numpy()[:, :H - 1].astype(int)
    low = (odd.astype(int) - 1) // 2
    even = low + low % 2
    assert np.array_equal(got[0], even) and np.array_equal(got[1], low) and np.array_equal(got[2], low + 1)
    assert np.array_equal(got[3], -even) and np.array_equal(got[4], even) and np.array_equal(got[5], even)
    check_rows(q, scales, torch.from_numpy(rows), np.arange(n), n, H)


def test_rows_near_middles():
    """Many values at and around the middles between whole numbers, for largest values of every kind."""
    rng = np.random.default_rng(3)
    n, H = 400, 1500
    m = np.abs(rng.standard_normal((n, 1))).astype(np.float32) * np.float32(10.0) ** rng.integers(-44, 37, (n, 1)).astype(np.float32)
    middle = ((2 * rng.integers(0, 127, (n, H)) + 1) / 254.0 * m.astype(np.float64)).astype(np.float32)
    for _ in range(2):
        middle = np.nextafter(middle, np.where(rng.random((n, H)) < 0.5, np.float32(-1e38), np.float32(3e38)))
    x = np.where(np.abs(middle) <= m, middle, m).astype(np.float32)
    x[:, 7] = m[:, 0]
    dev = put(torch.from_numpy(x), torch.float32)
    q, scales = Guarded((n, layer.row_pitch(H)), torch.int8), Guarded((n,), torch.float32)
    layer.quantize_rows(dev.t.data_ptr(), None, n, H, F32, q.t.data_ptr(), scales.t.data_ptr(), stream())
    torch.cuda.synchronize()
    check_rows(q, scales, torch.from_numpy(x), np.arange(n), n, H)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H", [5, 700, 3000, 9001])
def test_rows_that_are_not_finite(H, dtype):
    rng = np.random.default_rng(H)
    x = states(rng, 6, H, dtype)
    x[0, H - 1], x[1, 0], x[2, H // 2], x[3, 0] = float("nan"), float("inf"), -float("inf"), 0.0
    dev = put(x, torch_type(dtype))
    q, scales = Guarded((6, layer.row_pitch(H)), torch.int8), Guarded((6,), torch.float32)
    layer.quantize_rows(dev.t.data_ptr(), None, 6, H, dtype, q.t.data_ptr(), scales.t.data_ptr(), stream())
    torch.cuda.synchronize()
    check_rows(q, scales, x, np.arange(6), 6, H)
    assert torch.isnan(scales.t[:3]).all() and not torch.isnan(scales.t[3:]).any()


@pytest.mark.parametrize("shift", [2, 4, 6, 8, 12, 14])
@pytest.mark.parametrize("dtype", TYPES)
def test_rows_off_a_vectors_alignment(dtype, shift):
    if shift % (4 if dtype == F32 else 2):
        pytest.skip("not aligned to an element")
    rng = np.random.default_rng(shift)
    rows, H = 9, 1029
    x = states(rng, rows, H, dtype)
    dev = put(x, torch_type(dtype), shift)
    q, scales = Guarded((rows, layer.row_pitch(H)), torch.int8), Guarded((rows,), torch.float32)
    layer.quantize_rows(dev.t.data_ptr(), None, rows, H, dtype, q.t.data_ptr(), scales.t.data_ptr(), stream())
    out = Guarded((rows, H), torch_type(dtype), shift)
    layer.dequantize_rows(q.t.data_ptr(), scales.t.data_ptr(), None, rows, H, dtype, out.t.data_ptr(), stream())
    torch.cuda.synchronize()
    check_rows(q, scales, x, np.arange(rows), rows, H)
    assert torch.equal(out.t.cpu(), (q.t.cpu()[:, :H].float() * scales.t.cpu()[:, None]).to(torch_type(dtype))) and out.intact()


# ---- the norm ---------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("kind", LISTS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H", WIDTHS)
def test_rms_norm(H, dtype, kind):
    say("norm", H, dtype, kind)
    rng = np.random.default_rng(H + 1)
    rows, eps = 29, 1e-5
    x, y = states(rng, rows, H, dtype), states(rng, rows, H, dtype)
    w = torch.from_numpy(1.0 + 0.5 * rng.standard_normal(H)).float()
    x[3], y[3] = 0.0, 0.0
    frames, names = frame_list(kind, rows, rng)
    t = torch_type(dtype)
    dx, dr, dw = put(poisoned(x, names), t), put(poisoned(y, names), t), put(w, torch.float32)
    total, q, scales = Guarded((rows, H), t), Guarded((rows, layer.row_pitch(H)), torch.int8), Guarded((rows,), torch.float32)
    layer.rms_norm_i8(dx.t.data_ptr(), dr.t.data_ptr(), dw.t.data_ptr(), eps, pointer(frames), rows, H, dtype,
                      total.t.data_ptr(), q.t.data_ptr(), scales.t.data_ptr(), stream())
    torch.cuda.synchronize()
    z = (x + y).to(t)[names]
    assert torch.equal(total.t.cpu()[names], z)
    assert total.untouched(others(rows, names)) and total.intact()
    # (the factor is formed in fp64 from eps as a float)
    factor = ref.rms(z.double(), float(np.float32(eps)))
    check_rows(q, scales, z.float() * w, names, rows, H, factor)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H", [100, 2500])
def test_rms_norm_without_its_options(H, dtype):
    rng = np.random.default_rng(H)
    rows, eps = 11, 1e-6
    x = states(rng, rows, H, dtype)
    dx = put(x, torch_type(dtype))
    q, scales = Guarded((rows, layer.row_pitch(H)), torch.int8), Guarded((rows,), torch.float32)
    layer.rms_norm_i8(dx.t.data_ptr(), None, None, eps, None, rows, H, dtype, None, q.t.data_ptr(), scales.t.data_ptr(), stream())
    torch.cuda.synchronize()
    check_rows(q, scales, x, np.arange(rows), rows, H, ref.rms(x.double(), float(np.float32(eps))))


@pytest.mark.parametrize("which", ["x", "residual"])
def test_the_sum_may_replace_an_input(which):
    rng = np.random.default_rng(5)
    rows, H = 17, 1500
    x, y = states(rng, rows, H, BF16), states(rng, rows, H, BF16)
    dx, dr = put(x, torch.bfloat16), put(y, torch.bfloat16)
    into = dx if which == "x" else dr
    q, scales = Guarded((rows, layer.row_pitch(H)), torch.int8), Guarded((rows,), torch.float32)
    layer.rms_norm_i8(dx.t.data_ptr(), dr.t.data_ptr(), None, 1e-6, None, rows, H, BF16, into.t.data_ptr(), q.t.data_ptr(),
                      scales.t.data_ptr(), stream())
    torch.cuda.synchronize()
    z = (x + y).to(torch.bfloat16)
    assert torch.equal(into.t.cpu(), z) and into.intact()
    check_rows(q, scales, z.float(), np.arange(rows), rows, H, ref.rms(z.double(), float(np.float32(1e-6))))


def test_norms_of_huge_and_tiny_rows():
    """Squares beyond fp32's range on either side are held; a product with the weight that is beyond it is not finite."""
    rng = np.random.default_rng(6)
    rows, H = 6, 900
    x = torch.from_numpy(rng.standard_normal((rows, H))).float()
    x *= torch.tensor([1e30, 1e-30, 1e-40, 3e37, 1e-20, 1e20])[:, None]
    w = torch.full((H,), 3.0)
    w[11] = 1e3
    x[3, 11] = 2e36                                      # times 1e3: beyond fp32
    dx, dw = put(x, torch.float32), put(w, torch.float32)
    q, scales = Guarded((rows, layer.row_pitch(H)), torch.int8), Guarded((rows,), torch.float32)
    layer.rms_norm_i8(dx.t.data_ptr(), None, dw.t.data_ptr(), 1e-30, None, rows, H, F32, None, q.t.data_ptr(),
                      scales.t.data_ptr(), stream())
    torch.cuda.synchronize()
    assert torch.isnan(scales.t[3]) and not torch.isnan(scales.t[[0, 1, 2, 4, 5]]).any()
    check_rows(q, scales, x * w, np.arange(rows), rows, H, ref.rms(x.double(), float(np.float32(1e-30))))


def backward(dy, z, w, dres, dtype, rows, H, eps, frames=None, into=None, want_weight=True):
    out = into if into is not None else Guarded((rows, H), torch_type(dtype))
    dweight = Guarded((H,), torch.float32) if want_weight else None
    size = layer.rms_norm_workspace_size(rows, H)
    ws = torch.full((size + 256,), 0xFF, dtype=torch.uint8, device="cuda")
    at = (ws.data_ptr() + 255) // 256 * 256
    layer.rms_norm_backward(dy.t.data_ptr(), z.t.data_ptr(), None if w is None else w.t.data_ptr(), eps,
                            None if dres is None else dres.t.data_ptr(), pointer(frames), rows, H, dtype, out.t.data_ptr(),
                            dweight.t.data_ptr() if want_weight else None, at if want_weight else None,
                            size if want_weight else 0, stream())
    torch.cuda.synchronize()
    return out, dweight


def check_backward(out, dweight, dy, z, w, dres, dtype, rows, H, eps, names):
    dz, dw, bound, terms = ref.norm_backward(dy[names].double(), z[names].double(), w.double(), float(np.float32(eps)),
                                             None if dres is None else dres[names].double())
    got = out.t.cpu()[names].double()
    assert ((got - dz).abs() <= 1.001 * bound + half_step(dtype) * (dz.abs() + bound) + 1e-40).all()
    if dweight is not None:
        # a thread adds up to `rows` terms of three roundings each, four of which sums are added; then fp64 and one rounding
        assert ((dweight.t.cpu().double() - dw).abs() <= HALF * (len(names) + 8) * terms + 1e-40).all()
        assert dweight.intact()


@pytest.mark.parametrize("kind", LISTS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H", WIDTHS)
def test_rms_norm_backward(H, dtype, kind):
    say("norm backward", H, dtype, kind)
    rng = np.random.default_rng(H + 2)
    rows, eps, t = 43, 1e-5, torch_type(dtype)
    z, dy, dres = states(rng, rows, H, dtype), states(rng, rows, H, dtype), states(rng, rows, H, dtype)
    z[4] = 0.0
    w = torch.from_numpy(1.0 + 0.5 * rng.standard_normal(H)).float()
    frames, names = frame_list(kind, rows, rng)
    out, dweight = backward(put(poisoned(dy, names), t), put(poisoned(z, names), t), put(w, torch.float32),
                            put(poisoned(dres, names), t), dtype, rows, H, eps, frames)
    check_backward(out, dweight, dy, z, w, dres, dtype, rows, H, eps, names)
    assert out.untouched(others(rows, names)) and out.intact()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, H", [(1, 40), (1, 2048), (3, 5000), (5000, 70), (9000, 130)])
def test_rms_norm_backward_without_its_options(rows, H, dtype):
    rng = np.random.default_rng(rows)
    z, dy = states(rng, rows, H, dtype), states(rng, rows, H, dtype)
    t = torch_type(dtype)
    out, dweight = backward(put(dy, t), put(z, t), None, None, dtype, rows, H, 1e-6)
    check_backward(out, dweight, dy, z, torch.ones(H), None, dtype, rows, H, 1e-6, np.arange(rows))
    again, _ = backward(put(dy, t), put(z, t), None, None, dtype, rows, H, 1e-6, want_weight=False)
    assert torch.equal(again.t, out.t) and out.intact()


def test_norm_gradients_of_huge_and_tiny_rows():
    """Both terms of a gradient of ordinary size, where the sums and their gradients are far from it on either side."""
    rng = np.random.default_rng(12)
    rows, H = 5, 700
    size = torch.tensor([1e25, 1e-25, 1e30, 1e-15, 1e19])[:, None]
    z, dy = (torch.from_numpy(rng.standard_normal((rows, H)) + 1.0).float() * size for _ in range(2))
    w = torch.from_numpy(1.0 + 0.5 * rng.standard_normal(H)).float()
    out, dweight = backward(put(dy, torch.float32), put(z, torch.float32), put(w, torch.float32), None, F32, rows, H, 1e-30)
    for r in range(rows):
        check_backward(out, None, dy, z, w, None, F32, rows, H, 1e-30, np.array([r]))
    check_backward(out, dweight, dy, z, w, None, F32, rows, H, 1e-30, np.arange(rows))


@pytest.mark.parametrize("which", ["dy", "sum", "dresidual"])
def test_the_gradient_may_replace_an_input(which):
    rng = np.random.default_rng(8)
    rows, H = 21, 3000
    z, dy, dres = (states(rng, rows, H, BF16) for _ in range(3))
    w = torch.from_numpy(1.0 + 0.5 * rng.standard_normal(H)).float()
    t = torch.bfloat16
    bufs = {"dy": put(dy, t), "sum": put(z, t), "dresidual": put(dres, t)}
    out, dweight = backward(bufs["dy"], bufs["sum"], put(w, torch.float32), bufs["dresidual"], BF16, rows, H, 1e-6,
                            into=bufs[which])
    check_backward(out, dweight, dy, z, w, dres, BF16, rows, H, 1e-6, np.arange(rows))


def test_norm_gradient_against_differences():
    """The formula's derivative against central differences of y, in 64 bits, and the call against both."""
    rng = np.random.default_rng(9)
    rows, H, eps = 3, 50, float(np.float32(1e-3))
    z, dy = torch.from_numpy(rng.standard_normal((rows, H))).float(), torch.from_numpy(rng.standard_normal((rows, H))).float()
    w = torch.from_numpy(1.0 + 0.5 * rng.standard_normal(H)).float()

    def loss(zz, ww):
        return (dy.double() * (zz * ref.rms(zz, eps)[:, None] * ww)).sum()

    h = 1e-5
    dz, dw = torch.zeros(rows, H, dtype=torch.float64), torch.zeros(H, dtype=torch.float64)
    for k in range(H):
        e = torch.zeros(H, dtype=torch.float64)
        e[k] = h
        dw[k] = (loss(z.double(), w.double() + e) - loss(z.double(), w.double() - e)) / (2 * h)
        for r in range(rows):
            d = torch.zeros(rows, H, dtype=torch.float64)
            d[r, k] = h
            dz[r, k] = (loss(z.double() + d, w.double()) - loss(z.double() - d, w.double())) / (2 * h)
    # (central differences: h^2 times a third derivative of order 10, and 1e-16 / h times values of order 50)
    out, dweight = backward(put(dy, torch.float32), put(z, torch.float32), put(w, torch.float32), None, F32, rows, H, eps)
    assert (out.t.cpu().double() - dz).abs().max() < 1e-5
    assert (dweight.t.cpu().double() - dw).abs().max() < 1e-5
    assert not dz.abs().max() < 1e-2


# ---- activations ------------------------------------------------------------------------------------------------

def levels(rng, rows, H, dense=True):
    q = rng.integers(-127, 128, (rows, H))
    if not dense:
        q[rng.random((rows, H)) < 0.9] = 0
    return torch.from_numpy(q), torch.from_numpy(np.exp(rng.standard_normal(rows)) * 0.01).float()


def linear(q, s, wq, ws, bias, dtype, frames=None, shift=0):
    rows, A, H = q.shape[0], wq.shape[0], q.shape[1]
    gq, gs = ref.library_rows(q, s, H)
    gw, gws = ref.library_rows(wq, ws, H)
    gb = None if bias is None else put(bias, torch.float32)
    out = Guarded((rows, A), torch_type(dtype), shift)
    layer.linear_i8(gq.t.data_ptr(), gs.t.data_ptr(), gw.t.data_ptr(), gws.t.data_ptr(),
                    None if gb is None else gb.t.data_ptr(), pointer(frames), rows, H, A, dtype, out.t.data_ptr(), stream())
    torch.cuda.synchronize()
    return out


def check_linear(out, q, s, wq, ws, bias, dtype, names):
    total = q[names].double() @ wq.double().t()
    product = total * s[names].double()[:, None] * ws.double()[None, :]
    want = product + (0.0 if bias is None else bias.double())
    got = out.t.cpu()[names].double()
    # the sum as a float, the scales' product and its product with the sum: a half step each; one for the bias
    bound = HALF * (3.001 * product.abs() + want.abs()) + 1e-40
    assert ((got - want).abs() <= bound + half_step(dtype) * (want.abs() + bound)).all()
    assert out.untouched(others(out.t.shape[0], names)) and out.intact()


SHAPES = [(1, 1, 1), (1, 2048, 6000), (2, 64, 29), (3, 100, 29), (16, 300, 64), (17, 129, 65), (5, 4096, 33), (64, 500, 750),
          (65, 640, 31), (100, 16384, 20), (130, 1111, 473), (257, 256, 257), (300, 77, 1000), (515, 384, 130),
          (1000, 1000, 29), (700, 512, 600), (33, 900, 3000), (9, 4000, 5001)]


@pytest.mark.parametrize("kind", LISTS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, H, A", SHAPES)
def test_linear(rows, H, A, dtype, kind):
    say("linear", rows, H, A, dtype, kind)
    rng = np.random.default_rng(rows * 7 + H + A)
    q, s = levels(rng, rows, H)
    wq, ws = levels(rng, A, H)
    bias = torch.from_numpy(rng.standard_normal(A)).float()
    frames, names = frame_list(kind, rows, rng)
    out = linear(q, s, wq, ws, bias, dtype, frames)
    check_linear(out, q, s, wq, ws, bias, dtype, names)


@pytest.mark.parametrize("kind", ["all", "some", "odd entries"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, H, A", [(5700, 300, 5801), (6000, 128, 5700), (5900, 513, 5640), (9000, 200, 900)])
def test_linear_of_many_tiles(rows, H, A, dtype, kind):
    say("many tiles", rows, H, A, dtype, kind)
    rng = np.random.default_rng(rows + H)
    q, s = levels(rng, rows, H)
    wq, ws = levels(rng, A, H)
    bias = torch.from_numpy(rng.standard_normal(A)).float()
    frames, names = frame_list(kind, rows, rng)
    out = linear(q, s, wq, ws, bias, dtype, frames)
    check_linear(out, q, s, wq, ws, bias, dtype, names)


@pytest.mark.parametrize("dtype", TYPES)
def test_linear_without_bias_at_its_extremes(dtype):
    """Every product 127 * 127: sums of 16384 of them are exact."""
    rows, H, A = 40, 16384, 50
    q, s = torch.full((rows, H), 127), torch.full((rows,), 0.5)
    wq, ws = torch.full((A, H), -127), torch.full((A,), 2.0)
    q[3:6] = -127
    out = linear(q, s, wq, ws, None, dtype)
    check_linear(out, q, s, wq, ws, None, dtype, np.arange(rows))
    if dtype == F32:
        assert out.t[0, 0].item() == -127 * 127 * 16384 and out.t[4, 1].item() == 127 * 127 * 16384


@pytest.mark.parametrize("dtype, shift", [(F32, 4), (F32, 8), (BF16, 2), (BF16, 6), (BF16, 12)])
@pytest.mark.parametrize("rows, H, A", [(70, 200, 30), (300, 200, 300)])
def test_activations_off_a_vectors_alignment(rows, H, A, dtype, shift):
    rng = np.random.default_rng(shift)
    q, s = levels(rng, rows, H)
    wq, ws = levels(rng, A, H)
    out = linear(q, s, wq, ws, None, dtype, shift=shift)
    check_linear(out, q, s, wq, ws, None, dtype, np.arange(rows))


@pytest.mark.parametrize("A", [29, 500])
def test_a_row_that_is_not_finite_stays_alone(A):
    rng = np.random.default_rng(A)
    rows, H = 80, 300
    q, s = levels(rng, rows, H)
    wq, ws = levels(rng, A, H)
    s[13] = float("nan")
    q[13] = 0
    out = linear(q, s, wq, ws, None, F32).t.cpu()
    assert torch.isnan(out[13]).all() and not torch.isnan(out[torch.arange(rows) != 13]).any()


# ---- gradient of the weights ------------------------------------------------------------------------------------

def weight_gradient(grads, q, s, dtype, frames=None, want_bias=True, names=None, shift=0):
    rows, A, H = q.shape[0], grads.shape[1], q.shape[1]
    gq, gs = ref.library_rows(q, s, H)
    g = put(grads if names is None else poisoned(grads, names), torch_type(dtype), shift)
    dweight, dbias = Guarded((A, H), torch.float32), Guarded((A,), torch.float32)
    size = layer.weight_gradient_workspace_size(rows, H, A)
    ws = torch.full((size + 256,), 0xFF, dtype=torch.uint8, device="cuda")
    at = (ws.data_ptr() + 255) // 256 * 256
    layer.weight_gradient_i8(g.t.data_ptr(), gq.t.data_ptr(), gs.t.data_ptr(), pointer(frames), rows, H, A, dtype,
                             dweight.t.data_ptr(), dbias.t.data_ptr() if want_bias else None, at, size, stream())
    torch.cuda.synchronize()
    assert dweight.intact() and dbias.intact()
    return dweight, dbias


def check_gradient(dweight, dbias, grads, q, s, names):
    g, y = grads[names].double(), q[names].double() * s[names].double()[:, None]
    want, terms = g.t().contiguous() @ y, g.abs().t().contiguous() @ y.abs()
    # a term is one rounded product of gradient and scale times a whole number, in three parts; each of a sum's additions
    # is off by half a step of a partial sum, which is at most the sum of the terms' sizes
    bound = HALF * (3 * len(names) + 8) * terms + 1e-38
    assert ((dweight.t.cpu().double() - want).abs() <= bound).all()
    if dbias is not None:
        want, terms = g.sum(0), g.abs().sum(0)
        assert ((dbias.t.cpu().double() - want).abs() <= HALF * (len(names) + 8) * terms + 1e-38).all()


def gradients(rng, rows, A, dtype):
    """A softmax less one symbol a row."""
    g = rng.standard_normal((rows, A)) * 2
    g = np.exp(g - g.max(1, keepdims=True))
    g /= g.sum(1, keepdims=True)
    g[np.arange(rows), rng.integers(0, A, rows)] -= 1.0
    return torch.from_numpy(g).float().to(torch_type(dtype)).float()


GRADIENT_SHAPES = [(1, 1, 1), (1, 300, 29), (2, 64, 64), (7, 100, 29), (31, 129, 33), (64, 640, 65), (100, 1000, 29),
                   (333, 77, 500), (1000, 257, 257), (3000, 130, 20), (5000, 60, 3), (400, 2000, 300), (40, 16384, 21),
                   (90, 50, 5001)]


@pytest.mark.parametrize("kind", LISTS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, H, A", GRADIENT_SHAPES)
def test_weight_gradient(rows, H, A, dtype, kind):
    say("weight gradient", rows, H, A, dtype, kind)
    rng = np.random.default_rng(rows * 5 + H + A)
    q, s = levels(rng, rows, H, dense=H % 2 == 0)
    grads = gradients(rng, rows, A, dtype)
    frames, names = frame_list(kind, rows, rng)
    dweight, dbias = weight_gradient(grads, q, s, dtype, frames, names=names)
    check_gradient(dweight, dbias, grads, q, s, names)
    if not len(names):
        assert not dweight.t.any() and not dbias.t.any()


# (two tiles of symbols or more that the narrow kernel takes, and tiles of 128 symbols by 512 columns: several slabs, one)
MANY_SYMBOLS = [(130, 1999, 200), (3000, 300, 191), (5000, 520, 65), (33, 5000, 5001), (200, 1999, 5001), (4000, 1111, 2999), (9000, 700, 2001)]


@pytest.mark.parametrize("kind", LISTS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, H, A", MANY_SYMBOLS)
def test_weight_gradient_of_many_symbols(rows, H, A, dtype, kind):
    say("weight gradient, many symbols", rows, H, A, dtype, kind)
    rng = np.random.default_rng(rows + H + A)
    q, s = levels(rng, rows, H)
    grads = gradients(rng, rows, A, dtype)
    frames, names = frame_list(kind, rows, rng)
    dweight, dbias = weight_gradient(grads, q, s, dtype, frames, names=names)
    check_gradient(dweight, dbias, grads, q, s, names)
    again, _ = weight_gradient(grads, q, s, dtype, frames, want_bias=False, names=names)
    assert torch.equal(again.t, dweight.t)


@pytest.mark.parametrize("dtype, shift", [(F32, 4), (BF16, 2)])
def test_gradients_of_many_symbols_off_alignment_with_a_nan(dtype, shift):
    rng = np.random.default_rng(shift + 50)
    rows, H, A = 200, 1999, 5001
    q, s = levels(rng, rows, H)
    grads = gradients(rng, rows, A, dtype)
    check_gradient(*weight_gradient(grads, q, s, dtype, shift=shift), grads, q, s, np.arange(rows))
    grads[77, 5000] = float("nan")
    grads[78, 5] = float("inf")
    dweight, dbias = weight_gradient(grads, q, s, dtype, shift=shift)
    whole = torch.ones(A, dtype=torch.bool)
    whole[[5, 5000]] = False
    got = dweight.t.cpu()
    assert torch.isnan(got[~whole]).all() and torch.isfinite(got[whole]).all()
    assert not torch.isfinite(dbias.t.cpu()[~whole]).any() and torch.isfinite(dbias.t.cpu()[whole]).all()


def test_weight_gradient_of_many_symbols_holds_gradients_of_every_size():
    """As below, where symbols share tiles of 128 and are lifted by powers of two of their own."""
    rng = np.random.default_rng(13)
    rows, H, A = 240, 1999, 5001
    grads = (gradients(rng, rows, A, F32).double() * torch.from_numpy(10.0 ** rng.integers(-22, 23, (1, A)))).float()
    q, s = levels(rng, rows, H)
    s = s * torch.from_numpy(10.0 ** rng.integers(-2, 3, rows)).float()
    dweight, dbias = weight_gradient(grads, q, s, F32)
    y = q.double() * s.double()[:, None]
    want = grads.double().t().contiguous() @ y
    off = (dweight.t.cpu().double() - want).norm(dim=1) / want.norm(dim=1)
    assert off.max() < 2e-6


@pytest.mark.parametrize("A", [40, 100, 301])
@pytest.mark.parametrize("dtype", TYPES)
def test_weight_gradient_holds_gradients_of_every_size(dtype, A):
    """Symbols whose gradients are 1e-30 and 1e30 times the others', row scales from 1e-8 to 1e8: each sum is as exact as
    its own terms."""
    rng = np.random.default_rng(11)
    rows, H = 600, 200
    grads = gradients(rng, rows, A, dtype).double() * torch.from_numpy(10.0 ** rng.integers(-22, 23, (1, A)))
    grads = grads.float().to(torch_type(dtype)).float()
    q, s = levels(rng, rows, H)
    s = s * torch.from_numpy(10.0 ** rng.integers(-8, 8, rows)).float()
    dweight, dbias = weight_gradient(grads, q, s, dtype)
    check_gradient(dweight, dbias, grads, q, s, np.arange(rows))
    # (the products are as fp32 holds them: the sums' error in the 2-norm, column by column, is that of adding them up)
    y = q.double() * s.double()[:, None]
    want = grads.double().t().contiguous() @ y
    off = (dweight.t.cpu().double() - want).norm(dim=1) / want.norm(dim=1)
    assert off.max() < 2e-6                              # (16-bit products would be off by 2^-17 each: 4e-6)


@pytest.mark.parametrize("dtype, shift", [(F32, 4), (F32, 12), (BF16, 2), (BF16, 10)])
@pytest.mark.parametrize("A", [29, 300])
def test_gradients_off_a_vectors_alignment(A, dtype, shift):
    rng = np.random.default_rng(shift)
    rows, H = 150, 333
    q, s = levels(rng, rows, H)
    grads = gradients(rng, rows, A, dtype)
    dweight, dbias = weight_gradient(grads, q, s, dtype, shift=shift)
    check_gradient(dweight, dbias, grads, q, s, np.arange(rows))
    again, untouched = weight_gradient(grads, q, s, dtype, want_bias=False, shift=shift)
    assert torch.equal(again.t, dweight.t)
    assert untouched.untouched(torch.ones(A, dtype=torch.bool, device="cuda"))


@pytest.mark.parametrize("A", [29, 300])
def test_a_nan_shows_in_its_symbol(A):
    rng = np.random.default_rng(A)
    rows, H = 200, 140
    q, s = levels(rng, rows, H)
    grads = gradients(rng, rows, A, F32)
    grads[77, 5] = float("nan")
    dweight, dbias = weight_gradient(grads, q, s, F32)
    other = torch.arange(A) != 5
    got = dweight.t.cpu()
    assert torch.isnan(got[5]).all() and not torch.isnan(got[other]).any()
    assert torch.isnan(dbias.t[5]) and not torch.isnan(dbias.t.cpu()[other]).any()


def test_a_row_named_twice_counts_twice():
    rng = np.random.default_rng(12)
    rows, H, A = 50, 200, 30
    q, s = levels(rng, rows, H)
    grads = gradients(rng, rows, A, F32)
    names = rng.integers(0, rows, rows)
    entries = torch.from_numpy(np.concatenate([[rows], names]).astype(np.int32)).cuda()
    dweight, dbias = weight_gradient(grads, q, s, F32, entries)
    check_gradient(dweight, dbias, grads, q, s, names)
    wq, ws = levels(rng, A, H)
    check_linear(linear(q, s, wq, ws, None, F32, entries), q, s, wq, ws, None, F32, np.unique(names))


@pytest.mark.parametrize("count, want", [(-7, 0), (10 ** 9, 12)])
def test_a_count_out_of_range(count, want):
    """Below 0 it is 0, above `rows` it is `rows`."""
    rng = np.random.default_rng(13)
    rows, H, A = 12, 100, 30
    q, s = levels(rng, rows, H)
    wq, ws = levels(rng, A, H)
    entries = torch.from_numpy(np.concatenate([[count], np.arange(rows)]).astype(np.int32)).cuda()
    out = linear(q, s, wq, ws, None, F32, entries)
    check_linear(out, q, s, wq, ws, None, F32, np.arange(want))
    dweight, dbias = weight_gradient(gradients(rng, rows, A, F32), q, s, F32, entries)
    assert bool(dweight.t.any()) == bool(want)


def test_places_beyond_32_bits():
    """The last rows of tensors of more than 2^31 bytes and 2^31 elements."""
    rng = np.random.default_rng(14)
    rows, H, A = 1 << 24 | 77, 129, 130
    pitch = layer.row_pitch(H)
    assert rows * pitch > 2 ** 31 and rows * A > 2 ** 31
    names = [0, rows // 2, rows - 70, rows - 1]
    entries = torch.tensor([len(names)] + names, dtype=torch.int32)
    frames = torch.zeros(1 + rows, dtype=torch.int32, device="cuda")
    frames[:len(entries)] = entries.cuda()
    x = torch.empty((rows, H), dtype=torch.bfloat16, device="cuda")
    values = states(rng, len(names), H, BF16)
    x[names] = values.to(torch.bfloat16).cuda()
    q = torch.empty((rows, pitch), dtype=torch.int8, device="cuda")
    scales = torch.empty(rows, device="cuda")
    layer.quantize_rows(x.data_ptr(), frames.data_ptr(), rows, H, BF16, q.data_ptr(), scales.data_ptr(), stream())
    want_q, want_s = ref.to_levels(values)
    assert torch.equal(q[names][:, :H].cpu().double(), want_q)
    layer.dequantize_rows(q.data_ptr(), scales.data_ptr(), frames.data_ptr(), rows, H, BF16, x.data_ptr(), stream())
    assert torch.equal(x[names].cpu(), (q[names][:, :H].cpu().float() * scales[names].cpu()[:, None]).to(torch.bfloat16))
    del x
    wq, ws = levels(rng, A, H)
    gw, gws = ref.library_rows(wq, ws, H)
    logits = torch.empty((rows, A), dtype=torch.bfloat16, device="cuda")
    layer.linear_i8(q.data_ptr(), scales.data_ptr(), gw.t.data_ptr(), gws.t.data_ptr(), None, frames.data_ptr(), rows, H, A,
                    BF16, logits.data_ptr(), stream())
    got_q, got_s = q[names][:, :H].cpu(), scales[names].cpu()
    want = (got_q.double() * got_s.double()[:, None]) @ (wq.double() * ws.double()[:, None]).t()
    assert ((logits[names].cpu().double() - want).abs() <= 2.0 ** -8 * 1.001 * want.abs() + 1e-30).all()
    grads = gradients(rng, len(names), A, BF16)
    logits[names] = grads.to(torch.bfloat16).cuda()
    dweight, dbias = Guarded((A, H), torch.float32), Guarded((A,), torch.float32)
    size = layer.weight_gradient_workspace_size(rows, H, A)
    work = torch.empty(size + 256, dtype=torch.uint8, device="cuda")
    layer.weight_gradient_i8(logits.data_ptr(), q.data_ptr(), scales.data_ptr(), frames.data_ptr(), rows, H, A, BF16,
                             dweight.t.data_ptr(), dbias.t.data_ptr(), (work.data_ptr() + 255) // 256 * 256, size, stream())
    torch.cuda.synchronize()
    check_gradient(dweight, dbias, grads, got_q, got_s, np.arange(len(names)))


def test_more_rows_than_a_grid_has_in_a_line():
    """More than 2^26 rows, a wavefront each: 2^32 threads."""
    rows, H = (1 << 26) + 3, 2
    frames = torch.empty(1 + rows, dtype=torch.int32, device="cuda")
    lengths = torch.tensor([rows], dtype=torch.int32, device="cuda")
    layer.pack_frames(lengths.data_ptr(), rows, 1, frames.data_ptr(), stream())
    torch.cuda.synchronize()
    assert int(frames[0]) == rows and int(frames[1]) == 0 and int(frames[rows]) == rows - 1
    names = [0, (1 << 26) - 1, 1 << 26, rows - 1]
    frames[:5] = torch.tensor([4] + names, dtype=torch.int32, device="cuda")
    x = torch.empty((rows, H), dtype=torch.bfloat16, device="cuda")
    x[names] = torch.tensor([[1.0, -2.0], [3.0, 0.5], [0.0, 4.0], [-8.0, 8.0]], dtype=torch.bfloat16, device="cuda")
    want = x[names].clone()
    q, scales = torch.empty((rows, 128), dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")
    layer.quantize_rows(x.data_ptr(), frames.data_ptr(), rows, H, BF16, q.data_ptr(), scales.data_ptr(), stream())
    assert torch.equal(q[names][:, :H].cpu().double(), ref.to_levels(want.float().cpu())[0])
    x.zero_()
    layer.dequantize_rows(q.data_ptr(), scales.data_ptr(), frames.data_ptr(), rows, H, BF16, x.data_ptr(), stream())
    assert torch.equal(x[names].cpu(), (q[names][:, :H].cpu().float() * scales[names].cpu()[:, None]).to(torch.bfloat16))


# ---- how the calls may be used ----------------------------------------------------------------------------------

class Step:
    """A layer's forward and backward calls on buffers of its own."""

    def __init__(self, seed, T, B, H, A, dtype):
        self.T, self.B, self.H, self.A, self.dtype, self.rows = T, B, H, A, dtype, T * B
        self.rng = np.random.default_rng(seed)
        t, dev = torch_type(dtype), "cuda"
        rows, pitch = self.rows, layer.row_pitch(H)
        self.lengths = torch.zeros(B, dtype=torch.int32, device=dev)
        self.frames = torch.zeros(1 + rows, dtype=torch.int32, device=dev)
        self.x, self.residual, self.dy = (torch.zeros((rows, H), dtype=t, device=dev) for _ in range(3))
        self.w = torch.zeros((A, H), device=dev)
        self.norm_w = torch.zeros(H, device=dev)
        self.wq, self.ws = torch.zeros((A, pitch), dtype=torch.int8, device=dev), torch.zeros(A, device=dev)
        self.q, self.scales = torch.zeros((rows, pitch), dtype=torch.int8, device=dev), torch.zeros(rows, device=dev)
        self.total, self.dsum = torch.zeros_like(self.x), torch.zeros_like(self.x)
        self.logits, self.grads = torch.zeros((rows, A), dtype=t, device=dev), torch.zeros((rows, A), dtype=t, device=dev)
        self.dweight, self.dbias, self.dnorm = torch.zeros((A, H), device=dev), torch.zeros(A, device=dev), torch.zeros(H, device=dev)
        self.sizes = layer.weight_gradient_workspace_size(rows, H, A), layer.rms_norm_workspace_size(rows, H)
        self.work = [torch.empty(n + 256, dtype=torch.uint8, device=dev) for n in self.sizes]
        self.fill()

    def fill(self):
        r, n, H, A = self.rng, self.rows, self.H, self.A
        self.lengths.copy_(torch.from_numpy(r.integers(0, self.T + 1, self.B).astype(np.int32)))
        for buf, shape in ((self.x, (n, H)), (self.residual, (n, H)), (self.dy, (n, H)), (self.w, (A, H)), (self.norm_w, (H,)),
                           (self.grads, (n, A))):
            buf.copy_(torch.from_numpy(r.standard_normal(shape)).to(buf.dtype))

    def run(self, s):
        rows, H, A, d, f = self.rows, self.H, self.A, self.dtype, self.frames.data_ptr()
        at = [(w.data_ptr() + 255) // 256 * 256 for w in self.work]
        layer.pack_frames(self.lengths.data_ptr(), self.T, self.B, f, s)
        layer.quantize_rows(self.w.data_ptr(), None, A, H, F32, self.wq.data_ptr(), self.ws.data_ptr(), s)
        layer.rms_norm_i8(self.x.data_ptr(), self.residual.data_ptr(), self.norm_w.data_ptr(), 1e-6, f, rows, H, d,
                          self.total.data_ptr(), self.q.data_ptr(), self.scales.data_ptr(), s)
        layer.linear_i8(self.q.data_ptr(), self.scales.data_ptr(), self.wq.data_ptr(), self.ws.data_ptr(), None, f, rows, H, A,
                        d, self.logits.data_ptr(), s)
        layer.weight_gradient_i8(self.grads.data_ptr(), self.q.data_ptr(), self.scales.data_ptr(), f, rows, H, A, d,
                                 self.dweight.data_ptr(), self.dbias.data_ptr(), at[0], self.sizes[0], s)
        layer.rms_norm_backward(self.dy.data_ptr(), self.total.data_ptr(), self.norm_w.data_ptr(), 1e-6, None, f, rows, H, d,
                                self.dsum.data_ptr(), self.dnorm.data_ptr(), at[1], self.sizes[1], s)

    def results(self):
        torch.cuda.synchronize()
        return [t.clone() for t in (self.logits, self.dweight, self.dbias, self.dsum, self.dnorm, self.q, self.scales)]

    def clear(self):
        for t in (self.logits, self.dweight, self.dbias, self.dsum, self.dnorm, self.q, self.scales, self.total):
            t.zero_()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T, B, H, A", [(20, 7, 300, 29), (11, 30, 520, 300), (1, 5, 200, 700)])
def test_graphs_are_replayed_on_new_contents(T, B, H, A, dtype):
    step = Step(21, T, B, H, A, dtype)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step.run(side.cuda_stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step.run(torch.cuda.current_stream().cuda_stream)
    for _ in range(4):
        step.fill()
        step.clear()
        step.run(stream())
        want = step.results()
        step.clear()
        graph.replay()
        got = step.results()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert any(t.any() for t in got)


def test_a_graph_of_a_large_layer_between_eager_calls():
    step = Step(22, 12, 20, 1999, 5001, BF16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step.run(torch.cuda.current_stream().cuda_stream)
    for _ in range(3):
        step.fill()
        step.clear()                                     # (rows that this minibatch does not list stay as they were)
        step.run(stream())
        want = step.results()
        step.clear()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(step.results(), want))


def test_two_streams_at_once():
    """Two layers' steps on two streams, with workspaces of their own, as each alone; twice the same bits."""
    steps = [Step(31, 40, 30, 640, 29, BF16), Step(32, 16, 40, 384, 1000, F32)]
    want = []
    for s in steps:
        s.run(stream())
        want.append(s.results())
        s.clear()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for s, on in zip(steps, streams):
            s.run(on.cuda_stream)
    for s, w in zip(steps, want):
        assert all(torch.equal(a, b) for a, b in zip(s.results(), w))
