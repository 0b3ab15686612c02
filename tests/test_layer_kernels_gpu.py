"""The output layer's kernels for many rows, each with and without a list of rows, in both types; which kernel a size takes is asked of the rule that
launches follow (tests/layer_rules.py)."""
import numpy as np
import pytest
import torch

import layer_reference as ref
import layer_rules as rules
import test_layer_gpu as base
from layer_reference import HALF, Guarded, frame_list, others, pointer, poisoned, put, stream, torch_type
from paper_1512_02595_amd import ctc, layer

pytestmark = pytest.mark.gpu
F32, BF16 = ctc.DTYPE_F32, ctc.DTYPE_BF16
TYPES = [F32, BF16]
LISTS = ["all", "some", "odd entries"]

# rows, H, (wavefronts to a row, elements to a lane)
MANY_ROWS = [(2050, 513, (1, 16)), (2100, 600, (1, 16)), (2049, 1000, (1, 16)), (2061, 1029, (2, 16)), (2100, 1999, (2, 16)), (2051, 2048, (2, 16)),
             (2050, 2049, (4, 16)), (2055, 3204, (4, 16)), (2049, 4096, (4, 16)), (2053, 4097, (8, 16)), (2050, 8193, (8, 32)), (2100, 129, (1, 8))]


@pytest.mark.parametrize("kind", [*LISTS, "none"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, H, shape", MANY_ROWS)
def test_many_rows_to_8_bits(rows, H, shape, dtype, kind):
    print("rows", rows, H, dtype, kind, flush=True)
    assert rules.row_shape(rows, H) == shape
    rng = np.random.default_rng(rows + H)
    t = torch_type(dtype)
    x, y = base.states(rng, rows, H, dtype), base.states(rng, rows, H, dtype)
    w = torch.from_numpy(1.0 + 0.5 * rng.standard_normal(H)).float()
    x[7], y[7] = 0.0, 0.0
    frames, names = frame_list(kind, rows, rng)
    dx, dr, dw = put(poisoned(x, names), t), put(poisoned(y, names), t), put(w, torch.float32)
    q, scales = Guarded((rows, layer.row_pitch(H)), torch.int8), Guarded((rows,), torch.float32)
    layer.quantize_rows(dx.t.data_ptr(), pointer(frames), rows, H, dtype, q.t.data_ptr(), scales.t.data_ptr(), stream())
    torch.cuda.synchronize()
    base.check_rows(q, scales, x[names], names, rows, H)
    total, q, scales = Guarded((rows, H), t), Guarded((rows, layer.row_pitch(H)), torch.int8), Guarded((rows,), torch.float32)
    eps = 1e-5
    layer.rms_norm_i8(dx.t.data_ptr(), dr.t.data_ptr(), dw.t.data_ptr(), eps, pointer(frames), rows, H, dtype, total.t.data_ptr(),
                      q.t.data_ptr(), scales.t.data_ptr(), stream())
    torch.cuda.synchronize()
    z = (x + y).to(t)[names]
    assert torch.equal(total.t.cpu()[names], z) and total.untouched(others(rows, names)) and total.intact()
    base.check_rows(q, scales, z.float() * w, names, rows, H, ref.rms(z.double(), float(np.float32(eps))))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, H, shape", [m for m in MANY_ROWS if m[1] in (1000, 1999, 3204)])
def test_many_rows_that_are_not_finite(rows, H, shape, dtype):
    """Each wavefront of a row in turn has the value that spoils it; its neighbours are as they were."""
    assert rules.row_shape(rows, H) == shape
    rng = np.random.default_rng(H)
    x = base.states(rng, rows, H, dtype)
    bad = np.arange(0, rows, 5)
    x[bad, (bad * 37) % H] = torch.from_numpy(np.array([np.nan, np.inf, -np.inf])[np.arange(len(bad)) % 3]).float()
    dx = put(x, torch_type(dtype))
    q, scales = Guarded((rows, layer.row_pitch(H)), torch.int8), Guarded((rows,), torch.float32)
    layer.quantize_rows(dx.t.data_ptr(), None, rows, H, dtype, q.t.data_ptr(), scales.t.data_ptr(), stream())
    torch.cuda.synchronize()
    base.check_rows(q, scales, x, np.arange(rows), rows, H)
    layer.rms_norm_i8(dx.t.data_ptr(), None, None, 1e-6, None, rows, H, dtype, None, q.t.data_ptr(), scales.t.data_ptr(), stream())
    torch.cuda.synchronize()
    base.check_rows(q, scales, x, np.arange(rows), rows, H, ref.rms(x.double(), float(np.float32(1e-6))))


# rows, H, A, (rows, symbols) of a tile
MANY_TILES = [(42000, 200, 29, (128, 64)), (42000, 130, 61, (128, 64)), (45001, 129, 64, (128, 64)), (11000, 300, 4200, (256, 256)),
              (9500, 513, 4733, (256, 256)), (16001, 200, 2900, (256, 256)), (6000, 128, 5700, (128, 128)), (5700, 300, 5801, (128, 128))]


@pytest.mark.parametrize("kind", LISTS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, H, A, tile", MANY_TILES)
def test_activations_of_many_rows(rows, H, A, tile, dtype, kind):
    print("activations", rows, H, A, dtype, kind, flush=True)
    assert rules.product_tile(rows, H, A, kind != "all") == tile
    rng = np.random.default_rng(rows + A)
    q, s = base.levels(rng, rows, H)
    wq, ws = base.levels(rng, A, H)
    bias = torch.from_numpy(rng.standard_normal(A)).float()
    frames, names = frame_list(kind, rows, rng)
    base.check_linear(base.linear(q, s, wq, ws, bias, dtype, frames), q, s, wq, ws, bias, dtype, names)


@pytest.mark.parametrize("dtype, shift", [(F32, 4), (BF16, 2)])
@pytest.mark.parametrize("rows, H, A", [(42000, 140, 29), (11000, 140, 4200), (6000, 140, 5700)])
def test_few_of_many_rows_off_alignment_and_not_finite(rows, H, A, dtype, shift):
    """Tiles that are sized for a list's five eighths, and a list of a few rows, one tile and a part of one."""
    rng = np.random.default_rng(A)
    q, s = base.levels(rng, rows, H)
    wq, ws = base.levels(rng, A, H)
    names = np.sort(rng.choice(rows, 300, replace=False))
    s[names[::50]], q[names[::50]] = float("nan"), 0
    entries = torch.zeros(1 + rows, dtype=torch.int32)
    entries[0], entries[1:301] = 300, torch.from_numpy(names)
    out = base.linear(q, s, wq, ws, None, dtype, entries.cuda(), shift=shift)
    got, fine = out.t.cpu(), np.delete(names, np.arange(0, 300, 50))
    assert torch.isnan(got[names[::50]]).all() and not torch.isnan(got[fine]).any()
    product = q[fine].double() @ wq.double().t() * s[fine].double()[:, None] * ws.double()[None, :]
    bound = HALF * 4.001 * product.abs() + 1e-40
    assert ((got[fine].double() - product).abs() <= bound + ref.half_step(dtype) * (product.abs() + bound)).all()
    assert out.untouched(others(rows, names)) and out.intact()


# rows, H, A, symbols of a tile
MANY_SLABS = [(27200, 300, 29, 32), (33000, 64, 5, 32), (16000, 512, 60, 64), (12000, 640, 172, 64), (9000, 700, 2001, 128), (40000, 512, 500, 128),
              (40001, 600, 500, 128)]
EACH = 6


@pytest.mark.parametrize("kind", LISTS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, H, A, symbols", MANY_SLABS)
def test_each_product_of_the_weights_gradient_among_many_rows(rows, H, A, symbols, dtype, kind):
    """A symbol has a gradient in few rows only: sums round a few times, whatever the number of rows, and what a product loses shows."""
    print("weights' gradient", rows, H, A, dtype, kind, flush=True)
    assert rules.gradient_tile(rows, H, A)[0] == symbols and rules.gradient_tile(rows, H, A)[1] > 3
    rng = np.random.default_rng(rows + A)
    q = torch.from_numpy(rng.integers(-127, 128, (rows, H)).astype(np.int8))
    s = torch.from_numpy(np.exp(rng.standard_normal(rows)) * 0.01).float()
    frames, names = frame_list(kind, rows, rng)
    where = rng.choice(names, (A, EACH))
    grads = torch.zeros((rows, A))
    grads[torch.from_numpy(where), torch.arange(A)[:, None]] = torch.from_numpy(rng.standard_normal((A, EACH)) * 10.0 ** rng.integers(-3, 4, (A, 1))).float()
    grads = grads.to(torch_type(dtype)).float()
    dweight, dbias = base.weight_gradient(grads, q, s, dtype, frames, names=names)
    where = np.sort(where, 1)
    once = np.concatenate([np.ones((A, 1), bool), where[:, 1:] != where[:, :-1]], 1)          # (a row drawn twice holds one gradient)
    g = torch.where(torch.from_numpy(once), grads[torch.from_numpy(where), torch.arange(A)[:, None]].double(), 0.0)
    rows_q = q[torch.from_numpy(where)].double()                                              # [A, EACH, H]
    c = g * s[torch.from_numpy(where)].double()
    want, terms = (c[:, :, None] * rows_q).sum(1), (c.abs()[:, :, None] * rows_q.abs()).sum(1)
    # A product of gradient and scale is rounded once and held to 2 half steps of it by its parts, of which there are at most three, each added with at most a
    # half step of what is added up.  Wide tiles: or to 2^-38 of the symbol's largest.
    bound = HALF * (1 + 2 + 3 * EACH) * 1.001 * terms
    if symbols == 128:
        bound = bound + 2.0 ** -38 * c.abs().amax(1)[:, None] * rows_q.abs().sum(1)
    assert ((dweight.t.cpu().double() - want).abs() <= bound).all()
    assert ((dbias.t.cpu().double() - g.sum(1)).abs() <= HALF * (EACH + 2) * g.abs().sum(1)).all()


@pytest.mark.parametrize("kind", LISTS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, H", [(9000, 500), (9001, 1024), (5000, 1100), (4500, 2048), (4200, 3204), (4100, 5000), (4100, 8200)])
def test_norm_gradients_of_many_rows(rows, H, dtype, kind):
    """Workgroups that take three rows and more, one after another, for each width's kernel."""
    print("norm's gradient", rows, H, dtype, kind, flush=True)
    rng = np.random.default_rng(rows + H)
    t = torch_type(dtype)
    z, dy, dres = (base.states(rng, rows, H, dtype) for _ in range(3))
    w = torch.from_numpy(1.0 + 0.5 * rng.standard_normal(H)).float()
    frames, names = frame_list(kind, rows, rng)
    out, dweight = base.backward(put(poisoned(dy, names), t), put(poisoned(z, names), t), put(w, torch.float32), put(poisoned(dres, names), t), dtype,
                                 rows, H, 1e-5, frames)
    base.check_backward(out, dweight, dy, z, w, dres, dtype, rows, H, 1e-5, names)
    assert out.untouched(others(rows, names)) and out.intact()


@pytest.mark.parametrize("top", [60, 0, -100, -110, -120, -126, -130])
@pytest.mark.parametrize("rows, H, A, symbols", [(3000, 120, 29, 32), (3000, 120, 60, 64), (12000, 640, 172, 64), (9000, 700, 2001, 128)])
def test_the_smallest_products_of_the_weights_gradient(rows, H, A, symbols, top):
    """Each element is one product; a symbol's are of sizes from 2^top down to 2^-25 of it, so down to and below what fp32 and bf16 hold."""
    print("smallest products", rows, H, A, top, flush=True)
    assert rules.gradient_tile(rows, H, A)[0] == symbols
    rng = np.random.default_rng(rows + A)
    q = torch.from_numpy(rng.integers(1, 128, (rows, H)) * rng.choice([-1, 1], (rows, H)))
    q = torch.where(torch.arange(H)[None, :] % EACH == torch.arange(rows)[:, None] % EACH, q, 0)
    where = torch.from_numpy(rng.integers(0, rows // EACH, (A, EACH)) * EACH + np.arange(EACH))
    c = torch.from_numpy((1 + rng.random((A, EACH))) * 2.0 ** (top - 5 * np.arange(EACH))[None, :] * rng.choice([-1, 1], (A, EACH))).float()
    grads = torch.zeros(rows, A)
    grads[where, torch.arange(A)[:, None]] = c
    dweight, _ = base.weight_gradient(grads, q, torch.ones(rows), F32)
    column = torch.arange(H) % EACH
    size = c.double()[:, column]
    levels = q[where].double().sum(1)                    # (the one row of a symbol's that is not 0 there)
    # two half steps by the parts, at most three of which are added; bf16 ends at 2^-133, and the parts of wide tiles at 2^-38 of the largest; the result
    # is an fp32 number, of which there are none between multiples of 2^-149
    least = torch.full((A, 1), 2.0 ** -133, dtype=torch.float64) if symbols < 128 else 2.0 ** -38 * c.double().abs().amax(1, keepdim=True)
    bound = levels.abs() * (HALF * (2 + 3) * 1.001 * size.abs() + least) + 2.0 ** -149
    assert ((dweight.t.cpu().double() - size * levels).abs() <= bound).all()
