"""The norms around a block and their gradient against their definitions in 64 bits: widths, lists of rows, both types, pitches, and
every buffer that may be absent or be another."""
import numpy as np
import pytest
import torch

import block_reference as ref
from layer_reference import Guarded, HALF, frame_list, half_step, others, pointer, poisoned, put, stream, torch_type
from paper_1512_02595_amd import block, ctc

pytestmark = pytest.mark.gpu
F32, BF16 = ctc.DTYPE_F32, ctc.DTYPE_BF16
TYPES = [F32, BF16]
LISTS = ["all", "some", "none", "odd entries"]
WIDTHS = [1, 3, 64, 100, 511, 513, 1000, 1025, 1999, 2048, 2049, 4096, 4100, 8193, 9000, 16384]
EPS = 1e-5


def say(*a):
    print(*a, flush=True)


class Call:
    def __init__(self, rows, H, dtype, kind="all", pitch=None, seed=0, gate=True, residual=True, weights=True):
        rng = np.random.default_rng([rows, H, dtype, seed])
        self.rows, self.H, self.dtype, self.tt, self.pitch = rows, H, dtype, torch_type(dtype), pitch or H

        def held(scale=1.0):
            x = rng.standard_normal((rows, H)) * scale
            x[rng.random((rows, H)) < 0.03] = 0.0
            return torch.from_numpy(x).float().to(self.tt).float()

        self.frames, self.names = frame_list(kind, rows, rng)
        sizes = np.exp(rng.standard_normal((rows, 1)) * 2)
        self.x, self.z, self.dy, self.dz = held(sizes), held(sizes), held(), held()
        self.residual = held(sizes) if residual else None
        self.gate = held(3.0) if gate else None
        self.w = [torch.from_numpy(rng.standard_normal(H)).float() if weights else None for _ in range(3)]
        self.ones = [torch.ones(H) if w is None else w for w in self.w]
        self.w_dev = [None if w is None else put(w, torch.float32) for w in self.w]

    def dev(self, x):
        return None if x is None else put(poisoned(x, self.names), self.tt)

    def gate_dev(self):
        if self.gate is None:
            return None
        g = torch.full((self.rows, self.pitch), float("nan"))
        g[:, :self.H] = poisoned(self.gate, self.names)
        return put(g, self.tt)

    def listed(self, x):
        return None if x is None else x[self.names]


def at(g):
    return None if g is None else g.t.data_ptr()


# Below 2^-126 a type's step no longer shrinks with the value: 2^-133 in bf16, of which a stored result may be off by half; in fp32 2^-149, of which each operation
# may be off by half, and its result may yet be multiplied by a norm's factor, 1 / sqrt(EPS) < 2^9, and by weights below 2^3: a few times 2^-138.
SMALLEST = {F32: 2.0 ** -136, BF16: 2.0 ** -134 + 2.0 ** -136}


def within(what, got, want, bound, dtype):
    tolerance = bound + (HALF + half_step(dtype)) * (want.abs() + bound) + SMALLEST[dtype]
    off = (got.double() - want).abs() / tolerance
    worst = float(off.max()) if off.numel() else 0.0
    say("   %s %.3f of what is allowed" % (what, worst))
    assert worst <= 1


def forward(c, sum_at=None, normed_at=None, want_sum=True, want_normed=True):
    x, gate, residual = c.dev(c.x), c.gate_dev(), c.dev(c.residual)
    places = {"x": x, "residual": residual}
    total = places[sum_at] if sum_at else Guarded((c.rows, c.H), c.tt) if want_sum else None
    out = places[normed_at] if normed_at else Guarded((c.rows, c.H), c.tt) if want_normed else None
    block.block_norm(at(x), at(gate), c.pitch, at(residual), *map(at, c.w_dev), EPS, pointer(c.frames), c.rows, c.H, c.dtype, at(total), at(out), stream())
    torch.cuda.synchronize()
    eps = float(np.float32(EPS))
    want, bound = ref.block_norm(c.listed(c.x), c.listed(c.gate), c.listed(c.residual), c.ones[0], c.ones[1], eps, c.dtype == F32)
    rest = others(c.rows, c.names)
    z = None
    if total:
        z = total.t.cpu()[c.names]
        within("sum", z, want, bound, c.dtype)
        assert total.intact() and (sum_at or total.untouched(rest))
    if out:
        if z is None:
            z, slip = want, bound + half_step(c.dtype) * (want.abs() + bound)
            scale = c.ones[2].double().abs() / torch.sqrt((want * want).mean(1, keepdim=True) + eps)
            slip = scale * (slip + want.abs() * slip.max(1, keepdim=True).values / torch.sqrt((want * want).mean(1, keepdim=True) + eps))
        else:
            slip = 0.0
        y, b = ref.normed(z, c.ones[2], eps)
        within("normed", out.t.cpu()[c.names], y, b + slip, c.dtype)
        assert out.intact() and (normed_at or out.untouched(rest))


@pytest.mark.parametrize("kind", LISTS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H", WIDTHS)
def test_forward(H, dtype, kind):
    say("block norm", H, dtype, kind)
    forward(Call(37, H, dtype, kind, H + (H % 3)))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, H", [(1, 2048), (1, 100), (5000, 64), (3000, 300), (2500, 1100), (600, 5000)])
def test_forward_rows(rows, H, dtype):
    say("block norm", rows, H, dtype)
    forward(Call(rows, H, dtype, "all" if rows == 1 else "some", 3 * H))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H", [64, 700, 1999, 5001, 9001])
def test_forward_absent_and_shared_buffers(H, dtype):
    for kind in LISTS:
        for gate, residual, weights in ((False, True, True), (True, False, True), (True, True, False), (False, False, False)):
            say("block norm", H, dtype, kind, gate, residual, weights)
            forward(Call(37, H, dtype, kind, H, 1, gate, residual, weights))
        c = Call(41, H, dtype, kind, 2 * H, 2)
        forward(c, want_sum=False)
        forward(c, want_normed=False)
        for places in ((None, "x"), ("x", None), ("residual", None), (None, "residual"), ("x", "residual"), ("residual", "x")):
            say("   in place", places)
            forward(c, *places)


def backward(c, dx_at=None, dres_at=None, use_dy=True, use_dz=True, sums=(True, True, True), dresidual=True):
    x, gate = c.dev(c.x), c.gate_dev()
    dy, dz, z = c.dev(c.dy) if use_dy else None, c.dev(c.dz) if use_dz else None, c.dev(c.z) if use_dy else None
    places = {"x": x, "sum": z, "dnormed": dy, "dsum": dz}
    dx = places[dx_at] if dx_at else Guarded((c.rows, c.H), c.tt)
    dres = places[dres_at] if dres_at else Guarded((c.rows, c.H), c.tt) if dresidual else None
    dgate = None if gate is None else Guarded((c.rows, c.pitch), c.tt)
    dw = [Guarded((c.H,), torch.float32) if s else None for s in sums]
    size = block.block_norm_workspace_size(c.rows, c.H)
    ws = Guarded((size + 256,), torch.uint8)
    ws.t.fill_(0xFF)
    block.block_norm_backward(at(dy), at(dz), at(x), at(gate), c.pitch, at(z), *map(at, c.w_dev), EPS, pointer(c.frames), c.rows, c.H, c.dtype,
                              at(dx), at(dgate), at(dres), *map(at, dw), (ws.t.data_ptr() + 255) // 256 * 256 if any(sums) else None, size, stream())
    torch.cuda.synchronize()
    # (the partial sums: at least 256 workgroups share more rows than that; a workgroup of 32 teams takes 32 rows at once)
    per_group = -(-c.rows // 256) + 40
    want, bound = ref.block_norm_backward(c.listed(c.dy) if use_dy else None, c.listed(c.dz) if use_dz else None, c.listed(c.x), c.listed(c.gate),
                                          c.listed(c.z) if use_dy else None, *c.ones, float(np.float32(EPS)), per_group, c.dtype == F32)
    rest, H = others(c.rows, c.names), c.H
    outs = [("dx", dx, dx_at), ("dresidual", dres, dres_at), ("dgate", dgate, None)]
    for name, g, place in outs:
        if g is None:
            continue
        within(name, g.t.cpu()[c.names][:, :H], want[name], bound[name], c.dtype)
        assert g.intact() and (place or g.untouched(rest)), name
    if dgate is not None and c.pitch > H:
        assert bool((dgate.raw[dgate.span[0]:dgate.span[1]].view(c.rows, c.pitch, -1)[:, H:] == 0x5A).all())
    for name, g in zip(("dweight_after", "dscale", "dweight_before"), dw):
        if g is not None:
            within(name, g.t.cpu(), want[name], bound[name], F32)
            assert g.intact()
    assert ws.intact()


@pytest.mark.parametrize("kind", LISTS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H", WIDTHS)
def test_backward(H, dtype, kind):
    say("block norm back", H, dtype, kind)
    backward(Call(37, H, dtype, kind, H + (H % 3)))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, H", [(1, 2048), (1, 100), (5000, 64), (3000, 300), (2500, 1100), (600, 5000)])
def test_backward_rows(rows, H, dtype):
    say("block norm back", rows, H, dtype)
    backward(Call(rows, H, dtype, "all" if rows == 1 else "some", 3 * H))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H", [64, 700, 1999, 5001, 9001])
def test_backward_absent_and_shared_buffers(H, dtype):
    for kind in LISTS:
        for gate, weights in ((False, True), (True, False), (False, False)):
            say("block norm back", H, dtype, kind, gate, weights)
            backward(Call(37, H, dtype, kind, H, 1, gate, True, weights))
        c = Call(41, H, dtype, kind, 2 * H, 2)
        backward(c, use_dy=False)
        backward(c, use_dz=False)
        backward(c, sums=(False, False, False), dresidual=False)
        for sums in ((True, False, False), (False, True, False), (False, False, True)):
            backward(c, sums=sums)
        for places in (("x", "dsum"), ("dsum", "x"), ("dnormed", "sum"), ("sum", "dnormed"), (None, "dsum"), ("x", None)):
            say("   in place", places)
            backward(c, *places)
