"""The gradients that the GPU tests compare with (block_reference), against differences of the forward definitions: in 64 bits, on the CPU."""
import numpy as np
import pytest
import torch

import block_reference as ref

STEP = 1e-5      # a central difference is off by a sixth of its square times the third derivative, and by 2^-53 of the value over it: 1e-10 and 1e-11


def differences(f, x):
    """d f / d x of a scalar function, by central differences."""
    out = torch.zeros_like(x)
    flat, grad = x.view(-1), out.view(-1)
    for i in range(flat.numel()):
        old = float(flat[i])
        flat[i] = old + STEP
        up = float(f())
        flat[i] = old - STEP
        down = float(f())
        flat[i] = old
        grad[i] = (up - down) / (2 * STEP)
    return out


def agree(got, want):
    assert torch.allclose(got, want, rtol=1e-6, atol=1e-7), float((got - want).abs().max())


@pytest.mark.parametrize("lengths, forward", [([4, 2, 0], 3), ([5, 5, 1], 0), ([3, 5, 4], 2)])
def test_recurrence(lengths, forward):
    T, B, H = 5, 3, 3
    gen = torch.Generator().manual_seed(1)
    gates, candidates, weigh = (torch.randn(T, B, H, generator=gen, dtype=torch.float64) for _ in range(3))
    initial, weigh_final = (torch.randn(B, H, generator=gen, dtype=torch.float64) for _ in range(2))
    valid = (torch.arange(T)[:, None] < torch.tensor(lengths)[None])[:, :, None]

    def value():
        states, final, _ = ref.recurrence(gates, candidates, initial, lengths, forward, True)
        return (torch.where(valid, states, 0.0) * weigh).sum() + (final * weigh_final).sum()

    states, _, _ = ref.recurrence(gates, candidates, initial, lengths, forward, True)
    dg, dc, d0, *_ = ref.recurrence_backward(weigh, weigh_final, gates, candidates, states, initial, lengths, forward, True)
    agree(dg, differences(value, gates))
    agree(dc, differences(value, candidates))
    agree(d0, differences(value, initial))


@pytest.mark.parametrize("gated", [True, False])
def test_block_norm(gated):
    rows, H, eps = 3, 5, 1e-2
    gen = torch.Generator().manual_seed(2)
    x, residual, weigh_y, weigh_z = (torch.randn(rows, H, generator=gen, dtype=torch.float64) for _ in range(4))
    gate = 2 * torch.randn(rows, H, generator=gen, dtype=torch.float64) if gated else None
    after, scale, before = (1 + 0.3 * torch.randn(H, generator=gen, dtype=torch.float64) for _ in range(3))

    def value():
        z, _ = ref.block_norm(x, gate, residual, after, scale, eps, True)
        y, _ = ref.normed(z, before, eps)
        return (y * weigh_y).sum() + (z * weigh_z).sum()

    z, _ = ref.block_norm(x, gate, residual, after, scale, eps, True)
    grads, _ = ref.block_norm_backward(weigh_y, weigh_z, x, gate, z, after, scale, before, eps, 1, True)
    for name, of in (("dx", x), ("dresidual", residual), ("dweight_after", after), ("dscale", scale), ("dweight_before", before)):
        agree(grads[name], differences(value, of))
    if gated:
        agree(grads["dgate"], differences(value, gate))


def test_whole_numbers_of_4_bits():
    """The definition by exact comparison, against rational arithmetic."""
    from fractions import Fraction
    rng = np.random.default_rng(1)
    w = rng.standard_normal((40, 64)).astype(np.float32)
    w[:10] = rng.integers(-14, 15, (10, 64)).astype(np.float32)
    w[:10, 0] = 14.0
    w[20] = np.float32(2.0 ** -140) * rng.integers(-9, 10, 64).astype(np.float32)
    w[21], w[22, 3] = 0.0, np.inf
    q, s = ref.to_i4(torch.from_numpy(w), 64)
    for a in range(40):
        if a == 22:
            assert not q[a].any() and torch.isnan(s[a]).all()
            continue
        m = max(abs(Fraction(float(v))) for v in w[a])
        for k in range(64):
            want = round(7 * Fraction(float(w[a, k])) / m) if m else 0          # (round: ties to even)
            assert int(q[a, k]) == want, (a, k)
        assert abs(float(s[a, 0]) - float(m) / 7) <= 1e-15 * float(m)


def test_packed_order():
    """The header's order of the packed weights, byte by byte."""
    A, H, group = 18, 130, 64
    data = np.zeros((2, 2, 1024), dtype=np.uint8)
    want = np.random.default_rng(2).integers(-7, 8, (A, H))
    for r in range(A):
        for c in range(H):
            i, high = c % 128 % 64, c % 128 >= 64
            at = 256 * (i // 16) + 16 * (r % 16) + i % 16
            data[r // 16, c // 128, at] |= (int(want[r, c]) & 15) << (4 if high else 0)
    scales = np.zeros((2, 3, 16), dtype=np.float32)
    for r in range(A):
        scales[r // 16, :, r % 16] = (r + 1, 100 + r, 200 + r)
    q, s = ref.unpack_i4(data.reshape(-1), scales.reshape(-1), A, H, group)
    assert np.array_equal(q, want) and np.array_equal(s, np.stack([np.arange(A) + 1, np.arange(A) + 100, np.arange(A) + 200], 1))
