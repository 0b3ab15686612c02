"""The recurrent block's operators in 64 bits, on the CPU, each with a bound on what fp32 arithmetic may add to it.

A bound follows the formula: every quantity comes with the sum of the magnitudes of the terms that it is made of, and each
rounding on the way, or an exponential or a reciprocal good to a few units of its last place, adds its share of that.
"""
import numpy as np
import torch

from layer_reference import HALF

# z, 1 - z and their product: an exponential good to a unit in the last place (two half steps) and a half for each of two operations that correct
# it, a sum, a reciprocal good to a unit, a product, and the exponent's second part (1.5 half steps at most).
# Where results are in 16 bits the exponent's second part is left out: the product's rounding is an error of |g| half steps.
GATE = 9 * HALF


def gate_error(g, fine):
    return GATE + (0.0 if fine else HALF) * g.double().abs()


def sigmoid(g):
    """z and 1 - z, without a difference."""
    t = torch.exp(-g.abs())
    large, small = 1.0 / (1.0 + t), t / (1.0 + t)
    return torch.where(g >= 0, large, small), torch.where(g >= 0, small, large)


def turned(x, lengths, forward):
    """Channels >= forward with each utterance's frames from the last to the first (and back again)."""
    out = x.clone()
    for b, n in enumerate(lengths):
        out[:n, b, forward:] = x[:n, b, forward:].flip(0)
    return out


def recurrence(gates, candidates, initial, lengths, forward, fine):
    """(states [T, B, H], final [B, H], bound on either's error but for the rounding that stores it)."""
    T, B, H = gates.shape
    slack = gate_error(gates, fine).amax(0)
    z, _ = sigmoid(turned(gates.double(), lengths, forward))
    c = turned(candidates.double(), lengths, forward)
    h = torch.zeros(B, H, dtype=torch.float64) if initial is None else initial.double()
    # |dh| <= sum_s |dz_s| |c_s - h_(s-1)| prod (1 - z) <= slack max |c - h| (slack: the largest gate's): the weights z_s prod (1 - z) are at most 1 in sum
    most = h.abs()
    for b, n in enumerate(lengths):
        if n:
            most[b] = torch.maximum(most[b], c[:n, b].abs().amax(0))
    states, final, n = torch.zeros(T, B, H, dtype=torch.float64), h.clone(), torch.as_tensor(lengths)
    for s in range(T):
        there = (s < n)[:, None]
        h = torch.where(there, h + z[s] * (c[s] - h), h)
        states[s] = h
    final = h
    # (2^-50: what thousands of steps in fp64 add)
    return turned(states, lengths, forward), final, (2 * slack + 2.0 ** -40) * most


def recurrence_backward(dstates, dfinal, gates, candidates, states, initial, lengths, forward, fine):
    """(dgates, dcandidates, dinitial), and a bound on the error of each but for the rounding that stores it."""
    T, B, H = gates.shape
    slack = gate_error(gates, fine).amax(0)
    z, stays = sigmoid(turned(gates.double(), lengths, forward))
    c, h, dh = (turned(t.double(), lengths, forward) for t in (candidates, states, dstates))
    begin = torch.zeros(B, H, dtype=torch.float64) if initial is None else initial.double()
    d = torch.zeros(B, H, dtype=torch.float64) if dfinal is None else dfinal.double()
    n = torch.as_tensor(lengths)
    dg, dc, whole = (torch.zeros(T, B, H, dtype=torch.float64) for _ in range(3))
    most = d.abs()
    for s in range(T - 1, -1, -1):
        there = (s < n)[:, None]
        D = dh[s] + d
        before = h[s - 1] if s else begin
        dg[s], dc[s] = (torch.where(there, v, 0.0) for v in (D * (c[s] - before) * z[s] * stays[s], D * z[s]))
        whole[s] = torch.where(there, D.abs(), 0.0)
        most = torch.where(there, torch.maximum(most, D.abs()), most)
        d = torch.where(there, D * stays[s], d)
    # |dD| <= sum_s |dz_s| |D_s| prod (1 - z) <= slack max |D|, then D and the factors are rounded
    slip = slack * most + 2.0 ** -40 * most
    before = torch.cat((begin[None], h[:-1]))
    bound_c = z * (slip + (slack + 2 * HALF) * whole)
    bound_g = (c - before).abs() * z * stays * (slip + (2 * slack + 6 * HALF) * whole)
    bound_d = slip + slack * most
    return tuple(turned(t, lengths, forward) for t in (dg, dc)) + (d,) + tuple(turned(t, lengths, forward) for t in (bound_g, bound_c)) + (bound_d,)


def silu(p):
    z, stays = sigmoid(p)
    return p * z, z + p * z * stays, z + (p * z * stays).abs()


def block_norm(x, gate, residual, after, scale, eps, fine):
    """(z before it is rounded, bound)."""
    x = x.double()
    r = 1.0 / torch.sqrt((x * x).mean(1, keepdim=True) + eps)
    a = torch.ones_like(x) if gate is None else silu(gate.double())[0]
    term = x * r * after.double() * scale.double() * a
    res = torch.zeros_like(x) if residual is None else residual.double()
    z = term + res
    error = 0.0 if gate is None else gate_error(gate, fine)
    return z, (error + 8 * HALF) * term.abs() + HALF * z.abs()


def normed(z, before, eps):
    """(y of the stored z, bound)."""
    z = z.double()
    y = z / torch.sqrt((z * z).mean(1, keepdim=True) + eps) * before.double()
    return y, 4 * HALF * y.abs()


def block_norm_backward(dnormed, dsum, x, gate, z, after, scale, before, eps, per_group, fine):
    """dict of gradients, and one of bounds.  `per_group`: how many rows' shares are added up in fp32."""
    zero = torch.zeros_like(x, dtype=torch.float64)
    x = x.double()
    dy, dz, z = (zero if t is None else t.double() for t in (dnormed, dsum, z))
    after, scale, before = after.double(), scale.double(), before.double()
    v1, v2 = (x * x).mean(1, keepdim=True) + eps, (z * z).mean(1, keepdim=True) + eps
    f1, f2 = v1 ** -0.5, v2 ** -0.5
    c2, c2_abs = (dy * before * z).mean(1, keepdim=True) / v2, (dy * before * z).abs().mean(1, keepdim=True) / v2
    d = (dy * before - z * c2) * f2 + dz
    d_abs = ((dy * before).abs() + z.abs() * c2_abs) * f2 + dz.abs()
    if gate is None:
        a, slope, slope_abs = torch.ones_like(x), zero, zero
    else:
        a, slope, slope_abs = silu(gate.double())
    e, e_abs = d * a * after * scale, d_abs * (a * after * scale).abs()
    c1, c1_abs = (e * x).mean(1, keepdim=True) / v1, (e_abs * x.abs()).mean(1, keepdim=True) / v1
    factor = after * scale * x * f1
    out = {"dresidual": d, "dx": (e - x * c1) * f1, "dgate": d * factor * slope}
    error = 0.0 if gate is None else gate_error(gate, fine)
    D, E = 8 * HALF, error + 12 * HALF
    bound = {"dresidual": D * d_abs, "dx": (E + 6 * HALF) * e_abs * f1 + x.abs() * f1 * (((E + 6 * HALF) * e_abs * x.abs()).mean(1, keepdim=True) / v1 + 6 * HALF * c1_abs),
             "dgate": (D + 2 * error + 8 * HALF) * d_abs * factor.abs() * slope_abs}
    q, q_abs = d * a * x * f1, d_abs * (a * x * f1).abs()
    w = dy * z * f2
    sums = per_group * HALF
    out.update(dweight_after=(q * scale).sum(0), dscale=(q * after).sum(0), dweight_before=w.sum(0))
    bound.update(dweight_after=((E + 4 * HALF + sums) * q_abs * scale.abs()).sum(0), dscale=((E + 4 * HALF + sums) * q_abs * after.abs()).sum(0),
                 dweight_before=(5 * HALF + sums) * w.abs().sum(0))
    return out, bound


def to_i4(w, group):
    """(whole numbers [A, H] as float64, scales [A, groups] as float64, not yet rounded), by the definition."""
    A, H = w.shape
    parts = torch.nn.functional.pad(w.double(), (0, -H % group)).view(A, -1, group)
    m = parts.abs().amax(2, keepdim=True)
    fine = torch.isfinite(m)
    a, top = torch.where(fine, parts.abs(), 0.0), torch.where(fine & (m > 0), m, 1.0)
    j = torch.floor(7.0 * a / top)
    for step in (1.0, -1.0):                             # (the quotient may have been rounded over a whole number)
        j = torch.where(step * (7.0 * a - (j + (step > 0)) * top) >= (0.0 if step > 0 else 1e-320), j + step, j)
    twice, middle = 14.0 * a, (2.0 * j + 1.0) * top      # both exact: 24 bits and four more
    q = torch.where((twice > middle) | ((twice == middle) & (j % 2 == 1)), j + 1.0, j)
    q = torch.where(fine & (m > 0), q * torch.sign(parts), 0.0)
    return q.view(A, -1)[:, :H], torch.where(fine, m / 7.0, float("nan")).view(A, -1)


def unpack_i4(weight_q, weight_scales, A, H, group):
    """Whole numbers and scales out of the library's buffers (numpy), as the header lays them out; padding must be zeros."""
    across, tall = (H + 127) // 128, (A + 15) // 16
    tiles = weight_q.reshape(tall, across, 4, 16, 16)                            # [rows / 16, columns / 128, i / 16, r, i % 16]
    data = tiles.transpose(0, 3, 1, 2, 4).reshape(16 * tall, across, 64)
    low, high = (data.astype(np.int8) << 4) >> 4, data.astype(np.int8) >> 4
    q = np.concatenate([low, high], 2).reshape(16 * tall, across * 128)
    assert not q[A:].any() and not q[:, H:].any()
    groups = (H + group - 1) // group
    scales = weight_scales.reshape(tall, groups, 16).transpose(0, 2, 1).reshape(16 * tall, groups)
    assert not scales[A:].any()
    return q[:A, :H], scales[:A]
