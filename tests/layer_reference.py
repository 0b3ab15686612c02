"""The output layer's operators in 64 bits, on the CPU, and the buffers that their GPU tests call the library with.

Every buffer lies between two guard bands; rows that a call's list does not name hold NaN in its inputs and a pattern
in its outputs, so that a read or a write of one shows.
"""
import numpy as np
import torch

from paper_1512_02595_amd import ctc, layer

HALF = 2.0 ** -24                                       # half a step of fp32, relative
GUARD = 256
PATTERN = 0x5A


def torch_type(dtype):
    return torch.float32 if dtype == ctc.DTYPE_F32 else torch.bfloat16


def half_step(dtype):
    """What storing a result as `dtype` may add, relative to the result, beyond fp32's own rounding."""
    return 0.0 if dtype == ctc.DTYPE_F32 else 2.0 ** -8


class Guarded:
    """A tensor in the middle of a longer buffer; `intact` looks at what surrounds it."""

    def __init__(self, shape, dtype, shift=0):
        n = int(np.prod(shape)) * torch.empty(0, dtype=dtype).element_size()
        self.raw = torch.full((GUARD + n + GUARD + 64,), PATTERN, dtype=torch.uint8, device="cuda")
        start = GUARD + shift
        self.span = (start, start + n)
        self.t = self.raw[start:start + n].view(dtype).view(shape)

    def intact(self):
        a, b = self.span
        return bool((self.raw[:a] == PATTERN).all()) and bool((self.raw[b:] == PATTERN).all())

    def untouched(self, rows):
        """Whether the given rows (a truth value each) still hold the pattern."""
        a, b = self.span
        data = self.raw[a:b].view(self.t.shape[0], -1)
        return bool((data[rows] == PATTERN).all())


def put(values, dtype, shift=0):
    """float values on the GPU, guarded; `shift` in bytes moves the tensor off its alignment."""
    g = Guarded(values.shape, dtype, shift)
    g.t.copy_(values.to(dtype))
    return g


def frame_list(kind, rows, rng):
    """(the list as the library takes it, or None; the rows it names, in order, as a numpy array)."""
    if kind == "all":
        return None, np.arange(rows)
    names = rng.permutation(rows)
    if kind == "some":
        names = names[:max(1, (2 * rows) // 3)]
    if kind == "none":
        names = names[:0]
    entries = names.copy()
    if kind == "odd entries":                            # entries that are no row are skipped
        entries = np.concatenate([[-1], names[: rows // 2], [rows, 2 ** 31 - 1, -2 ** 31], names[rows // 2:rows - 4]])[:rows]
        names = np.array([e for e in entries if 0 <= e < rows], dtype=np.int64)
    out = np.zeros(1 + rows, dtype=np.int32)
    out[0] = len(entries)
    out[1:1 + len(entries)] = entries
    return torch.from_numpy(out).cuda(), names


def poisoned(values, names):
    """The same values with NaN in every row that is not named."""
    out = torch.full_like(values, float("nan"))
    out[torch.as_tensor(names, dtype=torch.long)] = values[torch.as_tensor(names, dtype=torch.long)]
    return out


def others(rows, names):
    keep = torch.ones(rows, dtype=torch.bool)
    keep[torch.as_tensor(names, dtype=torch.long)] = False
    return keep.cuda()


def pointer(t):
    return None if t is None else t.data_ptr()


def stream():
    return torch.cuda.current_stream().cuda_stream


def to_levels(u):
    """Rows of fp32 values as whole numbers and scales: (float64 [rows, H], float64 [rows]).  Exact in integers."""
    u = u.double().numpy()
    q = np.zeros_like(u)
    scales = np.zeros(u.shape[0])
    for r in range(u.shape[0]):
        row = u[r]
        if not np.isfinite(row).all():
            scales[r] = np.nan
            continue
        m = np.abs(row).max() if row.size else 0.0
        if m == 0.0:
            continue
        scales[r] = m / 127.0
        # (127 u and the quotient's rounding: the exact quotient is never nearer to a middle than 2^-33 of it unless it is one)
        q[r] = np.rint(127.0 * row / m)
    return torch.from_numpy(q), torch.from_numpy(scales)


def rms(z, eps):
    return 1.0 / torch.sqrt((z * z).mean(1) + eps)


def norm_backward(dy, z, w, eps, dres):
    """(dz, dweight, and what bounds the roundings of each) in float64."""
    H = z.shape[1]
    v = (z * z).mean(1, keepdim=True) + eps
    r = v.rsqrt()
    g = dy * w
    along = (g * z).mean(1, keepdim=True)
    dz = r * g - z * along * r / v
    size = (g * z).abs().mean(1, keepdim=True) * r / v * z.abs()
    bound = HALF * (5 * (r * g).abs() + 5 * size + 2 * dz.abs())
    if dres is not None:
        dz = dz + dres
        bound = bound + HALF * 2 * dres.abs()
    terms = dy * z * r
    return dz, terms.sum(0), bound, terms.abs().sum(0)


def library_rows(q, scales, H):
    """Rows in 8 bits as the library takes them, from whole numbers [rows, H] and scales."""
    rows = q.shape[0]
    g = Guarded((rows, layer.row_pitch(H)), torch.int8)
    g.t.zero_()
    g.t[:, :H] = q.to(torch.int8).cuda()
    return g, put(scales.float(), torch.float32)
