"""The gated linear recurrence and its gradient against their definitions in 64 bits: lengths from none to many, odd sizes, pitches,
both directions and types, states carried from call to call, and what may be done with the calls (graphs, buffers given twice)."""
import numpy as np
import pytest
import torch

import block_reference as ref
from layer_reference import Guarded, half_step, pointer, put, stream, torch_type, HALF
from paper_1512_02595_amd import block, ctc

pytestmark = pytest.mark.gpu
F32, BF16 = ctc.DTYPE_F32, ctc.DTYPE_BF16
TYPES = [F32, BF16]


def say(*a):
    print(*a, flush=True)


def lengths_of(kind, T, B, rng):
    if kind == "all":
        return None, [T] * B
    n = rng.integers(0, T + 1, B).astype(np.int32)
    n[rng.random(B) < 0.15] = 0
    if kind == "none":
        n[:] = 0
    elif B > 3:
        n[0], n[1], n[2] = T, -5, T + 7
    return torch.from_numpy(n).cuda(), [min(max(int(v), 0), T) for v in n]


class Call:
    """Inputs of a case on the host, held exactly by the type, and the library's buffers: rows behind an utterance's end and the columns
    between a row's and the next hold NaN in the inputs and a pattern in the outputs."""

    def __init__(self, T, B, H, dtype, kind="some", pitch=None, forward=None, carried=True, slow=False, shift=0, seed=0):
        rng = np.random.default_rng([T, B, H, dtype, seed])
        tt = torch_type(dtype)
        self.T, self.B, self.H, self.dtype, self.tt = T, B, H, dtype, tt
        self.pitch = pitch or 2 * H
        self.forward = H if forward is None else forward
        self.lengths, self.n = lengths_of(kind, T, B, rng)
        mean = rng.uniform(-12 if slow else -6, 1, (1, 1, H))

        def held(x):
            return torch.from_numpy(np.asarray(x)).float().to(tt).float()

        self.gates = held(rng.standard_normal((T, B, H)) * 2 + mean)
        self.candidates, self.states_in, self.dstates = (held(rng.standard_normal((T, B, H))) for _ in range(3))
        self.initial = torch.from_numpy(rng.standard_normal((B, H))).float() if carried else None
        self.dfinal = torch.from_numpy(rng.standard_normal((B, H))).float() if carried else None
        self.counts = torch.arange(T)[:, None] < torch.tensor(self.n)[None, :]
        full = torch.full((T, B, self.pitch), float("nan"))
        full[:, :, :H], full[:, :, H:2 * H] = self.gates, self.candidates
        full[~self.counts] = float("nan")
        self.inputs = put(full, tt, shift)
        self.ws_bytes = block.recurrence_workspace_size(T, B, H)
        self.ws = Guarded((self.ws_bytes + 256,), torch.uint8)
        self.ws.t.fill_(0xFF)
        self.ws_at = (self.ws.t.data_ptr() + 255) // 256 * 256

    def on_gpu(self, x, shift=0):
        x = x.clone()
        x[~self.counts] = float("nan")
        return put(x, self.tt, shift)

    def forward_call(self, initial=None, final=None, states=None):
        self.initial_dev = None if self.initial is None else put(self.initial, torch.float32)
        self.states = states or Guarded((self.T, self.B, self.H), self.tt)
        self.final = final or Guarded((self.B, self.H), torch.float32)
        block.recurrence(self.inputs.t.data_ptr(), self.pitch, pointer(self.lengths), None if self.initial is None else self.initial_dev.t.data_ptr(),
                         self.T, self.B, self.H, self.forward, self.dtype, self.states.t.data_ptr(), self.final.t.data_ptr(), self.ws_at,
                         self.ws_bytes, stream())

    def check_forward(self):
        torch.cuda.synchronize()
        want, final, bound = ref.recurrence(self.gates, self.candidates, self.initial, self.n, self.forward, self.dtype == F32)
        got = self.states.t.cpu().double()
        tolerance = bound[None] + (HALF + half_step(self.dtype)) * (want.abs() + bound[None])
        off = ((got - want).abs() / tolerance)[self.counts]
        worst = float(off.max()) if off.numel() else 0.0
        last = float(((self.final.t.cpu().double() - final).abs() / (bound + HALF * (final.abs() + bound) + 1e-300)).max())
        say("   states %.3f, final %.3f of what is allowed" % (worst, last))
        assert worst <= 1 and last <= 1
        behind = (~self.counts).flatten().cuda()
        data = self.states.raw[self.states.span[0]:self.states.span[1]].view(self.T * self.B, -1)
        assert bool((data[behind] == 0x5A).all())
        assert self.states.intact() and self.final.intact() and self.inputs.intact() and self.ws.intact()

    def backward_call(self, dinitial=None):
        self.d = [self.on_gpu(self.dstates), None if self.dfinal is None else put(self.dfinal, torch.float32), self.on_gpu(self.states_in)]
        self.initial_dev = None if self.initial is None else put(self.initial, torch.float32)
        self.dinputs = Guarded((self.T, self.B, self.pitch), self.tt)
        self.dinitial = dinitial or Guarded((self.B, self.H), torch.float32)
        block.recurrence_backward(self.d[0].t.data_ptr(), None if self.dfinal is None else self.d[1].t.data_ptr(), self.inputs.t.data_ptr(), self.pitch,
                                  self.d[2].t.data_ptr(), pointer(self.lengths), None if self.initial is None else self.initial_dev.t.data_ptr(),
                                  self.T, self.B, self.H, self.forward, self.dtype, self.dinputs.t.data_ptr(), self.dinitial.t.data_ptr(),
                                  self.ws_at, self.ws_bytes, stream())

    def check_backward(self):
        torch.cuda.synchronize()
        dg, dc, d0, bg, bc, b0 = ref.recurrence_backward(self.dstates, self.dfinal, self.gates, self.candidates, self.states_in, self.initial,
                                                         self.n, self.forward, self.dtype == F32)
        H, got = self.H, self.dinputs.t.cpu().double()
        for name, here, want, bound in (("dgates", got[:, :, :H], dg, bg), ("dcandidates", got[:, :, H:2 * H], dc, bc)):
            tolerance = bound + (HALF + half_step(self.dtype)) * (want.abs() + bound) + 2.0 ** -140
            off = ((here - want).abs() / tolerance)[self.counts]
            worst = float(off.max()) if off.numel() else 0.0
            say("   %s %.3f of what is allowed" % (name, worst))
            assert worst <= 1
        last = float(((self.dinitial.t.cpu().double() - d0).abs() / (b0 + HALF * (d0.abs() + b0) + 1e-300)).max())
        say("   dinitial %.3f" % last)
        assert last <= 1
        data = self.dinputs.raw[self.dinputs.span[0]:self.dinputs.span[1]].view(self.T * self.B, self.pitch, -1)
        assert bool((data[(~self.counts).flatten().cuda()] == 0x5A).all()) and bool((data[:, 2 * H:] == 0x5A).all())
        assert self.dinputs.intact() and self.dinitial.intact() and self.ws.intact()


# (T, B, H, pitch over 2 H, channels that run forward)
SIZES = [(1, 1, 1, 0, 1), (1, 3, 70, 0, 70), (2, 1, 64, 0, 0), (3, 5, 129, 7, 60), (7, 2, 256, 0, 128), (8, 3, 300, 1, 300), (9, 1, 33, 3, 16),
         (16, 2, 128, 0, 128), (17, 2, 127, 5, 1), (33, 3, 65, 1, 64), (63, 1, 500, 0, 250), (64, 4, 96, 0, 96), (65, 4, 96, 0, 48), (127, 2, 130, 0, 0),
         (128, 2, 258, 0, 258), (129, 3, 64, 64, 64), (200, 1, 1000, 0, 499), (256, 5, 40, 0, 40), (257, 2, 8, 2, 3), (511, 1, 16, 0, 16),
         (513, 3, 200, 0, 100), (1000, 2, 65, 1, 65), (1500, 1, 300, 0, 150), (4097, 1, 130, 0, 131 // 2), (20000, 1, 33, 0, 33), (50, 130, 64, 0, 64),
         (300, 70, 128, 0, 64), (1, 700, 512, 512, 512), (4, 2, 16384, 0, 16384), (140, 1, 4099, 3, 2050)]


@pytest.mark.parametrize("kind", ["all", "some", "none"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T, B, H, more, forward", SIZES)
def test_states(T, B, H, more, forward, dtype, kind):
    say("recurrence", T, B, H, more, forward, dtype, kind)
    c = Call(T, B, H, dtype, kind, 2 * H + more, forward, carried=kind != "all" or T % 2 == 1, slow=T > 200)
    c.forward_call()
    c.check_forward()


@pytest.mark.parametrize("kind", ["all", "some", "none"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T, B, H, more, forward", SIZES)
def test_gradient(T, B, H, more, forward, dtype, kind):
    say("recurrence back", T, B, H, more, forward, dtype, kind)
    c = Call(T, B, H, dtype, kind, 2 * H + more, forward, carried=kind != "all" or T % 2 == 1, slow=T > 200)
    c.backward_call()
    c.check_backward()
