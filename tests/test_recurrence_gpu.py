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
    elif kind in ("equal", "up", "down", "powers"):
        n = {"equal": np.full(B, T - 1), "up": np.linspace(0, T, B).astype(np.int32), "down": np.linspace(T + 3, -3, B).astype(np.int32),
             "powers": np.minimum(1 << rng.integers(0, T.bit_length() + 1, B), T + 1)}[kind].astype(np.int32)
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
         (300, 70, 128, 0, 64), (1, 700, 512, 512, 512), (4, 2, 16384, 0, 16384), (140, 1, 4099, 3, 2050), (700, 100, 65, 1, 65), (180, 140, 34, 0, 17),
         (260, 56, 128, 0, 64)]


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


@pytest.mark.parametrize("kind", ["equal", "up", "down", "powers"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T, B, H", [(65, 64, 2), (128, 65, 64), (129, 191, 5), (255, 7, 130), (256, 200, 3), (300, 129, 1), (511, 16, 1030)])
def test_utterances_in_every_order(T, B, H, dtype, kind):
    """Long utterances are begun first: lengths that are all the same, in order, against it, and powers of two."""
    say("orders", T, B, H, dtype, kind)
    c = Call(T, B, H, dtype, kind, None, H // 2)
    c.forward_call()
    c.check_forward()
    c.backward_call()
    c.check_backward()


@pytest.mark.parametrize("T, B, H, dtype", [(150, 130, 901, F32), (200, 190, 901, BF16)])
def test_gradient_of_more_than_the_caches_hold(T, B, H, dtype):
    """Rows that begin anywhere, of 400 MB: what is written stays in the caches."""
    say("large", T, B, H, dtype)
    c = Call(T, B, H, dtype, "some", 2 * H + 1, 300)
    c.backward_call()
    c.check_backward()


# ---- what may be done with the calls ----------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T, B, H, forward", [(1, 3, 200, 200), (40, 5, 130, 60), (300, 2, 128, 128), (5000, 1, 96, 48), (1, 600, 1025, 1025), (3, 600, 386, 129),
                                              (20, 400, 258, 257), (150, 300, 257, 129), (260, 300, 129, 129), (400, 100, 385, 128), (2000, 1, 385, 256)])
def test_states_carried_in_place(T, B, H, forward, dtype):
    """final_states in initial's place, dinitial in dfinal's: also where several workgroups share an utterance, or where one of them has a single channel, of
    which a lane of two brings the one before it, another workgroup's, too."""
    say("in place", T, B, H, forward, dtype)
    c = Call(T, B, H, dtype, "some", None, forward)
    place = put(c.initial, torch.float32)
    block.recurrence(c.inputs.t.data_ptr(), c.pitch, pointer(c.lengths), place.t.data_ptr(), T, B, H, forward, dtype,
                     Guarded((T, B, H), c.tt).t.data_ptr(), place.t.data_ptr(), c.ws_at, c.ws_bytes, stream())
    c.forward_call()
    c.check_forward()
    assert torch.equal(place.t, c.final.t) and place.intact()
    place = put(c.dfinal, torch.float32)
    c.backward_call()
    c.check_backward()
    block.recurrence_backward(c.d[0].t.data_ptr(), place.t.data_ptr(), c.inputs.t.data_ptr(), c.pitch, c.d[2].t.data_ptr(), pointer(c.lengths),
                              c.initial_dev.t.data_ptr(), T, B, H, forward, dtype, Guarded((T, B, c.pitch), c.tt).t.data_ptr(),
                              place.t.data_ptr(), c.ws_at, c.ws_bytes, stream())
    torch.cuda.synchronize()
    assert torch.equal(place.t, c.dinitial.t) and place.intact()


def test_without_last_states():
    say("no last states")
    for T in (1, 60, 700):
        c = Call(T, 2, 70, F32, "some")
        c.forward_call()
        states = Guarded((T, 2, 70), c.tt)
        block.recurrence(c.inputs.t.data_ptr(), c.pitch, pointer(c.lengths), c.initial_dev.t.data_ptr(), T, 2, 70, 70, F32, states.t.data_ptr(), None,
                         c.ws_at, c.ws_bytes, stream())
        c.backward_call()
        dinputs = Guarded((T, 2, c.pitch), c.tt)
        block.recurrence_backward(c.d[0].t.data_ptr(), c.d[1].t.data_ptr(), c.inputs.t.data_ptr(), c.pitch, c.d[2].t.data_ptr(), pointer(c.lengths),
                                  c.initial_dev.t.data_ptr(), T, 2, 70, 70, F32, dinputs.t.data_ptr(), None, c.ws_at, c.ws_bytes, stream())
        torch.cuda.synchronize()
        assert torch.equal(states.raw, c.states.raw) and torch.equal(dinputs.raw, c.dinputs.raw)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shift", [2, 4, 6, 10])
def test_alignments(shift, dtype):
    """Inputs that begin anywhere their type may, with rows of odd lengths."""
    if dtype == F32 and shift % 4:
        pytest.skip("no alignment of a float")
    say("alignment", shift, dtype)
    for H, pitch in ((101, 205), (64, 129), (2, 5), (3, 6)):
        c = Call(50, 3, H, dtype, "some", pitch, H // 2, shift=shift)
        c.forward_call()
        c.check_forward()
        c.backward_call()
        c.check_backward()


@pytest.mark.parametrize("T, at", [(30, 7), (30, 29), (300, 0), (300, 143), (300, 299), (4000, 2000)])
def test_values_that_are_not_finite(T, at):
    """A gate of infinite size is 0 or 1; an infinity or a NaN stays in its channel, behind its frame (the gradient: before it)."""
    say("not finite", T, at)
    c = Call(T, 1, 64, F32, "all", carried=True)
    c.forward_call()
    clean = c.states.t.clone()
    c.backward_call()
    clean_back = c.dinputs.t.clone()
    inputs = c.inputs.t
    inputs[at, 0, 3], inputs[at, 0, 5], inputs[at, 0, 64 + 9], inputs[at, 0, 11], inputs[at, 0, 64 + 13] = 1e30, -float("inf"), float("inf"), float("nan"), float("nan")
    c.forward_call()
    torch.cuda.synchronize()
    got, before = c.states.t[:, 0], c.initial_dev.t[0] if at == 0 else clean[at - 1, 0]
    assert float(got[at, 3]) == float(inputs[at, 0, 64 + 3]) and float(got[at, 5]) == float(before[5])
    assert bool(torch.isinf(got[at:, 9]).all()) and float(c.final.t[0, 9]) == float("inf")
    assert bool(torch.isnan(got[at:, [11, 13]]).all()) and bool(torch.isnan(c.final.t[0, [11, 13]]).all())
    assert torch.equal(got[:at], clean[:at, 0])
    untouched = [k for k in range(64) if k not in (3, 5, 9, 11, 13)]
    assert torch.equal(got[:, untouched], clean[:, 0, untouched])
    grads = c.d[0].t
    c.backward_call()
    torch.cuda.synchronize()
    assert torch.equal(c.dinputs.t[:, 0, untouched], clean_back[:, 0, untouched])
    # a NaN in a gate makes the gradients of its channel NaNs from its frame back, one in a candidate those of that frame's gate only
    assert bool(torch.isnan(c.dinputs.t[:at + 1, 0, 11]).all()) and torch.equal(c.dinputs.t[at + 1:, 0, 11], clean_back[at + 1:, 0, 11])
    assert bool(torch.isnan(c.dinputs.t[at, 0, 13])) and torch.equal(c.dinputs.t[:at, 0, 13], clean_back[:at, 0, 13])
    assert torch.equal(c.dinputs.t[:, 0, 64 + 13], clean_back[:, 0, 64 + 13])
    assert grads is not c.d[0].t


def test_gates_of_every_size():
    """z and 1 - z are good relative to themselves: slow channels forget what they should."""
    say("gates")
    g = torch.cat((torch.linspace(-90, 90, 4001), torch.tensor([0.0, -0.0, 1e-30, -1e-30, 150.0, -150.0, 3e38, -3e38])))
    H = g.numel()
    for dtype in TYPES:
        gates = g.to(torch_type(dtype)).float()
        inputs = torch.cat((gates, torch.ones(H)))[None].to(torch_type(dtype)).cuda()
        states, final = torch.empty(1, H, dtype=inputs.dtype, device="cuda"), torch.empty(1, H, device="cuda")
        block.recurrence(inputs.data_ptr(), 2 * H, None, None, 1, 1, H, H, dtype, states.data_ptr(), final.data_ptr(), None, 0, stream())
        torch.cuda.synchronize()
        z = ref.sigmoid(gates.double())[0]
        off = (final.cpu().double()[0] - z).abs() / ((ref.gate_error(gates, dtype == F32) + HALF) * z + 2.0 ** -125)
        say("   %.3f of what is allowed" % float(off.max()))
        assert float(off.max()) <= 1


def test_refuses_a_small_workspace():
    size = block.recurrence_workspace_size(1000, 2, 64)
    assert size > 0
    for call in ("recurrence", "recurrence_backward"):
        c = Call(1000, 2, 64, F32, "all")
        c.ws_bytes -= 1
        with pytest.raises(ctc.CTCError):
            c.forward_call() if call == "recurrence" else c.backward_call()


@pytest.mark.parametrize("T, B, H, forward", [(1, 4, 256, 256), (60, 3, 100, 50), (500, 40, 128, 64), (3000, 1, 64, 64)])
def test_replays_of_a_captured_call(T, B, H, forward):
    """Lengths, inputs and states are read afresh; two graphs that share a workspace, replayed in turn on one stream, do not disturb each other."""
    say("graphs", T, B, H)
    calls = [Call(T, B, H, F32, "some", None, forward, seed=s) for s in (1, 2)]
    for c in calls:                                      # (a workspace for both)
        c.ws, c.ws_at = calls[0].ws, calls[0].ws_at
        c.forward_call()
        c.backward_call()
    torch.cuda.synchronize()
    graphs = []
    side = torch.cuda.Stream()
    for c in calls:
        g = torch.cuda.CUDAGraph()
        args = (c.initial_dev, c.states, c.final, c.d, c.dinputs, c.dinitial)
        with torch.cuda.graph(g, stream=side):
            s = torch.cuda.current_stream().cuda_stream
            block.recurrence(c.inputs.t.data_ptr(), c.pitch, c.lengths.data_ptr(), args[0].t.data_ptr(), T, B, H, forward, F32, args[1].t.data_ptr(),
                             args[2].t.data_ptr(), c.ws_at, c.ws_bytes, s)
            block.recurrence_backward(args[3][0].t.data_ptr(), args[3][1].t.data_ptr(), c.inputs.t.data_ptr(), c.pitch, args[3][2].t.data_ptr(),
                                      c.lengths.data_ptr(), args[0].t.data_ptr(), T, B, H, forward, F32, args[4].t.data_ptr(),
                                      args[5].t.data_ptr(), c.ws_at, c.ws_bytes, s)
        graphs.append(g)
    for turn in range(4):
        for c, g in zip(calls, graphs):
            want = [t.t.clone() for t in (c.states, c.final, c.dinputs, c.dinitial)]
            for t in (c.states, c.final, c.dinputs, c.dinitial):
                t.t.fill_(7.0)
            eager = Call(T, B, H, F32, "some", None, forward, seed=9)         # (the program's own work in between)
            eager.forward_call()
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            there = c.counts.cuda()
            assert torch.equal(c.states.t[there], want[0][there]) and torch.equal(c.final.t, want[1])
            assert torch.equal(c.dinputs.t[there], want[2][there]) and torch.equal(c.dinitial.t, want[3])
    # other contents in the same buffers
    c = calls[0]
    c.lengths.copy_(calls[1].lengths)
    c.inputs.t.copy_(calls[1].inputs.t)
    c.initial_dev.t.copy_(calls[1].initial_dev.t)
    graphs[0].replay()
    torch.cuda.synchronize()
    there = calls[1].counts.cuda()
    assert torch.equal(c.states.t[there], calls[1].states.t[there]) and torch.equal(c.final.t, calls[1].final.t)


def test_calls_at_once():
    """Two streams, each with its own outputs and workspace, from two threads."""
    import threading
    say("two streams")
    calls = [Call(2000, 2, 200, F32, "some", seed=s) for s in (3, 4)]
    for c in calls:
        c.forward_call()
        c.backward_call()
    torch.cuda.synchronize()
    want = [[t.t.clone() for t in (c.states, c.final, c.dinputs, c.dinitial)] for c in calls]
    errors = []

    def work(c):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(20):
                    c.forward_call()
                    c.backward_call()
                torch.cuda.current_stream().synchronize()
        except Exception as e:                                                # noqa: BLE001 (told to the test)
            errors.append(e)

    threads = [threading.Thread(target=work, args=(c,)) for c in calls]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors
    for c, w in zip(calls, want):
        there = c.counts.cuda()
        assert torch.equal(c.states.t[there], w[0][there]) and torch.equal(c.final.t, w[1])
        assert torch.equal(c.dinputs.t[there], w[2][there]) and torch.equal(c.dinitial.t, w[3])


def test_beyond_2_31_elements():
    """More than 2^31 elements of inputs and of states: the last utterances and channels are those of a call of their own."""
    T, B, H = 1500, 1000, 1536
    say("beyond 2^31", T * B * H)
    gen = torch.Generator(device="cuda").manual_seed(1)
    inputs = torch.empty(T, B, 2 * H, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    states, final = torch.empty(T, B, H, dtype=torch.bfloat16, device="cuda"), torch.empty(B, H, device="cuda")
    lengths = torch.full((B,), T, dtype=torch.int32, device="cuda")
    lengths[-1] = T - 3
    block.recurrence(inputs.data_ptr(), 2 * H, lengths.data_ptr(), None, T, B, H, H - 64, BF16, states.data_ptr(), final.data_ptr(), *workspace(T, B, H), stream())
    torch.cuda.synchronize()
    part = inputs[:, -2:].contiguous()
    ps, pf = torch.zeros(T, 2, H, dtype=torch.bfloat16, device="cuda"), torch.empty(2, H, device="cuda")
    block.recurrence(part.data_ptr(), 2 * H, lengths[-2:].data_ptr(), None, T, 2, H, H - 64, BF16, ps.data_ptr(), pf.data_ptr(), *workspace(T, 2, H), stream())
    torch.cuda.synchronize()
    # (two ways to deal the frames out: the states agree but for fp64's roundings, which now and then are the other side of a bf16's middle)
    assert float((states[:T - 3, -2:].float() - ps[:T - 3].float()).abs().max()) <= 2.0 ** -7 * float(ps.abs().max())
    assert torch.allclose(final[-2:], pf, rtol=0, atol=2.0 ** -23 * float(pf.abs().max()))
    dinputs, d0 = torch.empty_like(inputs), torch.empty(B, H, device="cuda")
    block.recurrence_backward(states.data_ptr(), None, inputs.data_ptr(), 2 * H, states.data_ptr(), lengths.data_ptr(), None, T, B, H, H - 64, BF16,
                              dinputs.data_ptr(), d0.data_ptr(), *workspace(T, B, H), stream())
    torch.cuda.synchronize()
    ps.copy_(states[:, -2:])
    pd, p0 = torch.empty_like(part), torch.empty(2, H, device="cuda")
    block.recurrence_backward(ps.data_ptr(), None, part.data_ptr(), 2 * H, ps.data_ptr(), lengths[-2:].data_ptr(), None, T, 2, H, H - 64, BF16,
                              pd.data_ptr(), p0.data_ptr(), *workspace(T, 2, H), stream())
    torch.cuda.synchronize()
    assert float((dinputs[:T - 3, -2:].float() - pd[:T - 3].float()).abs().max()) <= 2.0 ** -7 * float(pd[:T - 3].abs().max())
    assert torch.allclose(d0[-2:], p0, rtol=0, atol=2.0 ** -22 * float(p0.abs().max()))


def workspace(T, B, H):
    size = block.recurrence_workspace_size(T, B, H)
    ws = torch.empty(size + 256, dtype=torch.uint8, device="cuda")
    workspace.kept = ws                                  # (until the next one: the calls above are waited for)
    return (ws.data_ptr() + 255) // 256 * 256, size
