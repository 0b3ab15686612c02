"""The operators of a recurrent block under the output layer, as cases that can be timed and compared with their plain forms.

Between the features and the output layer lies a stack of recurrent blocks.  A block is a projection of its input to a
gate, a candidate and an output gate, a gated linear recurrence over the frames, and a norm of what that makes, gated,
scaled and added to the residual stream, whose norm is the next block's input.  In training the projections are ordinary
matrix products; a streaming recogniser, which has a frame or a few at a time, keeps their weights (and the output
layer's) in 4 bits.

  call      "recurrence"        states of all frames from gates and candidates (block.recurrence)
            "recurrence back"   its gradient (block.recurrence_backward)
            "norm"              norm after a block, gate, residual scale, residual, norm before the next (block.block_norm)
            "norm back"         its gradient (block.block_norm_backward)
            "weights"           weights to 4 bits with a scale per group, and read back for comparison
                                (block.quantize_weights_i4, block.dequantize_weights_i4)
            "product"           rows in 8 bits by weights in 4 (block.linear_i4)

Fields of a case:

  dtype     "f32" or "bf16": type of states, gates, activations and gradients
  B, T      utterances and frames of the tensor: B * T rows, row t * B + b
  H, A      width of a state, rows of the weights (0 where a call has none)
  shortest  input lengths are uniform in [shortest, T]; 0: all frames count, and no lengths are passed
  forward   share of the channels that run forward in time: 1.0, or 0.5 in a layer of both directions
  pitch     matrices that a row of projections lies in: it is pitch * H elements from one row to the next
  carried   whether states from before are passed in, and gradients of the last states (streaming in chunks), or a residual
  group     columns to a scale of the weights

Gates are normal around a mean of the channel's own, so that some channels forget within a few frames and some remember
hundreds; candidates and gradients are normal.  Rows behind an utterance's end hold zeros and stay so.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

EPS = 1e-6
LEVELS = 7                   # the largest value in 4 bits
ROW_LEVELS = 127             # and in 8
BLOCK = 64                   # frames that the plain recurrence takes at a time
MOST_BYTES = 100_000_000     # a drawn case's rows in one tensor (27200 frames, 2048 wide, in 16 bits: 111 MB)
MOST_WEIGHTS = 12_000_000    # rows x columns of a drawn case's weights
MOST_PRODUCTS = 3_000_000_000       # and its products (256 rows, 2048 wide, by 6144)


def _case(name, call, dtype, B, T, H, A=0, shortest=0, forward=1.0, pitch=2, carried=False, group=0):
    return {"name": name, "call": call, "dtype": dtype, "B": B, "T": T, "H": H, "A": A, "shortest": shortest,
            "forward": forward, "pitch": pitch, "carried": carried, "group": group}


def listed():
    return [
        # one frame of one utterance, streaming: the states are carried from call to call
        _case("recurrence one frame", "recurrence", "bf16", 1, 1, 2048, carried=True),
        # a recurrent layer on an English minibatch
        _case("recurrence english", "recurrence", "bf16", 64, 750, 2048, shortest=100, pitch=3),
        # one long recording, in one piece
        _case("recurrence long", "recurrence", "f32", 1, 40000, 1024),
        # the gradient of a layer of both directions on an English minibatch
        _case("recurrence back english", "recurrence back", "bf16", 64, 750, 2048, shortest=100, forward=0.5, pitch=3),
        # sizes that are no multiple of anything, continued from a chunk before
        _case("recurrence back odd", "recurrence back", "f32", 27, 333, 1999, shortest=80, carried=True),
        # one frame of one utterance between two blocks
        _case("norm one frame", "norm", "bf16", 1, 1, 2048, pitch=1, carried=True),
        # an English minibatch between two blocks
        _case("norm english", "norm", "bf16", 64, 750, 2048, shortest=100, pitch=3, carried=True),
        # its gradient
        _case("norm back english", "norm back", "bf16", 64, 750, 2048, shortest=100, pitch=3, carried=True),
        # a width and a batch that are no multiple of anything
        _case("norm back odd", "norm back", "f32", 27, 333, 1999, shortest=80, pitch=1, carried=True),
        # the weights of an ideographic output layer
        _case("weights ideographs", "weights", "f32", 1, 1, 2048, 6000, group=128),
        # one frame of one utterance through that layer: every weight is read for one row
        _case("product one frame", "product", "f32", 1, 1, 2048, 6000, group=128),
        # four frames each of 64 utterances through a block's projections
        _case("product projections", "product", "bf16", 64, 4, 2048, 6144, group=64),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    call = rng.choice(["recurrence", "recurrence", "recurrence back", "recurrence back", "norm", "norm back", "weights",
                       "product", "product"])
    dtype = rng.choice(["f32", "bf16"])
    H = _log_uniform(rng, 64, 4096)
    if rng.random() < 0.4:
        H = max(64, H - H % 64)
    if call in ("weights", "product"):
        A = min(rng.choice([rng.randint(20, 64), _log_uniform(rng, 65, 16384)]), MOST_WEIGHTS // H)
        rows = 1 if call == "weights" else rng.choice([1, min(_log_uniform(rng, 2, 512), MOST_PRODUCTS // (A * H))])
        case = _case("", call, dtype, rows, 1, H, A, group=rng.choice([64, 128]))
        del case["name"]
        return case
    kind = rng.choice(["frame", "minibatch", "minibatch", "recording"])
    T = 1 if kind == "frame" else _log_uniform(rng, 16, 1500) if kind == "minibatch" else _log_uniform(rng, 1501, 40000)
    B = rng.randint(1, 4) if kind == "recording" else _log_uniform(rng, 1, 512)
    most = MOST_BYTES // (T * H * (4 if dtype == "f32" else 2))
    H = H if most else MOST_BYTES // (4 * T)
    B = max(1, min(B, most))
    shortest = 0 if T == 1 or rng.random() < 0.3 else max(1, int(T * rng.uniform(0.1, 0.9)))
    scan = call in ("recurrence", "recurrence back")
    case = _case("", call, dtype, B, T, H, 0, shortest, rng.choice([1.0, 1.0, 0.5]) if scan else 1.0,
                 rng.choice([2, 3]) if scan else rng.choice([1, 3]), rng.random() < 0.6)
    del case["name"]
    return case


def _type(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def prepare(case, seed):
    dev = torch.device("cuda:0")
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed))
    rng = np.random.default_rng(seed)
    B, T, H, A, call, dtype = case["B"], case["T"], case["H"], case["A"], case["call"], _type(case)
    rows, pitch = B * T, case["pitch"] * H

    def normal(*shape, scale=1.0):
        return torch.randn(shape, generator=gen, device=dev) * scale

    def zeros(*shape, dtype=torch.float32):
        return torch.zeros(shape, dtype=dtype, device=dev)

    s = {"case": case, "rows": rows, "lengths": None, "frames": None, "index": slice(None)}
    counts = torch.ones((T, B, 1), dtype=torch.bool, device=dev)
    if case["shortest"]:
        # lengths on the GPU, and the list of a minibatch's frames: their number, then the rows
        s["lengths"] = torch.from_numpy(rng.integers(case["shortest"], T + 1, B).astype(np.int32)).to(dev)
        counts = (torch.arange(T, device=dev)[:, None] < s["lengths"][None, :])[:, :, None]
        s["index"] = torch.nonzero(counts.flatten()).flatten()
        s["frames"] = torch.zeros(1 + rows, dtype=torch.int32, device=dev)
        s["frames"][0] = s["index"].numel()
        s["frames"][1:1 + s["index"].numel()] = s["index"].to(torch.int32)
    flat = counts.view(rows, 1)

    if call in ("recurrence", "recurrence back"):
        s["forward"] = H if case["forward"] == 1.0 else H // 2
        gates = normal(T, B, H, scale=1.5) - 6.0 * torch.rand((1, 1, H), generator=gen, device=dev) + 1.0
        s["inputs"] = zeros(T, B, pitch, dtype=dtype)
        s["inputs"][:, :, :H] = torch.where(counts, gates, 0.0)
        del gates
        s["inputs"][:, :, H:2 * H] = torch.where(counts, normal(T, B, H), 0.0)
        s["initial"] = normal(B, H) if case["carried"] else None
        if call == "recurrence":
            s["states"], s["final"] = zeros(T, B, H, dtype=dtype), zeros(B, H)
        else:
            s["states"] = torch.where(counts, normal(T, B, H, scale=0.5), 0.0).to(dtype)
            s["dstates"] = torch.where(counts, normal(T, B, H, scale=1e-3), 0.0).to(dtype)
            s["dfinal"] = normal(B, H, scale=1e-3) if case["carried"] else None
            s["dinputs"], s["dinitial"] = zeros(T, B, pitch, dtype=dtype), zeros(B, H)
    if call in ("norm", "norm back"):
        channels = torch.exp(0.5 * normal(1, H))
        s["x"] = torch.where(flat, normal(rows, H) * channels, 0.0).to(dtype)
        s["gate"] = zeros(rows, pitch, dtype=dtype)
        s["gate"][:, :H] = torch.where(flat, normal(rows, H, scale=1.5), 0.0)
        s["weight_after"], s["weight_before"] = 1.0 + 0.2 * normal(H), 1.0 + 0.2 * normal(H)
        s["scale"] = 0.3 + 0.1 * normal(H)
        stream = torch.where(flat, normal(rows, H) * channels, 0.0).to(dtype)
        if call == "norm":
            s["residual"] = stream if case["carried"] else None
            s["sum"], s["normed"] = zeros(rows, H, dtype=dtype), zeros(rows, H, dtype=dtype)
        else:
            s["sum"] = stream
            s["dnormed"] = torch.where(flat, normal(rows, H, scale=1e-3), 0.0).to(dtype)
            s["dsum"] = torch.where(flat, normal(rows, H, scale=1e-3), 0.0).to(dtype) if case["carried"] else None
            s["dx"], s["dresidual"] = zeros(rows, H, dtype=dtype), zeros(rows, H, dtype=dtype)
            s["dgate"] = zeros(rows, pitch, dtype=dtype)
            s["dweight_after"], s["dscale"], s["dweight_before"] = zeros(H), zeros(H), zeros(H)
    if call in ("weights", "product"):
        w = normal(A, H, scale=1.0 / math.sqrt(H))
        if call == "weights":
            s["weight"], s["values"] = w.to(dtype), zeros(A, H, dtype=dtype)
        else:
            # weights as 4 bits hold them, so that both forms begin with the same
            group = case["group"]
            parts = torch.nn.functional.pad(w, (0, -H % group)).view(A, -1, group)
            m = parts.abs().amax(2, keepdim=True)
            s["weight_q"] = torch.round(parts * (LEVELS / m.clamp(min=1e-30))).to(torch.int8).view(A, -1)[:, :H].contiguous()
            s["weight_scales"] = (m / LEVELS).view(A, -1).contiguous()
            x = normal(rows, H) * torch.exp(0.5 * normal(1, H))
            m = x.abs().amax(1).clamp(min=1e-30)
            q = torch.round(x * (ROW_LEVELS / m)[:, None]).to(torch.int8)
            s["q"], s["scales"] = torch.nn.functional.pad(q, (0, -H % 128)).contiguous(), m / ROW_LEVELS
            s["bias"] = 0.5 * normal(A)
            s["logits"] = zeros(rows, A, dtype=dtype)
    if own:
        _prepare_own(s)
    return s


def _prepare_own(s):
    """What a user's program keeps beside its data: workspaces, and the weights as the library lays them out."""
    from paper_1512_02595_amd import block, ctc
    c = s["case"]
    B, T, H, A, call = c["B"], c["T"], c["H"], c["A"], c["call"]
    dev = torch.device("cuda:0")
    size = (block.recurrence_workspace_size(T, B, H) if call in ("recurrence", "recurrence back") else
            block.block_norm_workspace_size(s["rows"], H) if call == "norm back" else 0)
    s["workspace"] = torch.empty(size + 256, dtype=torch.uint8, device=dev)
    s["ws_ptr"], s["ws_bytes"] = (s["workspace"].data_ptr() + 255) // 256 * 256, size
    if call in ("weights", "product"):
        weights, scales = block.weights_i4_sizes(A, H, c["group"])
        s["packed"] = torch.zeros(weights, dtype=torch.uint8, device=dev)
        s["packed_scales"] = torch.zeros(scales // 4, device=dev)
    if call == "product":
        # The library rounds a group's values to sevenths of its largest: those that stand for themselves come out as they
        # were.  (The largest of a group is a seven, unless the group is all zeros.)
        spread = s["weight_scales"].repeat_interleave(c["group"], 1)[:, :H]
        values = (s["weight_q"].float() * spread).contiguous()
        block.quantize_weights_i4(values.data_ptr(), A, H, c["group"], ctc.DTYPE_F32, s["packed"].data_ptr(),
                                  s["packed_scales"].data_ptr(), torch.cuda.current_stream().cuda_stream)


def run(s):
    return _own(s) if own else _plain(s)


def _address(t):
    return None if t is None else t.data_ptr()


def _own(s):
    from paper_1512_02595_amd import block, ctc
    c = s["case"]
    B, T, H, A, call, group = c["B"], c["T"], c["H"], c["A"], c["call"], c["group"]
    pitch = c["pitch"] * H
    dtype = ctc.DTYPE_F32 if c["dtype"] == "f32" else ctc.DTYPE_BF16
    stream = torch.cuda.current_stream().cuda_stream
    if call == "recurrence":
        block.recurrence(s["inputs"].data_ptr(), pitch, _address(s["lengths"]), _address(s["initial"]), T, B, H, s["forward"], dtype,
                         s["states"].data_ptr(), s["final"].data_ptr(), s["ws_ptr"], s["ws_bytes"], stream)
        return {"states": s["states"], "final": s["final"]}
    if call == "recurrence back":
        block.recurrence_backward(s["dstates"].data_ptr(), _address(s["dfinal"]), s["inputs"].data_ptr(), pitch,
                                  s["states"].data_ptr(), _address(s["lengths"]), _address(s["initial"]), T, B, H, s["forward"], dtype,
                                  s["dinputs"].data_ptr(), s["dinitial"].data_ptr(), s["ws_ptr"], s["ws_bytes"], stream)
        return {"dinputs": s["dinputs"][:, :, :2 * H], "dinitial": s["dinitial"]}
    if call == "norm":
        block.block_norm(s["x"].data_ptr(), s["gate"].data_ptr(), pitch, _address(s["residual"]), s["weight_after"].data_ptr(),
                         s["scale"].data_ptr(), s["weight_before"].data_ptr(), EPS, _address(s["frames"]), s["rows"], H, dtype,
                         s["sum"].data_ptr(), s["normed"].data_ptr(), stream)
        return {"sum": s["sum"], "normed": s["normed"]}
    if call == "norm back":
        block.block_norm_backward(s["dnormed"].data_ptr(), _address(s["dsum"]), s["x"].data_ptr(), s["gate"].data_ptr(), pitch,
                                  s["sum"].data_ptr(), s["weight_after"].data_ptr(), s["scale"].data_ptr(),
                                  s["weight_before"].data_ptr(), EPS, _address(s["frames"]), s["rows"], H, dtype, s["dx"].data_ptr(),
                                  s["dgate"].data_ptr(), s["dresidual"].data_ptr(), s["dweight_after"].data_ptr(),
                                  s["dscale"].data_ptr(), s["dweight_before"].data_ptr(), s["ws_ptr"], s["ws_bytes"], stream)
        return {"dx": s["dx"], "dgate": s["dgate"][:, :H], "dresidual": s["dresidual"], "dweight_after": s["dweight_after"],
                "dscale": s["dscale"], "dweight_before": s["dweight_before"]}
    if call == "weights":
        block.quantize_weights_i4(s["weight"].data_ptr(), A, H, group, dtype, s["packed"].data_ptr(),
                                  s["packed_scales"].data_ptr(), stream)
        block.dequantize_weights_i4(s["packed"].data_ptr(), s["packed_scales"].data_ptr(), A, H, group, dtype,
                                    s["values"].data_ptr(), stream)
        return {"values": s["values"]}
    block.linear_i4(s["q"].data_ptr(), s["scales"].data_ptr(), s["packed"].data_ptr(), s["packed_scales"].data_ptr(), group,
                    s["bias"].data_ptr(), None, s["rows"], H, A, dtype, s["logits"].data_ptr(), stream)
    return {"logits": s["logits"]}


def _whole(s, rows):
    """The listed rows in a tensor of all rows; the others hold zeros."""
    if s["frames"] is None:
        return rows
    out = torch.zeros((s["rows"], rows.shape[1]), dtype=rows.dtype, device=rows.device)
    out[s["index"]] = rows
    return out


def _ordered(s, x):
    """[T, B, H] with the frames of channels that run backward in time turned round, and so back again.  Frames that do
    not count stay where they are, behind the others."""
    F = s["forward"]
    if F == x.shape[2]:
        return x
    T, B = s["case"]["T"], s["case"]["B"]
    t = torch.arange(T, device=x.device)[:, None].expand(T, B)
    n = torch.full((B,), T, device=x.device) if s["lengths"] is None else s["lengths"].long()
    at = torch.where(t < n, n - 1 - t, t)[:, :, None].expand(-1, -1, x.shape[2] - F)
    return torch.cat((x[:, :, :F], torch.gather(x[:, :, F:], 0, at)), 2)


def _scan(keep, add, carry):
    """y_t = keep_t y_(t-1) + add_t over [T, B, H], `keep` and `add` by blocks of frames, doubling the stretch each frame covers."""
    out = torch.empty_like(add)
    for t0 in range(0, add.shape[0], BLOCK):
        k, a = keep[t0:t0 + BLOCK].clone(), add[t0:t0 + BLOCK].clone()
        d = 1
        while d < a.shape[0]:
            a[d:] = a[d:] + k[d:] * a[:-d]
            k[d:] = k[d:] * k[:-d]
            d *= 2
        out[t0:t0 + BLOCK] = a + k * carry
        carry = out[min(t0 + BLOCK, add.shape[0]) - 1]
    return out, carry


def _plain_recurrence(s):
    # in 64 bits: a slow channel's share that stays, nearly one, is taken to the power of hundreds
    c = s["case"]
    T, H, dtype = c["T"], c["H"], _type(c)
    counts = None if s["lengths"] is None else (torch.arange(T, device=s["inputs"].device)[:, None] < s["lengths"])[:, :, None]
    z = torch.sigmoid(_ordered(s, s["inputs"][:, :, :H]).float()).double()
    x = _ordered(s, s["inputs"][:, :, H:2 * H]).double()
    if counts is not None:
        z = torch.where(counts, z, 0.0)
    first = torch.zeros((c["B"], H), dtype=torch.float64, device=z.device) if s["initial"] is None else s["initial"].double()
    h, last = _scan(1.0 - z, z * x, first)
    # the order's own inverse; frames that do not count are zeros
    states = _ordered(s, h if counts is None else torch.where(counts, h, 0.0))
    return {"states": states.to(dtype), "final": last.float()}


def _plain_recurrence_back(s):
    c = s["case"]
    T, H, dtype = c["T"], c["H"], _type(c)
    dev = s["inputs"].device
    counts = torch.ones((T, 1, 1), dtype=torch.bool, device=dev)
    if s["lengths"] is not None:
        counts = (torch.arange(T, device=dev)[:, None] < s["lengths"])[:, :, None]
    nothing = torch.zeros((c["B"], H), dtype=torch.float64, device=dev)
    z = torch.where(counts, torch.sigmoid(_ordered(s, s["inputs"][:, :, :H]).float()).double(), 0.0)
    x = _ordered(s, s["inputs"][:, :, H:2 * H]).double()
    h = _ordered(s, s["states"]).double()
    before = torch.cat(((nothing if s["initial"] is None else s["initial"].double())[None], h[:-1]))
    dh = torch.where(counts, _ordered(s, s["dstates"]).double(), 0.0)
    # what reaches frame t from those behind it: e_t = (1 - z_(t+1)) (dh_(t+1) + e_(t+1)), the scan the other way
    keep = (1.0 - z).flip(0)
    e, dfirst = _scan(keep, keep * dh.flip(0), nothing if s["dfinal"] is None else s["dfinal"].double())
    e = torch.cat((e.flip(0)[1:], (nothing if s["dfinal"] is None else s["dfinal"].double())[None]))
    d = torch.where(counts, dh + e, 0.0)
    dgates = _ordered(s, d * (x - before) * z * (1.0 - z))
    dcandidates = _ordered(s, d * z)
    return {"dinputs": torch.cat((dgates, dcandidates), 2).to(dtype), "dinitial": dfirst.float()}


def _plain(s):
    c = s["case"]
    H, A, call, dtype, index = c["H"], c["A"], c["call"], _type(c), s["index"]
    if call == "recurrence":
        return _plain_recurrence(s)
    if call == "recurrence back":
        return _plain_recurrence_back(s)
    if call in ("norm", "norm back"):
        x, gate = s["x"][index].float(), s["gate"][index, :H].float()
        r1 = torch.rsqrt((x * x).mean(1, keepdim=True) + EPS)
        share = torch.sigmoid(gate)
        a, n = gate * share, x * r1
        if call == "norm":
            z = s["scale"] * a * (n * s["weight_after"])
            if s["residual"] is not None:
                z = z + s["residual"][index].float()
            z = z.to(dtype)
            v = z.float()
            y = v * torch.rsqrt((v * v).mean(1, keepdim=True) + EPS) * s["weight_before"]
            return {"sum": _whole(s, z), "normed": _whole(s, y.to(dtype))}
        z, dy = s["sum"][index].float(), s["dnormed"][index].float()
        r2 = torch.rsqrt((z * z).mean(1, keepdim=True) + EPS)
        m, g = z * r2, dy * s["weight_before"]
        dz = r2 * (g - m * (g * m).mean(1, keepdim=True))
        if s["dsum"] is not None:
            dz = dz + s["dsum"][index].float()
        dn = dz * s["scale"] * a * s["weight_after"]
        dx = r1 * (dn - n * (dn * n).mean(1, keepdim=True))
        dgate = dz * s["scale"] * (n * s["weight_after"]) * (share * (1.0 + gate * (1.0 - share)))
        return {"dx": _whole(s, dx.to(dtype)), "dgate": _whole(s, dgate.to(dtype)), "dresidual": _whole(s, dz.to(dtype)),
                "dweight_after": (dz * s["scale"] * a * n).sum(0), "dscale": (dz * a * (n * s["weight_after"])).sum(0),
                "dweight_before": (dy * m).sum(0)}
    group = c["group"]
    if call == "weights":
        # in 64 bits: which of two whole numbers is the nearer is a matter of the last bits
        parts = torch.nn.functional.pad(s["weight"].float(), (0, -H % group)).view(A, -1, group)
        m = parts.abs().amax(2, keepdim=True)
        q = torch.where(m > 0, torch.round(parts.double() * LEVELS / m.double()), 0.0).float()
        return {"values": (q * (m / LEVELS)).view(A, -1)[:, :H].to(dtype)}
    w = s["weight_q"].float() * s["weight_scales"].repeat_interleave(group, 1)[:, :H]
    y = s["q"][:, :H].float() * s["scales"][:, None]
    return {"logits": (torch.matmul(y, w.t()) + s["bias"]).to(dtype)}


def work(case):
    """Every row that counts read once and written once, in inputs and outputs each; the formulas' additions and products,
    with an exponential or a division as one."""
    B, T, H, A, call = case["B"], case["T"], case["H"], case["A"], case["call"]
    e = 4 if case["dtype"] == "f32" else 2
    n = B * (case["shortest"] + T) / 2 if case["shortest"] else B * T
    extra = 1 if case["carried"] else 0
    if call == "recurrence":
        return {"bytes": 3 * n * H * e + (1 + extra) * 4 * B * H, "flops": 7 * n * H}
    if call == "recurrence back":
        return {"bytes": 6 * n * H * e + (1 + 2 * extra) * 4 * B * H, "flops": 13 * n * H}
    if call == "norm":
        return {"bytes": (4 + extra) * n * H * e + 12 * H, "flops": 14 * n * H}
    if call == "norm back":
        return {"bytes": (7 + extra) * n * H * e + 24 * H, "flops": 36 * n * H}
    scales = 4 * A * -(-H // case["group"])
    if call == "weights":
        return {"bytes": A * H * (2 * e + 1) + 2 * scales, "flops": 5 * A * H}
    return {"bytes": n * (H + 4) + A * (H / 2 + 4) + scales + n * A * e, "flops": 2 * n * A * H}


def exact(case, seed):
    """The definitions in 64 bits, frame after frame and row after row.  What is defined as rounded on the way is the sum
    that the norm stores, and the whole numbers."""
    s = prepare(case, seed)
    B, T, H, A, call = case["B"], case["T"], case["H"], case["A"], case["call"]
    dev = torch.device("cuda:0")
    if call in ("recurrence", "recurrence back"):
        n = torch.full((B,), T, device=dev) if s["lengths"] is None else s["lengths"].long()
        utterances, F = torch.arange(B, device=dev), s["forward"]
        begin = torch.zeros((B, H), dtype=torch.float64, device=dev) if s["initial"] is None else s["initial"].double()
        if call == "recurrence":
            states, final = torch.zeros((T, B, H), dtype=torch.float64, device=dev), torch.zeros((B, H), dtype=torch.float64, device=dev)
        else:
            dinputs, dinitial = torch.zeros((T, B, 2 * H), dtype=torch.float64, device=dev), torch.zeros((B, H), dtype=torch.float64, device=dev)
        for part, reverse in ((slice(0, F), False), (slice(F, H), True)):
            width = part.stop - part.start
            if width == 0:
                continue
            candidates = slice(H + part.start, H + part.stop)

            def frame(i):
                """Where the i-th step of each utterance lies, and whether it has one."""
                there = (i < n)[:, None]
                return (torch.where(i < n, n - 1 - i, 0) if reverse else torch.full((B,), i, device=dev)), there

            if call == "recurrence":
                h = begin[:, part]
                for i in range(T):
                    t, there = frame(i)
                    z = 1.0 / (1.0 + torch.exp(-s["inputs"][t, utterances, part].double()))
                    h = torch.where(there, (1.0 - z) * h + z * s["inputs"][t, utterances, candidates].double(), h)
                    if bool(case["shortest"]):
                        states[t, utterances, part] = torch.where(there, h, states[t, utterances, part])
                    else:
                        states[t, utterances, part] = h
                final[:, part] = h
                continue
            d = torch.zeros((B, width), dtype=torch.float64, device=dev) if s["dfinal"] is None else s["dfinal"][:, part].double()
            for i in reversed(range(T)):
                t, there = frame(i)
                p = s["inputs"][t, utterances, part].double()
                z, stays = 1.0 / (1.0 + torch.exp(-p)), 1.0 / (1.0 + torch.exp(p))
                before = begin[:, part]
                if i:
                    t0, _ = frame(i - 1)
                    before = s["states"][t0, utterances, part].double()
                whole = s["dstates"][t, utterances, part].double() + d
                dp = whole * (s["inputs"][t, utterances, candidates].double() - before) * z * stays
                dinputs[t, utterances, part] = torch.where(there, dp, dinputs[t, utterances, part])
                dinputs[t, utterances, candidates] = torch.where(there, whole * z, dinputs[t, utterances, candidates])
                d = torch.where(there, whole * stays, d)
            dinitial[:, part] = d
        return {"states": states, "final": final} if call == "recurrence" else {"dinputs": dinputs, "dinitial": dinitial}
    if call in ("norm", "norm back"):
        rows = s["rows"]
        keep = torch.ones(rows, dtype=torch.bool, device=dev)
        if s["frames"] is not None:
            keep = torch.zeros(rows, dtype=torch.bool, device=dev)
            keep[s["frames"][1:1 + int(s["frames"][0])].long()] = True
        after, before, scale = s["weight_after"].double(), s["weight_before"].double(), s["scale"].double()
        step = max(1, 30_000_000 // H)
        out = {}

        def put(name, value, b):
            if name not in out:
                out[name] = torch.zeros((rows, H), dtype=torch.float64, device=dev)
            out[name][b] = torch.where(keep[b, None], value, 0.0)

        sums = {k: torch.zeros(H, dtype=torch.float64, device=dev) for k in ("dweight_after", "dscale", "dweight_before")}
        for i in range(0, rows, step):
            b = slice(i, min(i + step, rows))
            x, p = s["x"][b].double(), s["gate"][b, :H].double()
            v1 = torch.sum(x * x, dim=1)[:, None] / H + EPS
            gate = p / (1.0 + torch.exp(-p))
            normed = x / v1.sqrt()
            if call == "norm":
                z = scale * after * gate * normed
                if s["residual"] is not None:
                    z = z + s["residual"][b].double()
                put("sum", z, b)
                z = z.to(_type(case)).double()
                put("normed", before * z / (torch.sum(z * z, dim=1)[:, None] / H + EPS).sqrt(), b)
                continue
            z, dy = s["sum"][b].double(), s["dnormed"][b].double()
            v2 = torch.sum(z * z, dim=1)[:, None] / H + EPS
            dz = dy * before / v2.sqrt() - z * torch.sum(dy * before * z, dim=1)[:, None] / (H * v2 * v2.sqrt())
            if s["dsum"] is not None:
                dz = dz + s["dsum"][b].double()
            dz = torch.where(keep[b, None], dz, 0.0)
            put("dresidual", dz, b)
            dn = dz * scale * after * gate
            put("dx", dn / v1.sqrt() - x * torch.sum(dn * x, dim=1)[:, None] / (H * v1 * v1.sqrt()), b)
            e = torch.exp(-p)
            put("dgate", dz * scale * after * normed * (1.0 + e + p * e) / ((1.0 + e) * (1.0 + e)), b)
            sums["dweight_after"] += torch.sum(dz * scale * gate * normed, dim=0)
            sums["dscale"] += torch.sum(dz * after * gate * normed, dim=0)
            sums["dweight_before"] += torch.sum(torch.where(keep[b, None], dy * z / v2.sqrt(), 0.0), dim=0)
        if call == "norm":
            return {"sum": out["sum"], "normed": out["normed"]}
        return {"dx": out["dx"], "dgate": out["dgate"], "dresidual": out["dresidual"], **sums}
    group = case["group"]
    if call == "weights":
        values = torch.zeros((A, H), dtype=torch.float64, device=dev)
        for k in range(0, H, group):
            u = s["weight"][:, k:k + group].double()
            m = u.abs().max(dim=1).values[:, None]
            values[:, k:k + group] = torch.where(m > 0, torch.round(7.0 * u / torch.where(m > 0, m, 1.0)), 0.0) * m / 7.0
        return {"values": values}
    total = torch.zeros((s["rows"], A), dtype=torch.float64, device=dev)
    for i, k in enumerate(range(0, H, group)):
        q, w = s["q"][:, k:min(k + group, H)].double(), s["weight_q"][:, k:k + group].double().t().contiguous()
        total += (q @ w) * s["weight_scales"][:, i].double()
    return {"logits": total * s["scales"].double()[:, None] + s["bias"].double()}
