"""The output layer's operators, as cases that can be timed and compared with their plain forms.

CTC's activations are what an output layer makes of a network's last states, and CTC's gradient is where that layer's
backward pass begins.  The operators are those of such a layer whose states are held in 8 bits:

  call      "save"     rows are rounded to 8 bits with a scale each and read back: weights laid out per symbol, states kept
                       for the backward pass (layer.quantize_rows, layer.dequantize_rows)
            "norm"     residual added, root-mean-square norm, rows in 8 bits; read back for comparison
                       (layer.rms_norm_i8, layer.dequantize_rows)
            "norm back"    the norm's gradient (layer.rms_norm_backward)
            "product"  activations from rows and weights in 8 bits (layer.linear_i8)
            "weights"  the weights' gradient from CTC's gradient and the rows held in 8 bits (layer.weight_gradient_i8)

Fields of a case:

  dtype     "f32" or "bf16": type of states, activations and gradients
  B, T      utterances and frames of the tensor: B * T rows, row t * B + b
  H, A      width of a state, symbols of the alphabet (0 where a call has none)
  shortest  input lengths are uniform in [shortest, T]; 0: all rows count, and no list of rows is passed
  residual  whether the norm adds one, or its gradient has one to go on

States are normal with channels of unlike size, as a residual stream has them; weights are normal; the gradient of the
activations is a softmax less one symbol a frame, as CTC's is.  Rows behind an utterance's end hold zeros and stay so.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

LEVELS = 127                 # the largest value in 8 bits
EPS = 1e-6
NARROW = 64                  # alphabets of characters
MOST_STATES = 98_000_000     # rows x width of a drawn case (64 utterances of 750 frames, 2048 wide)
MOST_PRODUCTS = 240_000_000_000     # frames x width x symbols (64 utterances of up to 500 frames, 2048 wide, 6000 symbols)


def _case(name, call, dtype, B, T, H, A=0, shortest=0, residual=False):
    return {"name": name, "call": call, "dtype": dtype, "B": B, "T": T, "H": H, "A": A, "shortest": shortest,
            "residual": residual}


def listed():
    return [
        # the weights of an ideographic output layer, laid out after a step of the optimiser
        _case("save weights", "save", "f32", 6000, 1, 2048),
        # the states of an English minibatch kept for the backward pass
        _case("save states", "save", "bf16", 64, 750, 2048, shortest=100),
        # one frame of one utterance, streaming recognition
        _case("norm one frame", "norm", "bf16", 1, 1, 2048, residual=True),
        # the last norm of an English minibatch before its output layer
        _case("norm english", "norm", "bf16", 64, 750, 2048, shortest=100, residual=True),
        # its gradient, with the residual's own
        _case("norm back english", "norm back", "bf16", 64, 750, 2048, shortest=100, residual=True),
        # a width and a batch that are no multiple of anything
        _case("norm back odd", "norm back", "f32", 27, 333, 1999, shortest=80),
        # one frame of one utterance, ideographs: every weight is read for one row
        _case("product one frame", "product", "f32", 1, 1, 2048, 6000),
        # the English output layer
        _case("product english", "product", "f32", 64, 750, 2048, 29, shortest=100),
        # the Mandarin output layer
        _case("product mandarin", "product", "f32", 64, 500, 2048, 6000, shortest=100),
        # odd in every size
        _case("product odd", "product", "bf16", 27, 333, 1111, 4733, shortest=80),
        # the gradient of the English output layer's weights
        _case("weights english", "weights", "f32", 64, 750, 2048, 29, shortest=100),
        # and of the Mandarin one's, from activations in bf16
        _case("weights mandarin", "weights", "bf16", 64, 500, 2048, 6000, shortest=100),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    call = rng.choice(["save", "norm", "norm", "norm back", "product", "product", "product", "weights", "weights"])
    dtype = rng.choice(["f32", "bf16"])
    H = _log_uniform(rng, 64, 4096)
    if rng.random() < 0.4:
        H = max(64, H - H % 64)
    A = 0
    if call in ("product", "weights"):
        kind = rng.choice(["characters", "pairs", "ideographs"])
        A = rng.randint(20, NARROW) if kind == "characters" else _log_uniform(rng, NARROW + 1, 2048) if kind == "pairs" else _log_uniform(rng, 2049, 8000)
    # a frame at a time, or whole utterances
    T = 1 if call != "weights" and rng.random() < 0.25 else _log_uniform(rng, 16, 1500)
    B = _log_uniform(rng, 1, 512)
    most = MOST_STATES * 0.8 / (T * H)
    if A:
        most = min(most, MOST_PRODUCTS * 0.8 / (T * H * A), MOST_STATES * 1.6 / (T * A))
    B = max(1, min(B, int(most)))
    shortest = 0 if T == 1 or rng.random() < 0.2 else max(1, int(T * rng.uniform(0.1, 0.9)))
    case = _case("", call, dtype, B, T, H, A, shortest, rng.random() < 0.7)
    del case["name"]
    return case


def _type(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _states(gen, rows, H, dev):
    """Rows of a residual stream: normal values, the channels' sizes spread over a factor of four or so."""
    x = torch.randn((rows, H), generator=gen, device=dev)
    return x * torch.exp(0.5 * torch.randn((1, H), generator=gen, device=dev))


def _to_8_bits(x):
    """(int8 [rows, H], scale of each row): what the save call makes, for the calls that begin with such rows."""
    m = x.abs().amax(1).clamp(min=1e-30)
    return torch.round(x * (LEVELS / m)[:, None]).to(torch.int8), m / LEVELS


def _pitched(q):
    """Rows in 8 bits lie a multiple of 128 bytes apart, with zeros behind their H values."""
    H = q.shape[1]
    return torch.nn.functional.pad(q, (0, -H % 128)).contiguous()


def prepare(case, seed):
    dev = torch.device("cuda:0")
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed))
    rng = np.random.default_rng(seed)
    B, T, H, A, call, dtype = case["B"], case["T"], case["H"], case["A"], case["call"], _type(case)
    rows = B * T
    s = {"case": case, "rows": rows, "n": rows, "frames": None, "index": slice(None)}
    if case["shortest"]:
        # the list of a minibatch's frames, made once and used by every call of its step: their number, then the rows
        lengths = torch.from_numpy(rng.integers(case["shortest"], T + 1, B).astype(np.int32)).to(dev)
        valid = torch.nonzero((torch.arange(T, device=dev)[:, None] < lengths[None, :]).flatten()).flatten()
        s["n"], s["index"] = valid.numel(), valid
        s["frames"] = torch.zeros(1 + rows, dtype=torch.int32, device=dev)
        s["frames"][0] = valid.numel()
        s["frames"][1:1 + valid.numel()] = valid.to(torch.int32)
    counts = torch.zeros((rows, 1), dtype=torch.bool, device=dev)
    counts[s["index"]] = True
    pitch = H + -H % 128
    if call in ("save", "norm"):
        s["x"] = torch.where(counts, _states(gen, rows, H, dev), 0.0).to(dtype)
        s["q"] = torch.zeros((rows, pitch), dtype=torch.int8, device=dev)
        s["scales"] = torch.zeros(rows, device=dev)
        s["values"] = torch.zeros((rows, H), dtype=dtype, device=dev)
    if call in ("norm", "norm back"):
        s["weight"] = 1.0 + 0.2 * torch.randn(H, generator=gen, device=dev)
    if call == "norm":
        s["residual"] = torch.where(counts, _states(gen, rows, H, dev), 0.0).to(dtype) if case["residual"] else None
        s["sum"] = torch.zeros((rows, H), dtype=dtype, device=dev)
    if call == "norm back":
        s["sum"] = torch.where(counts, _states(gen, rows, H, dev), 0.0).to(dtype)
        s["dy"] = torch.where(counts, 1e-3 * torch.randn((rows, H), generator=gen, device=dev), 0.0).to(dtype)
        s["dresidual"] = (torch.where(counts, 1e-3 * torch.randn((rows, H), generator=gen, device=dev), 0.0).to(dtype)
                          if case["residual"] else None)
        s["dsum"] = torch.zeros((rows, H), dtype=dtype, device=dev)
        s["dweight"] = torch.zeros(H, device=dev)
    if call in ("product", "weights"):
        q, scales = _to_8_bits(torch.where(counts, _states(gen, rows, H, dev), 0.0))
        s["q"], s["scales"] = _pitched(q), scales
    if call == "product":
        q, scales = _to_8_bits(torch.randn((A, H), generator=gen, device=dev) / math.sqrt(H))
        s["weight_q"], s["weight_scales"] = _pitched(q), scales
        s["bias"] = 0.5 * torch.randn(A, generator=gen, device=dev)
        s["logits"] = torch.zeros((rows, A), dtype=dtype, device=dev)
    if call == "weights":
        g = torch.randn((rows, A), generator=gen, device=dev)
        g = torch.softmax(g if A > 2048 else 2.0 * g, 1)
        g[torch.arange(rows, device=dev), torch.randint(0, A, (rows,), generator=gen, device=dev)] -= 1.0
        s["grads"] = torch.where(counts, g, 0.0).to(dtype)
        s["dweight"] = torch.zeros((A, H), device=dev)
        s["dbias"] = torch.zeros(A, device=dev)
    if own:
        from paper_1512_02595_amd import layer
        size = (layer.rms_norm_workspace_size(rows, H) if call == "norm back" else
                layer.weight_gradient_workspace_size(rows, H, A) if call == "weights" else 0)
        s["workspace"] = torch.empty(size + 256, dtype=torch.uint8, device=dev)
        s["ws_ptr"], s["ws_bytes"] = (s["workspace"].data_ptr() + 255) // 256 * 256, size
    return s


def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    from paper_1512_02595_amd import ctc, layer
    c = s["case"]
    rows, H, A, call = s["rows"], c["H"], c["A"], c["call"]
    dtype = ctc.DTYPE_F32 if c["dtype"] == "f32" else ctc.DTYPE_BF16
    stream = torch.cuda.current_stream().cuda_stream
    frames = None if s["frames"] is None else s["frames"].data_ptr()
    if call == "save":
        layer.quantize_rows(s["x"].data_ptr(), frames, rows, H, dtype, s["q"].data_ptr(), s["scales"].data_ptr(), stream)
        layer.dequantize_rows(s["q"].data_ptr(), s["scales"].data_ptr(), frames, rows, H, dtype, s["values"].data_ptr(), stream)
        return {"values": s["values"]}
    if call == "norm":
        residual = None if s["residual"] is None else s["residual"].data_ptr()
        layer.rms_norm_i8(s["x"].data_ptr(), residual, s["weight"].data_ptr(), EPS, frames, rows, H, dtype,
                          s["sum"].data_ptr(), s["q"].data_ptr(), s["scales"].data_ptr(), stream)
        layer.dequantize_rows(s["q"].data_ptr(), s["scales"].data_ptr(), frames, rows, H, dtype, s["values"].data_ptr(), stream)
        return {"sum": s["sum"], "values": s["values"]}
    if call == "norm back":
        dresidual = None if s["dresidual"] is None else s["dresidual"].data_ptr()
        layer.rms_norm_backward(s["dy"].data_ptr(), s["sum"].data_ptr(), s["weight"].data_ptr(), EPS, dresidual, frames,
                                rows, H, dtype, s["dsum"].data_ptr(), s["dweight"].data_ptr(), s["ws_ptr"], s["ws_bytes"], stream)
        return {"dsum": s["dsum"], "dweight": s["dweight"]}
    if call == "product":
        layer.linear_i8(s["q"].data_ptr(), s["scales"].data_ptr(), s["weight_q"].data_ptr(), s["weight_scales"].data_ptr(),
                        s["bias"].data_ptr(), frames, rows, H, A, dtype, s["logits"].data_ptr(), stream)
        return {"logits": s["logits"]}
    layer.weight_gradient_i8(s["grads"].data_ptr(), s["q"].data_ptr(), s["scales"].data_ptr(), frames, rows, H, A, dtype,
                             s["dweight"].data_ptr(), s["dbias"].data_ptr(), s["ws_ptr"], s["ws_bytes"], stream)
    return {"dweight": s["dweight"], "dbias": s["dbias"]}


def _whole(s, rows, width):
    """The listed rows in a tensor of all rows; the others hold zeros."""
    if s["frames"] is None:
        return rows
    out = torch.zeros((s["rows"], width), dtype=rows.dtype, device=rows.device)
    out[s["index"]] = rows
    return out


def _rounded(u):
    """Rows as 8 bits hold them: (whole numbers, the largest value of each row).  In 64 bits: which of two whole numbers
    is the nearer is a matter of the last bits."""
    m = u.abs().amax(1, keepdim=True)
    q = torch.round(u.double() * LEVELS / m.double())
    return torch.where(m > 0, q, 0.0).float(), m


def _plain(s):
    c = s["case"]
    H, call, dtype, index = c["H"], c["call"], _type(c), s["index"]
    if call == "save":
        q, m = _rounded(s["x"][index].float())
        return {"values": _whole(s, (q * (m / LEVELS)).to(dtype), H)}
    if call == "norm":
        z = s["x"][index].float()
        if s["residual"] is not None:
            z = (z + s["residual"][index].float()).to(dtype).float()
        r = torch.rsqrt((z * z).mean(1, keepdim=True) + EPS)
        q, m = _rounded(z * s["weight"])
        return {"sum": _whole(s, z.to(dtype), H), "values": _whole(s, (q * (m * r / LEVELS)).to(dtype), H)}
    if call == "norm back":
        z, dy = s["sum"][index].float(), s["dy"][index].float()
        r = torch.rsqrt((z * z).mean(1, keepdim=True) + EPS)
        n, g = z * r, dy * s["weight"]
        dz = r * (g - n * (g * n).mean(1, keepdim=True))
        if s["dresidual"] is not None:
            dz = dz + s["dresidual"][index].float()
        return {"dsum": _whole(s, dz.to(dtype), H), "dweight": (dy * n).sum(0)}
    y = s["q"][index, :H].float() * s["scales"][index, None]
    if call == "product":
        w = s["weight_q"][:, :H].float() * s["weight_scales"][:, None]
        return {"logits": _whole(s, (torch.matmul(y, w.t()) + s["bias"]).to(dtype), c["A"])}
    g = s["grads"][index].float()
    return {"dweight": torch.matmul(g.t(), y), "dbias": g.sum(0)}


def work(case):
    """Every listed row of the inputs read once, every listed row of the outputs written once (what is read back for
    comparison included); the formulas' additions and products."""
    B, T, H, A, call = case["B"], case["T"], case["H"], case["A"], case["call"]
    e = 4 if case["dtype"] == "f32" else 2
    n = B * (case["shortest"] + T) / 2 if case["shortest"] else B * T
    extra = 1 if case["residual"] else 0
    if call == "save":
        return {"bytes": n * (H * 2 * (e + 1) + 8), "flops": 5 * n * H}
    if call == "norm":
        return {"bytes": n * (H * ((3 + extra) * e + 2) + 8) + 4 * H, "flops": 9 * n * H}
    if call == "norm back":
        return {"bytes": n * H * (3 + extra) * e + 8 * H, "flops": 12 * n * H}
    if call == "product":
        return {"bytes": n * (H + 4) + A * (H + 8) + n * A * e, "flops": 2 * n * A * H}
    return {"bytes": n * (H + 4 + A * e) + 4 * A * (H + 1), "flops": 2 * n * A * H}


def exact(case, seed):
    """The definitions in 64 bits, rows as blocks.  What is defined as rounded on the way is: the sum that the norm
    stores, its 32-bit product with the weight that is held in 8 bits, and the whole numbers themselves."""
    s = prepare(case, seed)
    H, A, call, rows = case["H"], case["A"], case["call"], s["rows"]
    dev = torch.device("cuda:0")
    keep = torch.ones(rows, dtype=torch.bool, device=dev)
    if s["frames"] is not None:
        keep = torch.zeros(rows, dtype=torch.bool, device=dev)
        keep[s["frames"][1:1 + int(s["frames"][0])].long()] = True
    step = max(1, 60_000_000 // max(H, A))
    blocks = [slice(i, min(i + step, rows)) for i in range(0, rows, step)]

    def held(u, scale_by):
        m = u.abs().max(dim=1).values[:, None]
        whole = torch.where(m > 0, torch.round(127.0 * u / torch.where(m > 0, m, 1.0)), 0.0)
        return whole * m / 127.0 * scale_by

    if call == "save":
        values = [torch.where(keep[b, None], held(s["x"][b].double(), 1.0), 0.0) for b in blocks]
        return {"values": torch.cat(values)}
    if call == "norm":
        sums, values = [], []
        for b in blocks:
            z = s["x"][b].double()
            if s["residual"] is not None:
                z = (z + s["residual"][b].double()).to(_type(case)).double()
            u = (z * s["weight"].double()).float().double()
            r = 1.0 / torch.sqrt(torch.sum(z * z, dim=1) / H + EPS)
            sums.append(z)
            values.append(torch.where(keep[b, None], held(u, r[:, None]), 0.0))
        return {"sum": torch.cat(sums), "values": torch.cat(values)}
    if call == "norm back":
        w, dw, dz = s["weight"].double(), torch.zeros(H, dtype=torch.float64, device=dev), []
        for b in blocks:
            z, dy = s["sum"][b].double(), torch.where(keep[b, None], s["dy"][b].double(), 0.0)
            v = torch.sum(z * z, dim=1)[:, None] / H + EPS
            # y = z w v^(-1/2):  dL/dz = dy w v^(-1/2) - z v^(-3/2) sum(dy w z) / H
            d = dy * w / v.sqrt() - z * torch.sum(dy * w * z, dim=1)[:, None] / (H * v * v.sqrt())
            if s["dresidual"] is not None:
                d += s["dresidual"][b].double()
            dz.append(torch.where(keep[b, None], d, 0.0))
            dw += torch.sum(dy * z / v.sqrt(), dim=0)
        return {"dsum": torch.cat(dz), "dweight": dw}
    if call == "product":
        w = (s["weight_q"][:, :H].double() * s["weight_scales"].double()[:, None]).t().contiguous()
        out = torch.zeros((rows, A), dtype=torch.float64, device=dev)
        for b in blocks:
            y = s["q"][b, :H].double() * s["scales"][b].double()[:, None]
            out[b] = torch.where(keep[b, None], y @ w + s["bias"].double(), 0.0)
        return {"logits": out}
    dw, db = torch.zeros((A, H), dtype=torch.float64, device=dev), torch.zeros(A, dtype=torch.float64, device=dev)
    for b in blocks:
        g = torch.where(keep[b, None], s["grads"][b].double(), 0.0)
        y = s["q"][b, :H].double() * s["scales"][b].double()[:, None]
        dw += g.t().contiguous() @ y
        db += g.sum(dim=0)
    return {"dweight": dw, "dbias": db}
