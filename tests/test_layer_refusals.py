"""What the output layer's calls refuse, found on the host before anything is enqueued (no GPU is touched: the addresses
are made up)."""
import ctypes
import os
import re

import pytest

from paper_1512_02595_amd import ctc, layer

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F32, BF16 = ctc.DTYPE_F32, ctc.DTYPE_BF16
INVALID, SMALL, UNSUPPORTED = ctc.STATUS_INVALID_VALUE, ctc.STATUS_WORKSPACE_TOO_SMALL, ctc.STATUS_UNSUPPORTED


def address(i):
    """Made-up buffers a GiB apart."""
    return (i + 1) << 30


# name: (arguments of a call that would be taken, by name, in order)
CALLS = {
    "pack_frames": dict(input_lengths=address(0), T=50, B=4, frames=address(1)),
    "quantize_rows": dict(x=address(0), frames=address(1), rows=200, H=100, dtype=F32, q=address(2), scales=address(3)),
    "dequantize_rows": dict(q=address(0), scales=address(1), frames=address(2), rows=200, H=100, dtype=F32, out=address(3)),
    "rms_norm_i8": dict(x=address(0), residual=address(1), weight=address(2), eps=1e-6, frames=address(3), rows=200, H=100,
                        dtype=F32, sum=address(4), q=address(5), scales=address(6)),
    "rms_norm_backward": dict(dy=address(0), sum=address(1), weight=address(2), eps=1e-6, dresidual=address(3),
                              frames=address(4), rows=200, H=100, dtype=F32, dsum=address(5), dweight=address(6),
                              workspace=address(7), workspace_bytes=1 << 29),
    "linear_i8": dict(q=address(0), scales=address(1), weight_q=address(2), weight_scales=address(3), bias=address(4),
                      frames=address(5), rows=200, H=100, A=29, dtype=F32, logits=address(6)),
    "weight_gradient_i8": dict(grads=address(0), q=address(1), scales=address(2), frames=address(3), rows=200, H=100, A=29,
                               dtype=F32, dweight=address(4), dbias=address(5), workspace=address(6),
                               workspace_bytes=1 << 29),
}
MAY_BE_NULL = {"frames", "residual", "weight", "bias", "dresidual", "dbias", "sum"}
OUTPUTS = {"frames", "q", "scales", "out", "sum", "dsum", "dweight", "dbias", "logits", "workspace"}


def status(name, **changed):
    args = dict(CALLS[name])
    assert set(changed) <= set(args)
    args.update(changed)
    return getattr(layer, name + "_status")(*args.values())


def buffers(name):
    return [k for k, v in CALLS[name].items() if isinstance(v, int) and v >= address(0)]


def test_every_declared_symbol_is_exported():
    text = open(os.path.join(ROOT, "include", "ctc_layer.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = set(re.findall(r"\b(ctc_[a-z_0-9]+)\s*\(", text))
    assert names == set(layer.EXPORTS)
    lib = layer.load()
    for n in names:
        assert getattr(lib, n) is not None
    assert layer.last_hip_error() == 0


@pytest.mark.parametrize("H, pitch", [(1, 128), (127, 128), (128, 128), (129, 256), (2048, 2048), (16384, 16384),
                                      (0, 0), (-5, 0), (16385, 0)])
def test_row_pitch(H, pitch):
    assert layer.row_pitch(H) == pitch


@pytest.mark.parametrize("name, what", [(n, k) for n in CALLS for k in buffers(n)])
def test_null_pointers(name, what):
    # "sum" is the norm's optional output and its gradient's required input; a call without dweight needs no workspace
    allowed = what in MAY_BE_NULL and (name, what) not in {("rms_norm_backward", "sum"), ("pack_frames", "frames")}
    allowed = allowed or (name, what) == ("rms_norm_backward", "dweight")
    if not allowed:
        assert status(name, **{what: None}) == INVALID
        assert status(name, **{what: 0}) == INVALID


@pytest.mark.parametrize("name, what", [(n, k) for n in CALLS for k in buffers(n)])
def test_misaligned_pointers(name, what):
    at = CALLS[name][what]
    assert status(name, **{what: at + 1}) == INVALID
    if what in ("q", "weight_q"):
        assert status(name, **{what: at + 8}) == INVALID
    if what == "workspace":
        assert status(name, **{what: at + 128}) == INVALID


@pytest.mark.parametrize("name", [n for n in CALLS if "rows" in CALLS[n]])
def test_sizes(name):
    for what in ("rows", "H", "A"):
        if what in CALLS[name]:
            assert status(name, **{what: 0}) == INVALID
            assert status(name, **{what: -1}) == INVALID
    assert status(name, H=16385) == UNSUPPORTED
    assert status(name, rows=(1 << 30) + 1) == UNSUPPORTED
    if "A" in CALLS[name]:
        assert status(name, A=(1 << 20) + 1) == UNSUPPORTED
    for dtype in (-1, 2, 77):
        assert status(name, dtype=dtype) == INVALID


def test_pack_frames_sizes():
    assert status("pack_frames", T=0) == INVALID
    assert status("pack_frames", B=0) == INVALID
    assert status("pack_frames", B=65536) == UNSUPPORTED
    assert status("pack_frames", T=1 << 30, B=2) == UNSUPPORTED


@pytest.mark.parametrize("name, a, b", [(n, a, b) for n in CALLS for a in buffers(n) for b in buffers(n)
                                        if a != b and a in OUTPUTS])
def test_overlapping_buffers(name, a, b):
    """An output may not overlap another buffer: neither by its first element nor begin at the same place."""
    inputs = {"dequantize_rows": {"q", "scales", "frames"}, "linear_i8": {"q", "scales", "frames"},
              "weight_gradient_i8": {"q", "scales", "frames"}, "rms_norm_backward": {"sum", "frames"},
              "rms_norm_i8": {"frames"}, "quantize_rows": {"frames"}}.get(name, set())
    if a in inputs:                                      # (two inputs may be one)
        return
    same = {("rms_norm_i8", "sum"): {"x", "residual"}, ("rms_norm_backward", "dsum"): {"dy", "sum", "dresidual"}}
    step = 256                                           # keeps every alignment
    if b not in same.get((name, a), set()):
        assert status(name, **{a: CALLS[name][b]}) == INVALID
    if name == "pack_frames":
        return
    if b not in ("weight", "bias", "weight_scales", "dweight", "dbias", "workspace") or (name, b) == ("weight_gradient_i8", "dweight"):
        assert status(name, **{a: CALLS[name][b] + step}) == INVALID


@pytest.mark.parametrize("name", ["rms_norm_i8", "rms_norm_backward"])
@pytest.mark.parametrize("eps", [0.0, -1e-6, float("inf"), float("nan"), 1e-60])
def test_eps(name, eps):
    assert status(name, eps=eps) == INVALID              # (1e-60 is 0 as a float)


def test_workspace():
    for name, needed in (("rms_norm_backward", layer.rms_norm_workspace_size(200, 100)),
                         ("weight_gradient_i8", layer.weight_gradient_workspace_size(200, 100, 29))):
        assert needed > 0 and needed % 256 == 0
        assert status(name, workspace_bytes=needed - 1) == SMALL
        assert status(name, workspace_bytes=0) == SMALL
    assert layer.rms_norm_workspace_size_status(0, 100)[0] == INVALID
    assert layer.rms_norm_workspace_size_status(1, 16385)[0] == UNSUPPORTED
    assert layer.weight_gradient_workspace_size_status(1, 1, 0)[0] == INVALID
    assert layer.weight_gradient_workspace_size_status(1, 1, (1 << 20) + 1)[0] == UNSUPPORTED
    assert layer.load().ctc_rms_norm_workspace_size(1, 1, None) == INVALID
    assert layer.load().ctc_weight_gradient_workspace_size(1, 1, 1, None) == INVALID
    with pytest.raises(ctc.CTCError):
        layer.weight_gradient_workspace_size(0, 1, 1)


def test_the_largest_sizes_are_counted_in_64_bits():
    for H, A in ((16384, 1 << 20), (16384, 4000), (16384, 64), (1, 1)):
        assert layer.weight_gradient_workspace_size(1 << 30, H, A) % 256 == 0
    assert layer.weight_gradient_workspace_size(1 << 30, 16384, 4000) >= (1 << 30) * 16384 * 2    # the rows, in 16 bits
    assert layer.rms_norm_workspace_size(1 << 30, 16384) >= 16384 * 4


def test_binding_refuses_what_is_no_argument():
    from paper_1512_02595_amd import _layer_binding
    layer.load()
    with pytest.raises(TypeError):
        _layer_binding.quantize_rows(1, 2)
    with pytest.raises(TypeError):
        _layer_binding.bind(1)
    with pytest.raises(TypeError):
        status("quantize_rows", H=10.5)
    with pytest.raises(TypeError):
        status("quantize_rows", x="here")
    with pytest.raises(OverflowError):
        status("quantize_rows", rows=1 << 40)
    with pytest.raises(OverflowError):
        status("weight_gradient_i8", workspace_bytes=-1)
    with pytest.raises(ctc.CTCError, match="ctc_quantize_rows"):
        layer.quantize_rows(*dict(CALLS["quantize_rows"], H=0).values())
    assert ctypes.sizeof(ctypes.c_void_p) == 8
