"""What the recurrent block's calls refuse, found on the host before anything is enqueued (no GPU is touched: the addresses
are made up)."""
import os
import re

import pytest

from paper_1512_02595_amd import block, ctc

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F32, BF16 = ctc.DTYPE_F32, ctc.DTYPE_BF16
INVALID, SMALL, UNSUPPORTED = ctc.STATUS_INVALID_VALUE, ctc.STATUS_WORKSPACE_TOO_SMALL, ctc.STATUS_UNSUPPORTED
GIB = 1 << 30


def address(i):
    """Made-up buffers a GiB apart."""
    return (i + 1) * GIB


# name: (arguments of a call that would be taken, by name, in order)
CALLS = {
    "recurrence": dict(inputs=address(0), input_pitch=300, input_lengths=address(1), initial=address(2), T=500, B=4, H=100,
                       forward_channels=50, dtype=F32, states=address(3), final=address(4), workspace=address(5),
                       workspace_bytes=1 << 29),
    "recurrence_backward": dict(dstates=address(0), dfinal=address(1), inputs=address(2), input_pitch=300, states=address(3),
                                input_lengths=address(4), initial=address(5), T=500, B=4, H=100, forward_channels=50, dtype=F32,
                                dinputs=address(6), dinitial=address(7), workspace=address(8), workspace_bytes=1 << 29),
    "block_norm": dict(x=address(0), gate=address(1), gate_pitch=300, residual=address(2), weight_after=address(3),
                       scale=address(4), weight_before=address(5), eps=1e-6, frames=address(6), rows=200, H=100, dtype=F32,
                       sum=address(7), normed=address(8)),
    "block_norm_backward": dict(dnormed=address(0), dsum=address(1), x=address(2), gate=address(3), gate_pitch=300, sum=address(4),
                                weight_after=address(5), scale=address(6), weight_before=address(7), eps=1e-6, frames=address(8),
                                rows=200, H=100, dtype=F32, dx=address(9), dgate=address(10), dresidual=address(11),
                                dweight_after=address(12), dscale=address(13), dweight_before=address(14), workspace=address(15),
                                workspace_bytes=1 << 29),
    "clear_frames": dict(x=address(0), pitch=100, input_lengths=address(1), T=500, B=4, width=80, dtype=F32),
    "quantize_weights_i4": dict(weights=address(0), A=29, H=300, group=128, dtype=F32, weight_q=address(1), weight_scales=address(2)),
    "dequantize_weights_i4": dict(weight_q=address(0), weight_scales=address(1), A=29, H=300, group=128, dtype=F32, out=address(2)),
    "linear_i4": dict(q=address(0), scales=address(1), weight_q=address(2), weight_scales=address(3), group=128, bias=address(4),
                      frames=address(5), rows=200, H=300, A=29, dtype=F32, logits=address(6)),
}
MAY_BE_NULL = {"recurrence": {"input_lengths", "initial", "final"},
               "recurrence_backward": {"dfinal", "input_lengths", "initial", "dinitial"},
               "block_norm": {"residual", "weight_after", "scale", "weight_before", "frames", "sum", "normed", "gate"},
               "block_norm_backward": {"dnormed", "dsum", "weight_after", "scale", "weight_before", "frames", "dresidual", "dweight_after",
                                       "dscale", "dweight_before"},
               "linear_i4": {"bias", "frames"}}
OUTPUTS = {"recurrence": {"states", "final", "workspace"}, "recurrence_backward": {"dinputs", "dinitial", "workspace"},
           "block_norm": {"sum", "normed"},
           "block_norm_backward": {"dx", "dgate", "dresidual", "dweight_after", "dscale", "dweight_before", "workspace"},
           "clear_frames": {"x"}, "quantize_weights_i4": {"weight_q", "weight_scales"}, "dequantize_weights_i4": {"out"}, "linear_i4": {"logits"}}
# outputs that may lie where an input does
MAY_BE = {("recurrence", "final"): {"initial"}, ("recurrence_backward", "dinitial"): {"dfinal"},
          ("block_norm", "sum"): {"x", "residual"}, ("block_norm", "normed"): {"x", "residual"},
          ("block_norm_backward", "dx"): {"x", "sum", "dnormed", "dsum"}, ("block_norm_backward", "dresidual"): {"x", "sum", "dnormed", "dsum"}}


def status(name, **changed):
    args = dict(CALLS[name])
    assert set(changed) <= set(args)
    args.update(changed)
    return getattr(block, name + "_status")(*args.values())


def buffers(name):
    return [k for k, v in CALLS[name].items() if isinstance(v, int) and v >= GIB]


def test_every_declared_symbol_is_exported():
    text = open(os.path.join(ROOT, "include", "ctc_block.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = set(re.findall(r"\b(ctc_[a-z_0-9]+)\s*\(", text))
    assert names == set(block.EXPORTS)
    lib = block.load()
    for n in names:
        assert getattr(lib, n) is not None


@pytest.mark.parametrize("name", CALLS)
def test_null_and_misaligned_buffers(name):
    for k in buffers(name):
        if k not in MAY_BE_NULL.get(name, ()):
            assert status(name, **{k: None}) == INVALID, k
        assert status(name, **{k: CALLS[name][k] + 1}) == INVALID, k
    for k in {"q", "weight_q", "weight_scales"} & set(CALLS[name]):
        assert status(name, **{k: CALLS[name][k] + 8}) == INVALID, k
    if "workspace" in CALLS[name]:
        assert status(name, workspace=CALLS[name]["workspace"] + 128) == INVALID


@pytest.mark.parametrize("name", CALLS)
def test_outputs_that_overlap_other_buffers(name):
    for out in OUTPUTS[name]:
        for k in buffers(name):
            if k == out:
                continue
            here = CALLS[name][k]
            if k not in MAY_BE.get((name, out), ()):
                assert status(name, **{out: here}) == INVALID, (out, k)
            if out != "workspace" or k not in OUTPUTS[name]:
                assert status(name, **{out: here - 256}) == INVALID, (out, k, "from below")


@pytest.mark.parametrize("name", CALLS)
def test_sizes_and_types(name):
    for k, v in CALLS[name].items():
        if k in ("T", "B", "rows", "H", "A"):
            for bad in (0, -1, -2 ** 31):
                assert status(name, **{k: bad}) == INVALID, k
        if k == "H":
            assert status(name, H=16385, **{p: 1 << 20 for p in ("input_pitch", "gate_pitch") if p in CALLS[name]}) == UNSUPPORTED
        if k in ("input_pitch", "gate_pitch"):
            least = 200 if k == "input_pitch" else 100
            for bad in (0, -1, least - 1):
                assert status(name, **{k: bad}) == INVALID
            assert status(name, **{k: (1 << 20) + 1}) == UNSUPPORTED
        if k == "dtype":
            assert status(name, dtype=2) == INVALID and status(name, dtype=-1) == INVALID
        if k == "eps":
            for bad in (0.0, -1e-6, float("nan"), float("inf")):
                assert status(name, eps=bad) == INVALID
        if k == "group":
            for bad in (0, -64, 32, 63, 65, 96, 192, 320, 16384 + 128):
                assert status(name, group=bad) == INVALID
        if k == "forward_channels":
            assert status(name, forward_channels=-1) == INVALID and status(name, forward_channels=101) == INVALID
        if k == "workspace_bytes" and name == "block_norm_backward":
            assert status(name, workspace_bytes=block.block_norm_workspace_size(200, 100) - 1) == SMALL
        elif k == "workspace_bytes":
            assert status(name, workspace_bytes=block.recurrence_workspace_size(500, 4, 100) - 1) == SMALL
    if "B" in CALLS[name]:
        assert status(name, B=65536) == UNSUPPORTED
        assert status(name, T=1 << 20, B=1 << 11) == UNSUPPORTED
    if "A" in CALLS[name]:
        assert status(name, A=(1 << 20) + 1) == UNSUPPORTED
    if "rows" in CALLS[name]:
        assert status(name, rows=(1 << 30) + 1) == UNSUPPORTED


def test_columns_that_are_cleared():
    for bad in (0, -1, 101):
        assert status("clear_frames", width=bad) == INVALID
    for bad in (0, -1, 79):
        assert status("clear_frames", pitch=bad) == INVALID
    assert status("clear_frames", pitch=(1 << 20) + 1) == UNSUPPORTED
    assert status("clear_frames", pitch=(1 << 20) + 1, width=(1 << 20) + 1) == UNSUPPORTED


def test_buffers_that_are_needed_together():
    assert status("block_norm", sum=None, normed=None) == INVALID
    assert status("block_norm_backward", dnormed=None, dsum=None) == INVALID
    assert status("block_norm_backward", sum=None) == INVALID
    assert status("block_norm_backward", gate=None) == INVALID
    assert status("block_norm_backward", dgate=None) == INVALID
    assert status("block_norm_backward", dx=CALLS["block_norm_backward"]["x"], dresidual=CALLS["block_norm_backward"]["x"]) == INVALID


def test_sizes_are_told_and_refused():
    assert block.weights_i4_sizes(29, 300, 128) == (2 * 3 * 1024, 2 * 3 * 64)
    assert block.weights_i4_sizes(16, 64, 64) == (1024, 64)
    assert block.weights_i4_sizes(17, 65, 64) == (2048, 2 * 2 * 64)
    for bad in ((0, 1, 64), (1, 0, 64), (1, 1, 63), (1, 1, 192)):
        assert block.weights_i4_sizes_status(*bad)[0] == INVALID
    assert block.weights_i4_sizes_status(1, 16385, 64)[0] == UNSUPPORTED
    for bad in ((0, 1, 1), (1, 0, 1), (1, 1, 0)):
        assert block.recurrence_workspace_size_status(*bad)[0] == INVALID
    for bad in ((1, 65536, 1), (1, 1, 16385), (1 << 20, 1 << 11, 1)):
        assert block.recurrence_workspace_size_status(*bad)[0] == UNSUPPORTED
    assert block.block_norm_workspace_size_status(0, 1)[0] == INVALID
    assert block.block_norm_workspace_size_status(1, 16385)[0] == UNSUPPORTED
    with pytest.raises(OverflowError):
        block.recurrence_workspace_size(2 ** 32 + 1, 1, 1)
    with pytest.raises(ctc.CTCError):
        block.block_norm(None, None, 0, None, None, None, None, 1e-6, None, 1, 1, F32, None, None)


def test_workspaces_never_shrink():
    for size, args in ((block.recurrence_workspace_size, [(1, 2, 100, 128, 129, 256, 257, 1000, 40000, 1 << 20),
                                                          (1, 2, 3, 4, 7, 8, 30, 31, 64, 512, 1000), (1, 64, 128, 129, 1000, 1999, 4096, 16384)]),):
        Ts, Bs, Hs = args
        for T in Ts:
            for B in Bs:
                for H in Hs:
                    here = size(T, B, H)
                    for T2, B2, H2 in ((2 * T, B, H), (T + 1, B, H), (T, B + 1, H), (T, 2 * B, H), (T, B, min(2 * H, 16384)), (T, B, min(H + 1, 16384))):
                        if T2 * B2 <= 1 << 30:
                            assert T * B > 1 << 30 or size(T2, B2, H2) >= here, (T, B, H, T2, B2, H2)
    for H in (1, 512, 513, 1024, 1025, 16384):
        sizes = [block.block_norm_workspace_size(rows, H) for rows in list(range(1, 3000)) + [4096, 5000, 1 << 20, 1 << 30]]
        assert sizes == sorted(sizes)
