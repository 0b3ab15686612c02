"""Zeros behind the utterances' ends: which elements are cleared, and that no other is touched."""
import numpy as np
import pytest
import torch

from layer_reference import Guarded, PATTERN, stream, torch_type
from paper_1512_02595_amd import block, ctc

pytestmark = pytest.mark.gpu
F32, BF16 = ctc.DTYPE_F32, ctc.DTYPE_BF16


def some_lengths(T, B, kind):
    rng = np.random.default_rng([T, B])
    n = rng.integers(0, T + 1, B)
    if kind == "beyond":                                # below 0 counts as 0, above T as T
        n = np.where(rng.random(B) < 0.5, -(2 ** 31), 2 ** 31 - 1)
    if kind == "all":
        n[:] = T
    return n.astype(np.int32)


def clear(x, n, T, B, pitch, width, dtype):
    lengths = torch.from_numpy(n).cuda()
    block.clear_frames(x.t.data_ptr(), pitch, lengths.data_ptr(), T, B, width, dtype, stream())
    torch.cuda.synchronize()


def check(x, n, T, B, pitch, width, size):
    data = x.raw[x.span[0]:x.span[1]]
    want = torch.full((T * B * pitch * size,), PATTERN, dtype=torch.uint8).view(T, B, pitch * size)
    behind = torch.arange(T)[:, None] >= torch.from_numpy(np.clip(n, 0, T).astype(np.int64))[None]
    want[:, :, :width * size][behind] = 0
    assert torch.equal(data.cpu(), want.flatten()[:data.numel()]) and x.intact()


@pytest.mark.parametrize("kind", ["some", "beyond", "all"])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T, B, width, more, shift", [(1, 1, 1, 0, 0), (1, 5, 3, 0, 0), (15, 3, 7, 2, 4), (16, 2, 8, 0, 0), (17, 4, 9, 0, 8), (40, 3, 1001, 0, 4),
                                                      (33, 70, 64, 128, 0), (100, 2, 4097, 3, 12), (3000, 1, 5, 1, 0), (7, 300, 130, 0, 0), (2, 1, 1 << 20, 0, 0)])
def test_rows_behind_the_ends(T, B, width, more, shift, dtype, kind):
    print("clear", T, B, width, more, shift, dtype, kind, flush=True)
    pitch, size = width + more, 4 if dtype == F32 else 2
    x, n = Guarded((T * B, pitch), torch_type(dtype), shift), some_lengths(T, B, kind)
    clear(x, n, T, B, pitch, width, dtype)
    check(x, n, T, B, pitch, width, size)


def test_columns_of_wider_rows():
    """Some columns of a matrix, whose last row ends with them."""
    print("columns", flush=True)
    T, B, pitch, width = 50, 6, 300, 100
    x = torch.ones(T, B, pitch, device="cuda")
    n = torch.tensor([50, 0, 10, 49, 1, 33], dtype=torch.int32, device="cuda")
    block.clear_frames(x.data_ptr() + 4 * 200, pitch, n.data_ptr(), T, B, width, F32, stream())
    want = torch.ones(T, B, pitch)
    for b, m in enumerate(n.tolist()):
        want[m:, b, 200:] = 0
    assert torch.equal(x.cpu(), want)


def test_beyond_2_31_bytes_and_replayed():
    """Offsets that pass 2^31 elements; a captured call reads the lengths afresh."""
    print("beyond", flush=True)
    T, B, width = 1100, 2, 1 << 20
    x = torch.ones(T, B, width, dtype=torch.bfloat16, device="cuda")
    n = torch.tensor([1099, 1100], dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block.clear_frames(x.data_ptr(), width, n.data_ptr(), T, B, width, BF16, stream())
    for a, b in ((1099, 1100), (1100, 1098), (1099, 1099)):
        n.copy_(torch.tensor([a, b]))
        x.fill_(1)
        graph.replay()
        torch.cuda.synchronize()
        assert float(x[:a, 0].min()) == 1 and float(x[:b, 1].min()) == 1
        assert not x[a:, 0].any() and not x[b:, 1].any()
