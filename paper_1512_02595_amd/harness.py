"""Torch-side plumbing around the binding: device buffers, streams, result download.

PyTorch is used for device memory and streams only; every step of the CTC path runs
in the HIP library.  Used by the GPU tests, the smoke check and the benchmark.
"""
from __future__ import annotations

import contextlib

import numpy as np
import torch

from . import ctc, layer, workloads


def require_gpu() -> torch.device:
    if not torch.cuda.is_available():
        raise RuntimeError("a HIP device is required: the CTC path has no CPU fallback")
    return torch.device("cuda:0")


class DeviceBatch:
    """A CTCBatch with its activations resident in HBM plus output and workspace buffers."""

    def __init__(self, batch: workloads.CTCBatch, dtype: int = ctc.DTYPE_F32, device=None,
                 poison: bool = True):
        self.device = device or require_gpu()
        self.batch = batch
        self.dtype = dtype
        if dtype == ctc.DTYPE_F32:
            host = torch.from_numpy(np.ascontiguousarray(batch.logits, dtype=np.float32))
            self.x = host.to(self.device)
        else:
            bits = workloads.bf16_bits(batch.logits).view(np.int16)
            self.x = torch.from_numpy(bits).to(self.device).view(torch.bfloat16)
        self.grads = torch.empty_like(self.x)
        self.costs = torch.empty(batch.B, dtype=torch.float32, device=self.device)
        self.ws_bytes = ctc.workspace_size(batch.T, batch.B, batch.A, batch.label_lengths,
                                           batch.input_lengths, dtype)
        self.ws = torch.empty(self.ws_bytes + 256, dtype=torch.uint8, device=self.device)
        self.ws_ptr = (self.ws.data_ptr() + 255) // 256 * 256
        if poison:
            self.poison()

    def poison(self):
        """Fill outputs and workspace with NaN bit patterns so that stale data cannot pass."""
        self.ws.fill_(0xFF)
        self.grads.view(torch.uint8).fill_(0xFF)
        self.costs.fill_(float("nan"))

    def run(self, stream=None, kernel_ms=None):
        b = self.batch
        s = torch.cuda.current_stream(self.device).cuda_stream if stream is None else stream
        ctc.loss_and_grad(self.x.data_ptr(), b.flat_labels, b.label_lengths, b.input_lengths,
                          b.T, b.B, b.A, b.blank, self.dtype, self.costs.data_ptr(),
                          self.grads.data_ptr(), self.ws_ptr, self.ws_bytes, s, kernel_ms)

    def run_loss(self, stream=None, kernel_ms=None):
        """Costs only (grads == NULL)."""
        b = self.batch
        s = torch.cuda.current_stream(self.device).cuda_stream if stream is None else stream
        ctc.loss_and_grad(self.x.data_ptr(), b.flat_labels, b.label_lengths, b.input_lengths,
                          b.T, b.B, b.A, b.blank, self.dtype, self.costs.data_ptr(),
                          None, self.ws_ptr, self.ws_bytes, s, kernel_ms)

    def run_best_path(self, stream=None, kernel_ms=None):
        """Most probable alignment: scores go to self.costs, states to self.alignment [B,T]."""
        b = self.batch
        if getattr(self, "alignment", None) is None:
            self.alignment = torch.full((b.B, b.T), -7, dtype=torch.int32, device=self.device)
        s = torch.cuda.current_stream(self.device).cuda_stream if stream is None else stream
        ctc.best_path(self.x.data_ptr(), b.flat_labels, b.label_lengths, b.input_lengths,
                      b.T, b.B, b.A, b.blank, self.dtype, self.costs.data_ptr(),
                      self.alignment.data_ptr(), self.ws_ptr, self.ws_bytes, s, kernel_ms)

    def best_path_results(self):
        """(scores float32 [B], states int32 [B,T]) on the host, after synchronising."""
        torch.cuda.synchronize(self.device)
        return self.costs.cpu().numpy(), self.alignment.cpu().numpy()

    def results(self):
        """(costs float32 [B], grads float32 [T,B,A]) on the host, after synchronising."""
        torch.cuda.synchronize(self.device)
        costs = self.costs.cpu().numpy()
        if self.dtype == ctc.DTYPE_F32:
            grads = self.grads.cpu().numpy()
        else:
            grads = self.grads.float().cpu().numpy()
        return costs, grads


def run_batch(batch: workloads.CTCBatch, dtype: int = ctc.DTYPE_F32):
    db = DeviceBatch(batch, dtype)
    db.run()
    return db.results()


class DeviceMetaBatch:
    """Buffers for ctc_loss_and_grad_device: lengths and padded labels live on the GPU.

    Sized by bounds (T, B, A, max_label); `load` writes one CTCBatch of that shape into the
    same device buffers, so a recorded graph can be replayed on new contents.
    """

    def __init__(self, T, B, A, max_label, blank=0, dtype: int = ctc.DTYPE_F32, device=None):
        self.device = device or require_gpu()
        self.T, self.B, self.A, self.max_label, self.blank, self.dtype = T, B, A, max_label, blank, dtype
        tdtype = torch.float32 if dtype == ctc.DTYPE_F32 else torch.bfloat16
        self.x = torch.zeros((T, B, A), dtype=tdtype, device=self.device)
        self.grads = torch.empty_like(self.x)
        self.costs = torch.empty(B, dtype=torch.float32, device=self.device)
        self.labels = torch.zeros((B, max(max_label, 1)), dtype=torch.int32, device=self.device)
        self.label_lengths = torch.zeros(B, dtype=torch.int32, device=self.device)
        self.input_lengths = torch.zeros(B, dtype=torch.int32, device=self.device)
        self.status = torch.full((1,), -1, dtype=torch.int32, device=self.device)
        self.ws_bytes = ctc.workspace_size_device(T, B, A, max_label, dtype)
        self.ws = torch.empty(self.ws_bytes + 256, dtype=torch.uint8, device=self.device)
        self.ws_ptr = (self.ws.data_ptr() + 255) // 256 * 256

    def load(self, batch: workloads.CTCBatch, raw_labels=None):
        """Copies a batch into the device buffers (in place).  `raw_labels` [B, max_label] overrides
        the padded label matrix (to plant invalid entries)."""
        assert (batch.T, batch.B, batch.A) == (self.T, self.B, self.A)
        if self.dtype == ctc.DTYPE_F32:
            self.x.copy_(torch.from_numpy(np.ascontiguousarray(batch.logits, dtype=np.float32)))
        else:
            bits = workloads.bf16_bits(batch.logits).view(np.int16)
            self.x.copy_(torch.from_numpy(bits).view(torch.bfloat16))
        pad = np.zeros((self.B, max(self.max_label, 1)), dtype=np.int32)
        off = 0
        for b in range(self.B):
            L = int(batch.label_lengths[b])
            pad[b, :min(L, self.max_label)] = batch.flat_labels[off:off + L][:self.max_label]
            off += L
        if raw_labels is not None:
            pad = np.ascontiguousarray(raw_labels, dtype=np.int32)
        self.labels.copy_(torch.from_numpy(pad))
        self.label_lengths.copy_(torch.from_numpy(np.ascontiguousarray(batch.label_lengths, dtype=np.int32)))
        self.input_lengths.copy_(torch.from_numpy(np.ascontiguousarray(batch.input_lengths, dtype=np.int32)))

    def poison(self):
        self.ws.fill_(0xFF)
        self.grads.view(torch.uint8).fill_(0xFF)
        self.costs.fill_(float("nan"))
        self.status.fill_(-1)

    def run(self, stream=None, want_grad=True, kernel_ms=None):
        s = torch.cuda.current_stream(self.device).cuda_stream if stream is None else stream
        ctc.loss_and_grad_device(self.x.data_ptr(), self.labels.data_ptr(), self.label_lengths.data_ptr(),
                                 self.input_lengths.data_ptr(), self.max_label, self.T, self.B, self.A,
                                 self.blank, self.dtype, self.costs.data_ptr(),
                                 self.grads.data_ptr() if want_grad else None, self.status.data_ptr(),
                                 self.ws_ptr, self.ws_bytes, s, kernel_ms)

    def results(self):
        """(status int, costs float32 [B], grads float32 [T,B,A]) on the host, after synchronising."""
        torch.cuda.synchronize(self.device)
        return int(self.status.item()), self.costs.cpu().numpy(), self.grads.float().cpu().numpy()


class OutputLayer:
    """The layer that makes CTC's activations, with its states in 8 bits, over the buffers of a minibatch [T, B].

    `forward` takes the last layer's states and the residual stream to activations [T, B, A] (`logits`, which may be a
    DeviceBatch's or DeviceMetaBatch's `x`), `weight_gradient` takes CTC's gradient to the weights' and the bias's, from the rows that
    the forward pass left in 8 bits, and `norm_backward` the gradient of the norm's output to its input's.  Frames behind an
    utterance's end take no part.

    All of a call's work is on `stream` (a handle; None: torch's current one), whose owner keeps the tensors until it is done.
    """

    def __init__(self, T, B, H, A, dtype: int = ctc.DTYPE_F32, eps=1e-6, logits=None, device=None):
        self.device = device or require_gpu()
        self.T, self.B, self.H, self.A, self.dtype, self.eps, self.rows = T, B, H, A, dtype, eps, T * B
        tdtype = torch.float32 if dtype == ctc.DTYPE_F32 else torch.bfloat16

        def zeros(*shape, dtype=torch.float32):
            return torch.zeros(shape, dtype=dtype, device=self.device)

        pitch = layer.row_pitch(H)
        # (the number of rows, then their indices: all of them, until set_lengths says otherwise)
        self.frames = torch.cat((torch.tensor([self.rows], dtype=torch.int32, device=self.device),
                                 torch.arange(self.rows, dtype=torch.int32, device=self.device)))
        self.norm_weight, self.bias = torch.ones(H, device=self.device), zeros(A)
        self.weight_q, self.weight_scales = zeros(A, pitch, dtype=torch.int8), zeros(A)
        self.sum, self.dsum = zeros(T, B, H, dtype=tdtype), zeros(T, B, H, dtype=tdtype)
        self.q, self.scales = zeros(self.rows, pitch, dtype=torch.int8), zeros(self.rows)
        self.logits = zeros(T, B, A, dtype=tdtype) if logits is None else logits
        assert tuple(self.logits.shape) == (T, B, A) and self.logits.dtype == tdtype and self._here(self.logits)
        self.dweight, self.dbias, self.dnorm_weight = zeros(A, H), zeros(A), zeros(H)
        self.ws_bytes = layer.weight_gradient_workspace_size(self.rows, H, A), layer.rms_norm_workspace_size(self.rows, H)
        # (the two gradients need nothing of each other and may be on two streams: a workspace each)
        self.ws = [torch.empty(n + 256, dtype=torch.uint8, device=self.device) for n in self.ws_bytes]
        self.ws_ptr = [(w.data_ptr() + 255) // 256 * 256 for w in self.ws]

    def _stream(self, stream):
        return torch.cuda.current_stream(self.device).cuda_stream if stream is None else stream

    def _on(self, stream):
        """Where torch does its part of a call: on the call's stream."""
        s = self._stream(stream)
        if s == torch.cuda.current_stream(self.device).cuda_stream:
            return contextlib.nullcontext()
        return torch.cuda.stream(torch.cuda.ExternalStream(s, device=self.device))

    def _here(self, t):
        """Whether the library may be given the tensor's address."""
        return t.device == self.frames.device and t.is_contiguous()

    def _states(self, t):
        assert t.numel() == self.rows * self.H and t.dtype == self.sum.dtype and self._here(t)
        return t.data_ptr()

    def set_weights(self, weight, bias=None, norm_weight=None, stream=None):
        """fp32 weights [A, H] to 8 bits, and copies of the others: once per step of the optimiser."""
        assert tuple(weight.shape) == (self.A, self.H) and weight.dtype == torch.float32 and self._here(weight)
        layer.quantize_rows(weight.data_ptr(), None, self.A, self.H, ctc.DTYPE_F32, self.weight_q.data_ptr(),
                            self.weight_scales.data_ptr(), self._stream(stream))
        with self._on(stream):
            if bias is not None:
                self.bias.copy_(bias)
            if norm_weight is not None:
                self.norm_weight.copy_(norm_weight)

    def set_lengths(self, input_lengths, stream=None):
        """int32 [B] on the GPU: the frames of this minibatch, for all calls until the next one's (before the first: all)."""
        assert tuple(input_lengths.shape) == (self.B,) and input_lengths.dtype == torch.int32 and self._here(input_lengths)
        layer.pack_frames(input_lengths.data_ptr(), self.T, self.B, self.frames.data_ptr(), self._stream(stream))

    def forward(self, x, residual=None, stream=None):
        s = self._stream(stream)
        layer.rms_norm_i8(self._states(x), None if residual is None else self._states(residual), self.norm_weight.data_ptr(),
                          self.eps, self.frames.data_ptr(), self.rows, self.H, self.dtype, self.sum.data_ptr(), self.q.data_ptr(),
                          self.scales.data_ptr(), s)
        layer.linear_i8(self.q.data_ptr(), self.scales.data_ptr(), self.weight_q.data_ptr(), self.weight_scales.data_ptr(),
                        self.bias.data_ptr(), self.frames.data_ptr(), self.rows, self.H, self.A, self.dtype,
                        self.logits.data_ptr(), s)
        return self.logits

    def weight_gradient(self, grads, stream=None):
        assert tuple(grads.shape) == (self.T, self.B, self.A) and grads.dtype == self.logits.dtype and self._here(grads)
        layer.weight_gradient_i8(grads.data_ptr(), self.q.data_ptr(), self.scales.data_ptr(), self.frames.data_ptr(), self.rows,
                                 self.H, self.A, self.dtype, self.dweight.data_ptr(), self.dbias.data_ptr(), self.ws_ptr[0],
                                 self.ws_bytes[0], self._stream(stream))
        return self.dweight, self.dbias

    def norm_backward(self, dy, dresidual=None, stream=None):
        """(gradient of the norm's input [T, B, H], of its weight); frames behind an utterance's end get zeros, as in CTC's gradient."""
        given = [None if t is None else self._states(t) for t in (dy, dresidual)]
        with self._on(stream):
            # The library leaves such rows as they were, which may be the last minibatch's.  (A fill: 28900 of 48000 rows of 2048 fp32 133 us -> 225, bf16
            # 90 -> 118; which rows they are only the GPU knows.  An input in `dsum`'s own place is read afterwards.)
            if self.dsum.data_ptr() in given:
                aside = self.dsum.clone()
                given = [aside.data_ptr() if at == self.dsum.data_ptr() else at for at in given]
            self.dsum.zero_()
        layer.rms_norm_backward(given[0], self.sum.data_ptr(), self.norm_weight.data_ptr(), self.eps, given[1],
                                self.frames.data_ptr(), self.rows, self.H, self.dtype, self.dsum.data_ptr(),
                                self.dnorm_weight.data_ptr(), self.ws_ptr[1], self.ws_bytes[1], self._stream(stream))
        return self.dsum, self.dnorm_weight
