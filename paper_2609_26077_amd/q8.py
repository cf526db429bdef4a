"""An 8-bit linear layer over the C-ABI with torch-owned device buffers.

`RMSNormQ8` adds the residual, normalizes and writes int8 codes with a scale
per token (and an 8-bit checkpoint of the residual stream); `LinearQ8`
multiplies such codes by a weight's, with a scale per channel; both have the
backward pass, which reads the 8-bit checkpoints.  `quantize` makes the codes
of any matrix (a weight's rows are its output channels), `dequantize` the values
they stand for.

Codes are int8 [rows][pitch(cols)], zero past cols; scales are float32 [rows],
or [rows][pitch / 128] for a checkpoint.  Allocation, checks and marshalling
only: the arithmetic happens in the library's HIP kernels.  Every call runs on
`stream` (default: torch's current one) and allocates its outputs there; an
object's workspace is used by one call at a time.
"""
from __future__ import annotations

from contextlib import nullcontext
from typing import NamedTuple, Optional

import torch

from . import (FMM_BF16, FMM_F16, FMM_F32, fmm_norm_desc, fmm_q8_desc, fmm_q8_dequantize,
               fmm_q8_linear_backward, fmm_q8_linear_backward_scratch_size, fmm_q8_matmul,
               fmm_q8_matmul_scratch_size, fmm_q8_pitch, fmm_q8_quantize, fmm_rmsnorm_q8, fmm_rmsnorm_q8_backward,
               fmm_rmsnorm_q8_backward_scratch_size)
from .runner import _require

GROUP = 128
TYPES = {torch.float32: FMM_F32, torch.bfloat16: FMM_BF16, torch.float16: FMM_F16}


def pitch(cols: int) -> int:
    """Codes of one row: cols rounded up to 128."""
    return (cols + GROUP - 1) // GROUP * GROUP


def _type(dtype) -> int:
    t = TYPES.get(dtype)
    if t is None:
        raise ValueError(f"dtype {dtype}, expected float32, bfloat16 or float16")
    return t


def _device(device):
    d = torch.device(device)
    if d.type == "cuda" and d.index is None:
        d = torch.device("cuda", torch.cuda.current_device())
    return d


def _aligned(x, name, nbytes=16):
    """The kernels read these by 16-byte vectors."""
    if x.data_ptr() % nbytes:
        raise ValueError(f"{name}: not {nbytes}-byte aligned")


def _on(stream):
    """Outputs are allocated on the stream that writes them, so that torch's
    allocator reuses their memory in that stream's order."""
    if stream is None:
        return nullcontext()
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream)
    return torch.cuda.stream(stream)


def _matrix(x, name):
    if not isinstance(x, torch.Tensor):
        raise ValueError(f"{name}: expected a torch.Tensor, got {type(x).__name__}")
    if x.dim() != 2:
        raise ValueError(f"{name}: shape {tuple(x.shape)}, expected a matrix")


def quantize(x, codes=None, scales=None, stream=None):
    """(codes, scales) of the rows of x (float32, bfloat16 or float16)."""
    _matrix(x, "x")
    rows, cols = x.shape
    t = _type(x.dtype)
    _require(x, "x", (rows, cols), x.dtype, x.device)
    with torch.cuda.device(x.device), _on(stream):
        if codes is None:
            codes = torch.empty((rows, pitch(cols)), dtype=torch.int8, device=x.device)
        else:
            _require(codes, "codes", (rows, pitch(cols)), torch.int8, x.device)
            _aligned(codes, "codes")
        if scales is None:
            scales = torch.empty(rows, dtype=torch.float32, device=x.device)
        else:
            _require(scales, "scales", (rows,), torch.float32, x.device)
        fmm_q8_quantize(t, rows, cols, x, codes, scales, stream)
    return codes, scales


def dequantize(codes, scales, cols, dtype=torch.float32, out=None, stream=None):
    """The values that codes stand for (rows x cols).  scales: one per row, or
    the [rows][pitch / 128] of a checkpoint."""
    _matrix(codes, "codes")
    t = _type(dtype)
    rows, cols = codes.shape[0], int(cols)
    _require(codes, "codes", (rows, pitch(cols)), torch.int8, codes.device)
    _aligned(codes, "codes")
    if not isinstance(scales, torch.Tensor):
        raise ValueError(f"scales: expected a torch.Tensor, got {type(scales).__name__}")
    group = GROUP if scales.dim() == 2 else 0
    _require(scales, "scales", (rows, pitch(cols) // GROUP) if group else (rows,), torch.float32, codes.device)
    with torch.cuda.device(codes.device), _on(stream):
        if out is None:
            out = torch.empty((rows, cols), dtype=dtype, device=codes.device)
        else:
            _require(out, "out", (rows, cols), dtype, codes.device)
        fmm_q8_dequantize(t, rows, cols, group, codes, scales, out, stream)
    return out


class NormOutput(NamedTuple):
    h: torch.Tensor                        # x + residual (x itself where there is no residual)
    codes: torch.Tensor                    # int8 codes of the normalized rows ...
    scales: torch.Tensor                   # ... and their scales
    rstd: torch.Tensor                     # 1 / rms of h
    saved_codes: Optional[torch.Tensor]    # the checkpoint of h: codes ...
    saved_scales: Optional[torch.Tensor]   # ... and a scale per 128 columns


class RMSNormQ8:
    """The RMS norm of `rows` tokens of `cols` channels, with the residual's
    addition and an 8-bit output, on one device."""

    def __init__(self, rows, cols, dtype=torch.bfloat16, eps=1e-6, device="cuda:0"):
        self.rows, self.cols, self.dtype = int(rows), int(cols), dtype
        self.device = _device(device)
        self.desc = fmm_norm_desc(self.rows, self.cols, _type(dtype), float(eps))
        self.scratch_bytes = fmm_rmsnorm_q8_backward_scratch_size(self.desc)
        self.scratch = None     # the backward pass's workspace, from its first call on

    def _rows(self, x, name):
        _require(x, name, (self.rows, self.cols), self.dtype, self.device)

    def _floats(self, x, name, n):
        _require(x, name, (n,), torch.float32, self.device)

    def forward(self, x, residual=None, gain=None, checkpoint=False, inplace=False, stream=None) -> NormOutput:
        """h = x + residual; codes and scales of h / rms(h) * gain.  checkpoint:
        also the 8-bit checkpoint of h that `backward` takes.  inplace: h
        replaces the residual."""
        self._rows(x, "x")
        if residual is not None:
            self._rows(residual, "residual")
        elif inplace:
            raise ValueError("inplace: there is no residual to replace")
        if gain is not None:
            _require(gain, "gain", (self.cols,), self.dtype, self.device)
        R, P, dev = self.rows, pitch(self.cols), self.device
        with torch.cuda.device(dev), _on(stream):
            h = x if residual is None else residual if inplace else torch.empty_like(x)
            codes = torch.empty((R, P), dtype=torch.int8, device=dev)
            scales = torch.empty(R, dtype=torch.float32, device=dev)
            rstd = torch.empty(R, dtype=torch.float32, device=dev)
            saved = saved_scales = None
            if checkpoint:
                saved = torch.empty((R, P), dtype=torch.int8, device=dev)
                saved_scales = torch.empty((R, P // GROUP), dtype=torch.float32, device=dev)
            fmm_rmsnorm_q8(self.desc, x, residual, gain, None if residual is None else h, codes, scales, saved,
                           saved_scales, rstd, stream)
        return NormOutput(h, codes, scales, rstd, saved, saved_scales)

    def backward(self, dy, rstd, gain=None, h=None, saved=None, dh=None, need_gain=True, stream=None):
        """(gradient of x and of the residual, gradient of the gain or None) from
        dy, the gradient of the normalized rows, and dh, that of h from its other
        uses.  The forward pass's h comes as it was stored (h) or as its 8-bit
        checkpoint (saved = (saved_codes, saved_scales))."""
        R, P, dev = self.rows, pitch(self.cols), self.device
        self._rows(dy, "dy")
        self._floats(rstd, "rstd", R)
        if gain is not None:
            _require(gain, "gain", (self.cols,), self.dtype, dev)
        if dh is not None:
            self._rows(dh, "dh")
        if (h is None) == (saved is None):
            raise ValueError("h or saved: exactly one of them")
        codes = scales = None
        if h is not None:
            self._rows(h, "h")
        else:
            codes, scales = saved
            _require(codes, "saved codes", (R, P), torch.int8, dev)
            _aligned(codes, "saved codes")
            _require(scales, "saved scales", (R, P // GROUP), torch.float32, dev)
        with torch.cuda.device(dev), _on(stream):
            dx = torch.empty_like(dy)
            dgain = None
            if need_gain:
                dgain = torch.empty(self.cols, dtype=torch.float32, device=dev)
                if self.scratch is None:
                    self.scratch = torch.empty(max(self.scratch_bytes, 16), dtype=torch.uint8, device=dev)
            fmm_rmsnorm_q8_backward(self.desc, dy, dh, h, codes, scales, rstd, gain, dx, dgain, self.scratch,
                                    self.scratch_bytes, stream)
        return dx, dgain


class LinearQ8:
    """C (M x N) = A W^T of 8-bit operands: M tokens of K channels with a scale
    each, N output channels with a scale each; and its gradients."""

    def __init__(self, M, N, K, dtype=torch.bfloat16, device="cuda:0"):
        self.M, self.N, self.K, self.dtype = int(M), int(N), int(K), dtype
        self.device = _device(device)
        self.desc = fmm_q8_desc(self.M, self.N, self.K, _type(dtype))
        with torch.cuda.device(self.device):
            self.scratch_bytes = fmm_q8_matmul_scratch_size(self.desc)
        # the forward workspace, and the backward one from its first call on
        self.scratch = (torch.empty(self.scratch_bytes, dtype=torch.uint8, device=self.device)
                        if self.scratch_bytes else None)
        self.grad_scratch_bytes, self.grad_scratch = 0, None

    def _operand(self, codes, scales, name, rows):
        _require(codes, name, (rows, pitch(self.K)), torch.int8, self.device)
        _aligned(codes, name)
        _require(scales, name + " scales", (rows,), torch.float32, self.device)

    def matmul(self, a, sa, w, sw, bias=None, C=None, stream=None):
        """C = (codes a x scales sa) (codes w x scales sw)^T + bias."""
        self._operand(a, sa, "a", self.M)
        self._operand(w, sw, "w", self.N)
        if bias is not None:
            _require(bias, "bias", (self.N,), torch.float32, self.device)
        if C is not None:
            _require(C, "C", (self.M, self.N), self.dtype, self.device)
        with torch.cuda.device(self.device), _on(stream):
            if C is None:
                C = torch.empty((self.M, self.N), dtype=self.dtype, device=self.device)
            fmm_q8_matmul(self.desc, a, sa, w, sw, bias, C, self.scratch, self.scratch_bytes, stream)
        return C

    def backward(self, dy, a, sa, w, sw, need_x=True, need_w=True, bias=False, stream=None):
        """(dX, dW, dbias) from dy (M x N) and the 8-bit operands; None for what
        is not wanted (bias: whether its gradient is)."""
        _require(dy, "dy", (self.M, self.N), self.dtype, self.device)
        _aligned(dy, "dy")
        self._operand(a, sa, "a", self.M)
        self._operand(w, sw, "w", self.N)
        with torch.cuda.device(self.device), _on(stream):
            if self.grad_scratch is None:
                self.grad_scratch_bytes = fmm_q8_linear_backward_scratch_size(self.desc)
                self.grad_scratch = torch.empty(max(self.grad_scratch_bytes, 256), dtype=torch.uint8,
                                                device=self.device)
            dev = self.device
            dx = torch.empty((self.M, self.K), dtype=self.dtype, device=dev) if need_x else None
            dw = torch.empty((self.N, self.K), dtype=self.dtype, device=dev) if need_w else None
            dbias = torch.empty(self.N, dtype=torch.float32, device=dev) if bias else None
            fmm_q8_linear_backward(self.desc, dy, a, sa, w, sw, dx, dw, dbias, self.grad_scratch,
                                   self.grad_scratch_bytes, stream)
        return dx, dw, dbias
