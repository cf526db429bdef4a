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
`stream` (default: torch's current one) and allocates its outputs there.  Any
streams and threads may use an object at once: it keeps a workspace for each
stream that a backward call came on.
"""
from __future__ import annotations

from contextlib import contextmanager
from threading import Lock
from typing import NamedTuple, Optional

import torch

from . import (FMM_BF16, FMM_F16, FMM_F32, _check, _lib, fmm_norm_desc, fmm_q8_desc,
               fmm_q8_linear_backward_scratch_size, fmm_rmsnorm_q8_backward_scratch_size)
from .runner import _require

GROUP = 128
TYPES = {torch.float32: FMM_F32, torch.bfloat16: FMM_BF16, torch.float16: FMM_F16}

# A call's host time is a small product's whole time, so what follows avoids the
# 3 us of torch.cuda.current_stream() and the device context where it can, and
# passes torch.empty sizes rather than a tuple of them (1.25 us and 1.6).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
if _raw_stream is None:
    def _raw_stream(index):
        return torch.cuda.current_stream(index).cuda_stream


class _Workspace:
    """The backward pass's memory of an object, a block for each stream: what a call
    on one adds up never passes through another's.  The lock is held over a call's
    launches, which another thread's on the same stream must not fall between.  A
    call that is being captured gets a block of the graph's, since its replays may
    run beside later calls.  (A block that all objects' calls share, from the
    allocator, costs more: 256 tokens of 2048 x 2048 21 us, 17.5 where three objects
    with their own take turns.)"""

    def __init__(self):
        self.lock, self.blocks = Lock(), {}

    def __reduce__(self):       # a copy of an object starts without one
        return _Workspace, ()

    def get(self, handle, nbytes, device):
        if torch.cuda.is_current_stream_capturing():
            return torch.empty(nbytes, dtype=torch.uint8, device=device)
        block = self.blocks.get(handle)
        if block is None:
            block = self.blocks[handle] = torch.empty(nbytes, dtype=torch.uint8, device=device)
        return block


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


def _tensor(x, name, shape, dtype, device):
    """_require, with the usual case decided without building what a message needs."""
    try:
        if x.dtype is dtype and x.shape == shape and x.device == device and x.is_contiguous():
            return
    except AttributeError:
        pass
    _require(x, name, shape, dtype, device)


def _codes(x, name, shape, device):
    """Codes are read by 16-byte vectors."""
    _tensor(x, name, shape, torch.int8, device)
    if x.data_ptr() % 16:
        raise ValueError(f"{name}: not 16-byte aligned")


def _ptr(x):
    return None if x is None else x.data_ptr()


@contextmanager
def _switched(index, stream):
    """The device, and the stream where one is given, made current: outputs are
    allocated on the stream that writes them, so that torch's allocator reuses
    their memory in that stream's order."""
    with torch.cuda.device(index):
        if stream is None:
            yield _raw_stream(index)
        else:
            if isinstance(stream, int):
                # (torch takes a null handle for "any stream of its pool", not for the default stream)
                stream = torch.cuda.ExternalStream(stream) if stream else torch.cuda.default_stream(index)
            if stream.device_index != index:
                raise ValueError(f"stream: of device {stream.device_index}, expected {index}")
            with torch.cuda.stream(stream):
                yield stream.cuda_stream


def _run(device, stream, call, *tensors):
    """call(stream handle), on the device and the stream.  A stream that the
    caller names may not be the one the inputs were allocated on: the allocator
    is told, so that it does not hand out their memory before the call is done.
    A kernel that is handed host memory faults, so nothing else gets past here (the
    tensors are known to be on `device`; the first is never None)."""
    if not tensors[0].is_cuda:
        raise ValueError(f"device {device}, expected a GPU")
    index = device.index
    if stream is None and torch.cuda.current_device() == index:
        return call(_raw_stream(index))
    with _switched(index, stream) as handle:
        out = call(handle)
        if stream is not None:
            used = torch.cuda.current_stream(index)
            for x in tensors:
                if x is not None:
                    x.record_stream(used)
    return out


def _matrix(x, name):
    if not isinstance(x, torch.Tensor):
        raise ValueError(f"{name}: expected a torch.Tensor, got {type(x).__name__}")
    if x.dim() != 2:
        raise ValueError(f"{name}: shape {tuple(x.shape)}, expected a matrix")


def quantize(x, codes=None, scales=None, stream=None):
    """(codes, scales) of the rows of x (float32, bfloat16 or float16)."""
    _matrix(x, "x")
    t = _type(x.dtype)
    rows, cols = x.shape
    dev, shape = x.device, (rows, pitch(cols))
    if not x.is_contiguous():
        raise ValueError("x: not contiguous")
    if codes is not None:
        _codes(codes, "codes", shape, dev)
    if scales is not None:
        _tensor(scales, "scales", (rows,), torch.float32, dev)

    def call(handle):
        q = torch.empty(*shape, dtype=torch.int8, device=dev) if codes is None else codes
        s = torch.empty(rows, dtype=torch.float32, device=dev) if scales is None else scales
        _check(_lib.fmm_q8_quantize(t, rows, cols, x.data_ptr(), q.data_ptr(), s.data_ptr(), handle), "fmm_q8_quantize")
        return q, s

    return _run(dev, stream, call, x, codes, scales)


def dequantize(codes, scales, cols, dtype=torch.float32, out=None, stream=None):
    """The values that codes stand for (rows x cols).  scales: one per row, or
    the [rows][pitch / 128] of a checkpoint."""
    _matrix(codes, "codes")
    t = _type(dtype)
    rows, cols, dev = codes.shape[0], int(cols), codes.device
    p = pitch(cols)
    _codes(codes, "codes", (rows, p), dev)
    if not isinstance(scales, torch.Tensor):
        raise ValueError(f"scales: expected a torch.Tensor, got {type(scales).__name__}")
    group = GROUP if scales.dim() == 2 else 0
    _tensor(scales, "scales", (rows, p // GROUP) if group else (rows,), torch.float32, dev)
    if out is not None:
        _tensor(out, "out", (rows, cols), dtype, dev)

    def call(handle):
        o = torch.empty(rows, cols, dtype=dtype, device=dev) if out is None else out
        _check(_lib.fmm_q8_dequantize(t, rows, cols, group, codes.data_ptr(), scales.data_ptr(), o.data_ptr(), handle),
               "fmm_q8_dequantize")
        return o

    return _run(dev, stream, call, codes, scales, out)


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
        P = pitch(self.cols)
        self._x, self._q, self._s = (self.rows, self.cols), (self.rows, P), (self.rows, P // GROUP)   # shapes
        self.scratch_bytes = fmm_rmsnorm_q8_backward_scratch_size(self.desc)
        self.scratch = _Workspace()

    def forward(self, x, residual=None, gain=None, checkpoint=False, inplace=False, stream=None) -> NormOutput:
        """h = x + residual; codes and scales of h / rms(h) * gain.  checkpoint:
        also the 8-bit checkpoint of h that `backward` takes.  inplace: h
        replaces the residual."""
        dev, dtype, R = self.device, self.dtype, self.rows
        _tensor(x, "x", self._x, dtype, dev)
        if residual is not None:
            _tensor(residual, "residual", self._x, dtype, dev)
        elif inplace:
            raise ValueError("inplace: there is no residual to replace")
        if gain is not None:
            _tensor(gain, "gain", (self.cols,), dtype, dev)

        def call(handle):
            h = x if residual is None else residual if inplace else torch.empty_like(x)
            codes = torch.empty(*self._q, dtype=torch.int8, device=dev)
            scales = torch.empty(R, dtype=torch.float32, device=dev)
            rstd = torch.empty(R, dtype=torch.float32, device=dev)
            saved = saved_scales = None
            if checkpoint:
                saved = torch.empty(*self._q, dtype=torch.int8, device=dev)
                saved_scales = torch.empty(*self._s, dtype=torch.float32, device=dev)
            _check(_lib.fmm_rmsnorm_q8(self.desc, x.data_ptr(), _ptr(residual), _ptr(gain),
                                       None if residual is None else h.data_ptr(), codes.data_ptr(), scales.data_ptr(),
                                       _ptr(saved), _ptr(saved_scales), rstd.data_ptr(), handle), "fmm_rmsnorm_q8")
            return NormOutput(h, codes, scales, rstd, saved, saved_scales)

        return _run(dev, stream, call, x, residual, gain)

    def backward(self, dy, rstd, gain=None, h=None, saved=None, dh=None, need_gain=True, stream=None):
        """(gradient of x and of the residual, gradient of the gain or None) from
        dy, the gradient of the normalized rows, and dh, that of h from its other
        uses.  The forward pass's h comes as it was stored (h) or as its 8-bit
        checkpoint (saved = (saved_codes, saved_scales))."""
        dev, dtype = self.device, self.dtype
        _tensor(dy, "dy", self._x, dtype, dev)
        _tensor(rstd, "rstd", (self.rows,), torch.float32, dev)
        if gain is not None:
            _tensor(gain, "gain", (self.cols,), dtype, dev)
        if dh is not None:
            _tensor(dh, "dh", self._x, dtype, dev)
        if (h is None) == (saved is None):
            raise ValueError("h or saved: exactly one of them")
        codes = scales = None
        if h is not None:
            _tensor(h, "h", self._x, dtype, dev)
        else:
            codes, scales = saved
            _codes(codes, "saved codes", self._q, dev)
            _tensor(scales, "saved scales", self._s, torch.float32, dev)

        def call(handle):
            dx = torch.empty_like(dy)
            dgain = torch.empty(self.cols, dtype=torch.float32, device=dev) if need_gain else None
            with self.scratch.lock:
                scratch = self.scratch.get(handle, self.scratch_bytes, dev) if need_gain and self.scratch_bytes else None
                _check(_lib.fmm_rmsnorm_q8_backward(self.desc, dy.data_ptr(), _ptr(dh), _ptr(h), _ptr(codes), _ptr(scales),
                                                    rstd.data_ptr(), _ptr(gain), dx.data_ptr(), _ptr(dgain),
                                                    _ptr(scratch), self.scratch_bytes, handle),
                       "fmm_rmsnorm_q8_backward")
            return dx, dgain

        return _run(dev, stream, call, dy, rstd, gain, h, codes, scales, dh)


class LinearQ8:
    """C (M x N) = A W^T of 8-bit operands: M tokens of K channels with a scale
    each, N output channels with a scale each; and its gradients."""

    def __init__(self, M, N, K, dtype=torch.bfloat16, device="cuda:0"):
        self.M, self.N, self.K, self.dtype = int(M), int(N), int(K), dtype
        self.device = _device(device)
        self.desc = fmm_q8_desc(self.M, self.N, self.K, _type(dtype))
        self._a, self._w = (self.M, pitch(self.K)), (self.N, pitch(self.K))   # shapes
        self.grad_scratch_bytes, self.grad_scratch = None, _Workspace()     # (sized by the first backward call)

    def _operands(self, a, sa, w, sw):
        dev = self.device
        _codes(a, "a", self._a, dev)
        _tensor(sa, "a scales", (self.M,), torch.float32, dev)
        _codes(w, "w", self._w, dev)
        _tensor(sw, "w scales", (self.N,), torch.float32, dev)

    def matmul(self, a, sa, w, sw, bias=None, C=None, stream=None):
        """C = (codes a x scales sa) (codes w x scales sw)^T + bias."""
        dev = self.device
        self._operands(a, sa, w, sw)
        if bias is not None:
            _tensor(bias, "bias", (self.N,), torch.float32, dev)
        if C is not None:
            _tensor(C, "C", (self.M, self.N), self.dtype, dev)

        def call(handle):
            out = torch.empty(self.M, self.N, dtype=self.dtype, device=dev) if C is None else C
            _check(_lib.fmm_q8_matmul(self.desc, a.data_ptr(), sa.data_ptr(), w.data_ptr(), sw.data_ptr(), _ptr(bias),
                                      out.data_ptr(), handle), "fmm_q8_matmul")
            return out

        return _run(dev, stream, call, a, sa, w, sw, bias, C)

    def backward(self, dy, a, sa, w, sw, need_x=True, need_w=True, bias=False, stream=None):
        """(dX, dW, dbias) from dy (M x N) and the 8-bit operands; None for what
        is not wanted (bias: whether its gradient is)."""
        dev = self.device
        _tensor(dy, "dy", (self.M, self.N), self.dtype, dev)
        if dy.data_ptr() % 16:
            raise ValueError("dy: not 16-byte aligned")
        self._operands(a, sa, w, sw)

        def call(handle):
            if self.grad_scratch_bytes is None:
                self.grad_scratch_bytes = fmm_q8_linear_backward_scratch_size(self.desc)
            dx = torch.empty(self.M, self.K, dtype=self.dtype, device=dev) if need_x else None
            dw = torch.empty(self.N, self.K, dtype=self.dtype, device=dev) if need_w else None
            dbias = torch.empty(self.N, dtype=torch.float32, device=dev) if bias else None
            with self.grad_scratch.lock:
                scratch = self.grad_scratch.get(handle, self.grad_scratch_bytes, dev)
                _check(_lib.fmm_q8_linear_backward(self.desc, dy.data_ptr(), a.data_ptr(), sa.data_ptr(), w.data_ptr(),
                                                   sw.data_ptr(), _ptr(dx), _ptr(dw), _ptr(dbias),
                                                   scratch.data_ptr(), self.grad_scratch_bytes, handle),
                       "fmm_q8_linear_backward")
            return dx, dw, dbias

        return _run(dev, stream, call, dy, a, sa, w, sw)
