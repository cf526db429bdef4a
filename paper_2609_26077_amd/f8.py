"""Linear layers on e4m3 operands over the C-ABI with torch-owned device buffers.

`quantize` makes the codes of activations, with a power-of-two scale for each
128 columns of a row, `quantize_weight` those of a weight or of many experts' (a
scale for each 128 x 128), `dequantize` the values that codes stand for.  `LinearF8`
multiplies activations by a weight, `GroupedLinearF8` each expert's rows by the
expert's weight; both have 8-bit gradients, from the codes that the forward pass took.

Codes are torch.float8_e4m3fn [rows][pitch(cols)], zero past cols; scales are
torch.float8_e8m0fnu [rows][scale_pitch(cols)], of a weight [ceil(rows / 128)][...].
Allocation, checks and marshalling only: the arithmetic happens in the library's
HIP kernels.  Every call runs on `stream` (default: torch's current one) and
allocates its outputs there.  Any streams and threads may use an object at
once: it keeps a workspace for each stream that a backward call came on.
"""
from __future__ import annotations

import torch

from . import _check, _lib, fmm_f8_desc, fmm_f8_linear_backward_scratch_size
from .q8 import _device, _matrix, _ptr, _run, _tensor, _type, _Workspace, pitch

BLOCK = 128
CODES, SCALES = torch.float8_e4m3fn, torch.float8_e8m0fnu


def scale_pitch(cols: int) -> int:
    """Scales of one row: one for each 128 columns, rounded up to 16."""
    return ((cols + BLOCK - 1) // BLOCK + 15) // 16 * 16


def _bytes(x, name, shape, dtype, device):
    """Codes and scales are read by vectors."""
    _tensor(x, name, shape, dtype, device)
    if x.data_ptr() % 16:
        raise ValueError(f"{name}: not 16-byte aligned")


def _coded(x, name, codes, scales, lead, rows, srows, cols, fill, stream):
    """(codes, scales) of x, provided or new, from fill(x, codes, scales, stream handle)."""
    if not x.is_contiguous():
        raise ValueError("x: not contiguous")
    dev, qs, ss = x.device, (*lead, rows, pitch(cols)), (*lead, srows, scale_pitch(cols))
    if codes is not None:
        _bytes(codes, "codes", qs, CODES, dev)
    if scales is not None:
        _bytes(scales, "scales", ss, SCALES, dev)

    def call(handle):
        q = torch.empty(*qs, dtype=CODES, device=dev) if codes is None else codes
        s = torch.empty(*ss, dtype=SCALES, device=dev) if scales is None else scales
        _check(fill(x.data_ptr(), q.data_ptr(), s.data_ptr(), handle), name)
        return q, s

    return _run(dev, stream, call, x, codes, scales)


def quantize(x, codes=None, scales=None, stream=None):
    """(codes, scales) of the rows of x (float32, bfloat16 or float16)."""
    _matrix(x, "x")
    t = _type(x.dtype)
    rows, cols = x.shape
    return _coded(x, "fmm_f8_quantize", codes, scales, (), rows, rows, cols,
                  lambda *p: _lib.fmm_f8_quantize(t, rows, cols, *p), stream)


def quantize_weight(x, codes=None, scales=None, stream=None):
    """(codes, scales) of a weight (N x K) or of experts' (experts x N x K)."""
    if not isinstance(x, torch.Tensor):
        raise ValueError(f"x: expected a torch.Tensor, got {type(x).__name__}")
    if x.dim() not in (2, 3):
        raise ValueError(f"x: shape {tuple(x.shape)}, expected a matrix or one for each expert")
    t = _type(x.dtype)
    lead, (rows, cols) = tuple(x.shape[:-2]), x.shape[-2:]
    count = lead[0] if lead else 1
    return _coded(x, "fmm_f8_quantize_weight", codes, scales, lead, rows, -(-rows // BLOCK), cols,
                  lambda *p: _lib.fmm_f8_quantize_weight(t, count, rows, cols, *p), stream)


def dequantize(codes, scales, cols, dtype=torch.float32, out=None, stream=None):
    """The values that codes stand for, in `cols` columns: of activations, or of a
    weight or experts' (told by the rows of `scales`)."""
    if not isinstance(codes, torch.Tensor) or not isinstance(scales, torch.Tensor):
        raise ValueError("codes, scales: expected torch.Tensors")
    if codes.dim() not in (2, 3):
        raise ValueError(f"codes: shape {tuple(codes.shape)}, expected a matrix or one for each expert")
    t = _type(dtype)
    cols, dev = int(cols), codes.device
    lead, rows = tuple(codes.shape[:-2]), codes.shape[-2]
    _bytes(codes, "codes", (*lead, rows, pitch(cols)), CODES, dev)
    blocks = 1 if not lead and scales.dim() == 2 and scales.shape[0] == rows else BLOCK
    _bytes(scales, "scales", (*lead, -(-rows // blocks), scale_pitch(cols)), SCALES, dev)
    if out is not None:
        _tensor(out, "out", (*lead, rows, cols), dtype, dev)
    count = lead[0] if lead else 1

    def call(handle):
        o = torch.empty(*lead, rows, cols, dtype=dtype, device=dev) if out is None else out
        _check(_lib.fmm_f8_dequantize(t, count, rows, cols, blocks, codes.data_ptr(), scales.data_ptr(), o.data_ptr(),
                                      handle), "fmm_f8_dequantize")
        return o

    return _run(dev, stream, call, codes, scales, out)


class _Layer:
    def __init__(self, rows, experts, N, K, dtype, device, lead):
        self.rows, self.experts, self.N, self.K, self.dtype = int(rows), int(experts), int(N), int(K), dtype
        self.device = _device(device)
        self.desc = fmm_f8_desc(self.rows, self.experts, self.N, self.K, _type(dtype))
        P, SP = pitch(self.K), scale_pitch(self.K)
        self._a, self._sa = (self.rows, P), (self.rows, SP)                                     # shapes
        self._w, self._sw = (*lead, self.N, P), (*lead, -(-self.N // BLOCK), SP)
        self._c, self._bias, self._dw = (self.rows, self.N), (*lead, self.N), (*lead, self.N, self.K)
        self.grad_scratch_bytes, self.grad_scratch = None, _Workspace()     # (sized by the first backward call)

    def _operands(self, a, sa, w, sw, offsets):
        dev = self.device
        _bytes(a, "a", self._a, CODES, dev)
        _bytes(sa, "a scales", self._sa, SCALES, dev)
        _bytes(w, "w", self._w, CODES, dev)
        _bytes(sw, "w scales", self._sw, SCALES, dev)
        if offsets is not None:
            _tensor(offsets, "offsets", (self.experts + 1,), torch.int32, dev)

    def _matmul(self, a, sa, w, sw, offsets, bias, C, stream):
        dev = self.device
        self._operands(a, sa, w, sw, offsets)
        if bias is not None:
            _tensor(bias, "bias", self._bias, torch.float32, dev)
        if C is not None:
            _tensor(C, "C", self._c, self.dtype, dev)

        def call(handle):
            out = torch.empty(*self._c, dtype=self.dtype, device=dev) if C is None else C
            _check(_lib.fmm_f8_matmul(self.desc, a.data_ptr(), sa.data_ptr(), w.data_ptr(), sw.data_ptr(), _ptr(offsets),
                                      _ptr(bias), out.data_ptr(), handle), "fmm_f8_matmul")
            return out

        return _run(dev, stream, call, a, sa, w, sw, offsets, bias, C)

    def _backward(self, dy, a, sa, w, sw, offsets, need_x, need_w, bias, stream):
        dev = self.device
        _tensor(dy, "dy", self._c, self.dtype, dev)
        self._operands(a, sa, w, sw, offsets)

        def call(handle):
            if self.grad_scratch_bytes is None:
                self.grad_scratch_bytes = fmm_f8_linear_backward_scratch_size(self.desc)
            dx = torch.empty(*self._a[:1], self.K, dtype=self.dtype, device=dev) if need_x else None
            dw = torch.empty(*self._dw, dtype=self.dtype, device=dev) if need_w else None
            dbias = torch.empty(*self._bias, dtype=torch.float32, device=dev) if bias else None
            with self.grad_scratch.lock:
                scratch = self.grad_scratch.get(handle, self.grad_scratch_bytes, dev)
                _check(_lib.fmm_f8_linear_backward(self.desc, dy.data_ptr(), a.data_ptr(), sa.data_ptr(), w.data_ptr(),
                                                   sw.data_ptr(), _ptr(offsets), _ptr(dx), _ptr(dw), _ptr(dbias),
                                                   scratch.data_ptr(), self.grad_scratch_bytes, handle),
                       "fmm_f8_linear_backward")
            return dx, dw, dbias

        return _run(dev, stream, call, dy, a, sa, w, sw, offsets)


class LinearF8(_Layer):
    """C (M x N) = A W^T of e4m3 operands: M tokens of K channels with a scale for each
    128 of them, N output channels with a scale for each 128 x 128; and its gradients."""

    def __init__(self, M, N, K, dtype=torch.bfloat16, device="cuda:0"):
        super().__init__(M, 1, N, K, dtype, device, ())

    def matmul(self, a, sa, w, sw, bias=None, C=None, stream=None):
        """C = (codes a x scales sa) (codes w x scales sw)^T + bias (float32)."""
        return self._matmul(a, sa, w, sw, None, bias, C, stream)

    def backward(self, dy, a, sa, w, sw, need_x=True, need_w=True, bias=False, stream=None):
        """(dX, dW, dbias) from dy (M x N) and the 8-bit operands; None for what
        is not wanted (bias: whether its gradient is)."""
        return self._backward(dy, a, sa, w, sw, None, need_x, need_w, bias, stream)


class GroupedLinearF8(_Layer):
    """The same for `experts` weights: expert e has the rows offsets[e] .. offsets[e + 1] - 1
    (offsets: int32, on the device, read there).  Rows of no expert are left as they were in
    C, and hold nothing of use in what a call allocates."""

    def __init__(self, rows, experts, N, K, dtype=torch.bfloat16, device="cuda:0"):
        super().__init__(rows, experts, N, K, dtype, device, (int(experts),))

    def matmul(self, a, sa, w, sw, offsets, bias=None, C=None, stream=None):
        """C[m] = a[m] w[e]^T + bias[e], e the expert of row m (bias: float32, experts x N)."""
        if offsets is None:
            raise ValueError("offsets: expected a torch.Tensor, got None")
        return self._matmul(a, sa, w, sw, offsets, bias, C, stream)

    def backward(self, dy, a, sa, w, sw, offsets, need_x=True, need_w=True, bias=False, stream=None):
        """(dX, dW, dbias), experts x ... for the last two; zeros for experts without rows."""
        if offsets is None:
            raise ValueError("offsets: expected a torch.Tensor, got None")
        return self._backward(dy, a, sa, w, sw, offsets, need_x, need_w, bias, stream)
