"""The end of a training step's backward pass over the C-ABI: the global norm of
many gradients, and clipping by it.  Checks and marshalling only: the arithmetic
happens in the library's HIP kernels."""
from __future__ import annotations

import ctypes

import torch

from . import _check, _lib, fmm_clip_scratch_size
from .q8 import TYPES, _run

_SCRATCH = fmm_clip_scratch_size()


def _list(ts, name):
    ts = list(ts)
    for t in ts:
        if not isinstance(t, torch.Tensor):
            raise ValueError(f"{name}: expected torch.Tensors, got {type(t).__name__}")
    if not all(map(torch.Tensor.is_contiguous, ts)):
        i = next(i for i, t in enumerate(ts) if not t.is_contiguous())
        raise ValueError(f"{name}[{i}]: not contiguous")
    return ts


def _apart(spans, what):
    """Refuse memory ranges that overlap: workgroups write them in any order."""
    spans.sort()
    for (_, end), (start, _) in zip(spans, spans[1:]):
        if start < end:
            raise ValueError(f"{what}: tensors overlap")


def clip(grads, max_norm, out=None, stream=None):
    """The norm (float32, on the device) of all elements of `grads` together, which are scaled in
    place, or into `out`, by min(1, max_norm / (norm + 1e-6)).

    grads: tensors of float32, bfloat16 or float16 (mixed or not) on one device.  Nothing is
    copied to the host: a norm that is not finite is for the caller to see, and gives
    gradients of zeros (infinity) or NaN."""
    most = float(max_norm)
    if not most >= 0.0:
        raise ValueError(f"max_norm: {max_norm}, expected a number >= 0")
    ins = _list(grads, "grads")
    if not ins:
        raise ValueError("grads: no tensors")
    outs = ins if out is None else _list(out, "out")
    if len(outs) != len(ins):
        raise ValueError(f"out: {len(outs)} tensors, expected {len(ins)}")
    dev, n = ins[0].device, len(ins)
    dtypes = [t.dtype for t in ins]
    try:
        types = [TYPES[d] for d in dtypes]
    except KeyError:
        raise ValueError(f"grads: dtypes {set(dtypes)}, expected float32, bfloat16 or float16") from None
    if any(t.device != dev for t in ins):
        raise ValueError(f"grads: on {[str(d) for d in {t.device for t in ins}]}, expected one device")
    sizes, at = list(map(torch.Tensor.numel, ins)), list(map(torch.Tensor.data_ptr, ins))
    to = at
    if out is not None:
        to = list(map(torch.Tensor.data_ptr, outs))
        if [t.dtype for t in outs] != dtypes or list(map(torch.Tensor.numel, outs)) != sizes:
            raise ValueError("out: other dtypes or sizes than grads")
        if any(t.device != dev for t in outs):
            raise ValueError(f"out: not on {dev}")
    width = [4 if t == 0 else 2 for t in types]
    written = [(p, p + s * w) for p, s, w in zip(to, sizes, width) if s]
    if out is not None:
        # an output may be its own input, and nothing else's (an input may come twice)
        written += {(p, p + s * w) for p, q, s, w in zip(at, to, sizes, width) if s and p != q}
    _apart(written, "grads" if out is None else "out")

    def call(handle):
        norm = torch.empty((), dtype=torch.float32, device=dev)
        scratch = torch.empty(_SCRATCH, dtype=torch.uint8, device=dev)
        _check(_lib.fmm_clip((ctypes.c_int32 * n)(*types), (ctypes.c_int64 * n)(*sizes), (ctypes.c_void_p * n)(*at),
                             (ctypes.c_void_p * n)(*to), n, most, norm.data_ptr(), scratch.data_ptr(), _SCRATCH, handle),
               "fmm_clip")
        return norm

    return _run(dev, stream, call, *ins, *(outs if out is not None else ()))
