"""The end of a training step's backward pass over the C-ABI: the global norm of
many gradients, and clipping by it.  Checks and marshalling only: the arithmetic
happens in the library's HIP kernels."""
from __future__ import annotations

import numpy as np
import torch
from torch.autograd.graph import increment_version

from . import FMM_F32, _check, _lib, fmm_clip_scratch_size
from .q8 import TYPES, _run

_SCRATCH = fmm_clip_scratch_size()


# What a call costs is the walk over its tensors (six questions to each, 50 ns a question), so they are
# asked by map, and all else is done on arrays.
_Tensor = torch.Tensor


def _table(ts, name):
    """(types, sizes, addresses, device index) of tensors."""
    if not set(map(type, ts)) <= {_Tensor, torch.nn.Parameter}:
        for t in ts:
            if not isinstance(t, _Tensor):
                raise ValueError(f"{name}: expected torch.Tensors, got {type(t).__name__}")
    if not all(map(_Tensor.is_contiguous, ts)):
        i = next(i for i, t in enumerate(ts) if not t.is_contiguous())
        raise ValueError(f"{name}[{i}]: not contiguous")
    try:
        types = np.array([TYPES[t.dtype] for t in ts], dtype=np.int32)
    except KeyError:
        raise ValueError(f"{name}: dtypes {set(t.dtype for t in ts)}, expected float32, bfloat16 or float16") from None
    devices = set(map(_Tensor.get_device, ts))
    if len(devices) > 1:
        raise ValueError(f"{name}: on {sorted(str(d) for d in set(t.device for t in ts))}, expected one device")
    return (types, np.array(list(map(_Tensor.numel, ts)), dtype=np.int64),
            np.array(list(map(_Tensor.data_ptr, ts)), dtype=np.int64), devices.pop())


def _apart(to, size, at, what):
    """Refuse outputs that overlap one another, or an input other than their own: workgroups
    read and write them in any order."""
    some = size > 0
    order = np.argsort(to[some], kind="stable")
    start, end = to[some][order], (to + size)[some][order]
    clash = (start[1:] < end[:-1]).any()
    if not clash and at is not to:
        other = some & (at != to)
        first = np.searchsorted(end, at[other], side="right")       # the first output that ends past the input's start
        clash = (np.append(start, np.iinfo(np.int64).max)[first] < (at + size)[other]).any()
    if clash:
        raise ValueError(f"{what}: tensors overlap")


def clip(grads, max_norm, out=None, stream=None):
    """The norm (float32, on the device) of all elements of `grads` together, which are scaled in
    place, or into `out`, by min(1, max_norm / (norm + 1e-6)).

    grads: tensors of float32, bfloat16 or float16 (mixed or not) on one device.  Nothing is
    copied to the host: a norm that is not finite is for the caller to see, and gives
    gradients of zeros (infinity) or NaN.  What is written counts as written in place: torch's
    version counters move, so a graph that has kept such a tensor refuses its backward pass."""
    most = float(max_norm)
    if not most >= 0.0:
        raise ValueError(f"max_norm: {max_norm}, expected a number >= 0")
    ins = list(grads)
    if not ins:
        raise ValueError("grads: no tensors")
    types, sizes, at, index = _table(ins, "grads")
    n, dev, to = len(ins), ins[0].device, at
    nbytes = sizes * np.where(types == FMM_F32, 4, 2)
    outs = () if out is None else list(out)
    if out is not None:
        if len(outs) != n:
            raise ValueError(f"out: {len(outs)} tensors, expected {n}")
        to_types, to_sizes, to, to_index = _table(outs, "out")
        if (to_types != types).any() or (to_sizes != sizes).any():
            raise ValueError("out: other dtypes or sizes than grads")
        if to_index != index:
            raise ValueError(f"out: on {outs[0].device}, expected {dev}")
    _apart(to, nbytes, at, "grads" if out is None else "out")

    def call(handle):
        norm = torch.empty((), dtype=torch.float32, device=dev)
        scratch = torch.empty(_SCRATCH, dtype=torch.uint8, device=dev)
        _check(_lib.fmm_clip(types.ctypes.data, sizes.ctypes.data, at.ctypes.data, to.ctypes.data, n, most, norm.data_ptr(),
                             scratch.data_ptr(), _SCRATCH, handle), "fmm_clip")
        increment_version(ins if out is None else outs)      # (a graph that has kept one of them has to refuse)
        return norm

    return _run(dev, stream, call, *ins, *outs)
