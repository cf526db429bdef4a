"""The 8-bit linear layer's definitions in numpy: codes by the stated binary32
rule (so that they can be compared bit for bit), everything else in binary64."""
from __future__ import annotations

import numpy as np

GROUP = 128
EPS32 = 2.0 ** -24          # half an ulp of binary32, relative
HALF_ULP = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}     # 24, 8 and 11 significant bits
SMALLEST = {"fp32": 2.0 ** -149, "bf16": 2.0 ** -133, "fp16": 2.0 ** -24}   # least subnormal


def pitch(cols):
    return -(-cols // GROUP) * GROUP


def codes_of(v):
    """(codes, scales) of the rows (last axis) of a float32 array, by the rule."""
    v = np.asarray(v, dtype=np.float32)
    mag = np.abs(v)
    amax = mag.max(axis=-1) if v.shape[-1] else np.zeros(v.shape[:-1], np.float32)
    bad = ~np.isfinite(v).all(axis=-1)
    a = np.where(bad, np.float32(1), np.maximum(amax, np.float32(1e-12))).astype(np.float32)
    with np.errstate(invalid="ignore"):
        q = np.rint(v * (np.float32(127) / a)[..., None])
    q = np.where(bad[..., None], 0, q).astype(np.int8)
    s = np.where(bad, np.float32(np.nan), a / np.float32(127)).astype(np.float32)
    return q, s


def padded_codes(v):
    q, s = codes_of(v)
    return np.pad(q, ((0, 0), (0, pitch(v.shape[1]) - v.shape[1]))), s


def checkpoint(h):
    """Codes and scales of each group of 128 columns."""
    R, K = h.shape
    P = pitch(K)
    q, s = codes_of(np.pad(h, ((0, 0), (0, P - K))).reshape(R, P // GROUP, GROUP))
    return q.reshape(R, P), s


def values(q, s, cols):
    """binary64 values of codes (scales [rows], or [rows][groups])."""
    s = np.asarray(s, np.float64)
    s = np.repeat(s, GROUP, axis=1)[:, :cols] if s.ndim == 2 else s[:, None]
    return q[:, :cols].astype(np.float64) * s


def norm_gradient(h, rstd, dy, gain, dh):
    """(dx, dgain, bound of the terms of dx, bound of those of dgain), binary64."""
    xh, w = h * rstd[:, None], dy * gain
    c = (w * xh).mean(axis=1, keepdims=True)
    dx = rstd[:, None] * (w - xh * c) + dh
    terms = np.abs(rstd[:, None]) * (np.abs(w) + np.abs(xh) * np.abs(w * xh).mean(axis=1, keepdims=True)) + np.abs(dh)
    return dx, (dy * xh).sum(axis=0), terms, np.abs(dy * xh).sum(axis=0)
