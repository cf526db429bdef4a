"""The e4m3 layers' definitions in numpy: codes and scales by the stated rule,
everything computed from them in binary64."""
from __future__ import annotations

import numpy as np

BLOCK = 128
HALF_ULP = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}     # half a step, relative
SMALLEST = {"fp32": 2.0 ** -149, "bf16": 2.0 ** -133, "fp16": 2.0 ** -24}   # least subnormal


def _e4m3(code):
    """The number that a code from 0 to 126 stands for."""
    e, m = code >> 3, code & 7
    return m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)


TABLE = np.array([_e4m3(c) for c in range(127)])       # 0 .. 448, ascending


def pitch(cols):
    return -(-cols // BLOCK) * BLOCK


def scale_pitch(cols):
    return -(-(-(-cols // BLOCK)) // 16) * 16


def exponent(a):
    """The least e >= -126 with a <= 448 2^e (0 for a = 0)."""
    a = np.asarray(a, np.float64)
    m, x = np.frexp(a)
    return np.where(a > 0, np.maximum(np.where(m <= 0.875, x - 9, x - 8), -126), 0).astype(np.int64)


def nearest(u):
    """Codes of |u| <= 448: nearest, ties to the even code; 0x7f for NaN; the sign in bit 7."""
    mag = np.abs(u)
    bad = np.isnan(mag)
    mag = np.where(bad, 0.0, mag)
    hi = np.clip(np.searchsorted(TABLE, mag), 1, 126)
    lo = hi - 1
    below, above = mag - TABLE[lo], TABLE[hi] - mag
    c = np.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)
    return np.where(bad, 0x7f, c | np.where(np.signbit(u), 0x80, 0)).astype(np.uint8)


def _blocked(x, br):
    """x [..., R, K] padded, as [..., R / br, br, P / 128, 128]."""
    R, K = x.shape[-2:]
    x = np.pad(x, [(0, 0)] * (x.ndim - 2) + [(0, -R % br), (0, pitch(K) - K)])
    return x.reshape(*x.shape[:-2], x.shape[-2] // br, br, x.shape[-1] // BLOCK, BLOCK)


def codes(x, br=1):
    """(codes [..., R, P], scale bytes [..., R / br, SP]) with blocks of br x 128."""
    x = np.asarray(x, np.float64)
    R, K = x.shape[-2:]
    b = _blocked(x, br)
    fin = np.where(np.isfinite(b), b, 0.0)
    e = exponent(np.abs(fin).max(axis=(-3, -1), initial=0.0))
    u = np.where(np.isfinite(b), b, np.nan) * 2.0 ** -e[..., :, None, :, None].astype(np.float64)
    q = nearest(u).reshape(*x.shape[:-2], b.shape[-4] * br, pitch(K))[..., :R, :]
    s = (e + 127).astype(np.uint8)
    pad = [(0, 0)] * (s.ndim - 1) + [(0, scale_pitch(K) - s.shape[-1])]
    return q, np.pad(s, pad, constant_values=127)


def values(q, s, cols, br=1):
    """binary64 values of codes."""
    R, P = q.shape[-2:]
    mag = np.append(TABLE, np.nan)[q & 0x7f]
    v = np.where(q & 0x80, -mag, mag)
    e = np.repeat(np.repeat(s[..., :P // BLOCK].astype(np.int64) - 127, br, axis=-2)[..., :R, :], BLOCK, axis=-1)
    return (v * 2.0 ** e.astype(np.float64))[..., :cols]


def rounded(x, br=1):
    """The values of the codes of x."""
    return values(*codes(x, br), np.shape(x)[-1], br)


def rounded_columns(x, starts):
    """The values of the codes of x with blocks of 128 rows of a column, counted from each start."""
    out = np.zeros(np.shape(x))
    for a, b in zip(starts, list(starts[1:]) + [len(x)]):
        if b > a:
            out[a:b] = rounded(np.asarray(x)[a:b].T).T
    return out


def spans(offsets, rows):
    """[(first row, last row + 1)] of the experts, by the rule for offsets that are out of order."""
    top, cut = 0, []
    for o in offsets:
        top = max(top, min(max(int(o), 0), rows))
        cut.append(top)
    return list(zip(cut, cut[1:]))
