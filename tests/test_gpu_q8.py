"""The 8-bit linear layer on the GPU against binary64 (tests/q8_reference.py).

Bars.  u = 2^-24 is half an ulp of binary32, u_T that of the output's type.
* codes, stored h: equal (the rule is a sequence of binary32 operations, none
  of which depends on an order of summation);
* 1 / rms: a row's squares are summed by threads (at most 40 in a chain) and
  then across them (6 + 16 steps): 64 u relative, and 4 u for the root and
  division; a norm's scale 4 u more;
* the norm's gradients: the same sum inside c, then a handful of operations:
  80 u times the sum of the terms' magnitudes, and u_T |dx| for the store; the
  gain's sum over rows (rows + 16) u times its terms' magnitudes;
* the product: the integer sum is exact; its conversion, two scales and the
  bias's addition each cost u: 4 u |acc sa sw| + 2 u |bias|, and u_T |C|;
* the linear gradients, S = the sum of the terms' magnitudes: n u S for adding n
  terms in any order, 2^-19 S for the matrix core's own sums (as in
  gpu_helpers), and the operand's rounding: 2^-8 S for bf16 (one operand to 8
  bits), 2^-16 S for fp16 (two parts), 2^-23 S for
  fp32 (three), and u_T |result|.
"""
from __future__ import annotations

import numpy as np
import pytest

import q8_reference as ref

pytestmark = pytest.mark.gpu

U = ref.EPS32
TYPES = ["fp32", "bf16", "fp16"]
ROUNDING = {"fp32": 2.0 ** -23, "bf16": 2.0 ** -8, "fp16": 2.0 ** -16}


@pytest.fixture(scope="module")
def torch():
    import torch
    return torch


@pytest.fixture(scope="module")
def q8():
    from paper_2609_26077_amd import q8
    return q8


def dtype_of(torch, t):
    return {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}[t]


def randn(torch, seed, *shape, t="fp32", scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (scale * torch.randn(*shape, generator=g)).to(dtype_of(torch, t)).cuda()


def f32(x):
    return x.detach().float().cpu().numpy()


def f64(x):
    return x.detach().double().cpu().numpy()


def within(got, want, bound, what):
    err = np.abs(got - want)
    bad = ~(err <= bound)
    assert not bad.any(), f"{what}: {bad.sum()} outside, worst {np.max(err / np.maximum(bound, 1e-300)):.3g} of the bound"


def codes(torch, seed, rows, cols):
    """Codes over the whole int8 range, -128 included, and scales."""
    g = torch.Generator().manual_seed(seed)
    q = torch.zeros((rows, ref.pitch(cols)), dtype=torch.int8)
    q[:, :cols] = torch.randint(-128, 128, (rows, cols), generator=g, dtype=torch.int8)
    s = torch.rand(rows, generator=g) * 0.05 + 1e-3
    return q.cuda(), s.cuda()


# ---- rows -------------------------------------------------------------------------
WIDTHS = [1, 7, 8, 127, 128, 129, 511, 513, 1301, 2048, 2056, 4096, 4100, 8192, 8200, 16385, 32768, 32771]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, c) for c in WIDTHS] + [(5, 129), (515, 513), (515, 2047), (515, 4095),
                                                                  (515, 8191), (70, 9001), (9, 40000), (0, 100), (3, 0)])
def test_quantize_codes(torch, q8, t, rows, cols):
    x = randn(torch, rows * 7 + cols, rows, cols, t=t, scale=3.0)
    q, s = q8.quantize(x)
    want_q, want_s = ref.padded_codes(f32(x))
    assert np.array_equal(q.cpu().numpy(), want_q)
    assert np.array_equal(s.cpu().numpy(), want_s)
    # nearest multiples of the scale, in binary64
    if rows and cols:
        v = ref.values(want_q, s.cpu().numpy(), cols)
        within(v, f64(x), (0.5 + 2.0 ** -15) * f64(s)[:, None], "half a step")


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("cols", [1, 130, 2047, 4097, 33000])
def test_quantize_rows_without_a_scale(torch, q8, t, cols):
    """Zero rows, tiny rows, the type's largest values, NaN and infinities (each in a row of its own), ties."""
    x = randn(torch, 3, 9, cols, t=t)
    x[0] = 0
    x[1] = 1e-20 if t != "fp16" else 6e-8
    x[2, cols // 2] = float("nan")
    x[3, cols - 1] = float("inf")
    x[4, 0] = float("-inf")
    x[5] = torch.finfo(x.dtype).max
    x[6] = torch.finfo(x.dtype).min
    x[7] = 0.5
    x[7, 0] = 127.0          # x 127 / a = 0.5 exactly: to even, 0
    q, s = q8.quantize(x)
    want_q, want_s = ref.padded_codes(f32(x))
    assert np.array_equal(q.cpu().numpy(), want_q)
    assert np.array_equal(s.cpu().numpy(), want_s, equal_nan=True)
    assert np.isnan(want_s[2:5]).all() and np.isfinite(np.delete(want_s, [2, 3, 4])).all()


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("offset", [1, 2, 3, 5])
def test_rows_off_vector_alignment(torch, q8, t, offset):
    """Matrices that begin at any element of a buffer; outputs stay inside theirs."""
    rows, cols = 6, 1301
    buf = randn(torch, 9, rows * cols + 16, t=t)
    x = buf[offset:offset + rows * cols].view(rows, cols)
    q, s = q8.quantize(x)
    want_q, want_s = ref.padded_codes(f32(x))
    assert np.array_equal(q.cpu().numpy(), want_q) and np.array_equal(s.cpu().numpy(), want_s)
    out = torch.full((rows * cols + 16,), 7.0, dtype=x.dtype, device="cuda")
    q8.dequantize(q, s, cols, x.dtype, out=out[offset:offset + rows * cols].view(rows, cols))
    o = f64(out)
    assert (o[:offset] == 7).all() and (o[offset + rows * cols:] == 7).all()
    v = ref.values(want_q, want_s, cols)
    within(o[offset:offset + rows * cols].reshape(rows, cols), v, (ref.HALF_ULP[t] + U) * np.abs(v), "values")


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 127), (4, 128), (33, 1301), (2, 20000)])
def test_dequantize(torch, q8, t, rows, cols):
    q, s = codes(torch, 5, rows, cols)
    v = ref.values(q.cpu().numpy(), s.cpu().numpy(), cols)
    within(f64(q8.dequantize(q, s, cols, dtype_of(torch, t))), v, (ref.HALF_ULP[t] + U) * np.abs(v), "rows")
    sg = torch.rand((rows, ref.pitch(cols) // 128), generator=torch.Generator().manual_seed(1)).cuda()
    v = ref.values(q.cpu().numpy(), sg.cpu().numpy(), cols)
    within(f64(q8.dequantize(q, sg, cols, dtype_of(torch, t))), v,
           (ref.HALF_ULP[t] + U) * np.abs(v) + ref.SMALLEST[t], "groups")


NORMS = ([(1, c) for c in WIDTHS]
         + [(5, 129), (515, 513), (515, 2047), (515, 4095), (515, 8191), (70, 9001), (9, 40000)])


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rows,cols", NORMS)
@pytest.mark.parametrize("parts", ["all", "bare"])
def test_norm(torch, q8, t, rows, cols, parts):
    """parts: residual, gain and checkpoint, or none of them."""
    x = randn(torch, rows + cols, rows, cols, t=t, scale=2.0)
    n = q8.RMSNormQ8(rows, cols, x.dtype, eps=1e-5)
    res = gain = None
    h = f32(x)
    if parts == "all":
        res, gain = randn(torch, 11, rows, cols, t=t), 1 + randn(torch, 12, cols, t=t, scale=0.2)
        h = h + f32(res)                                           # binary32
    o = n.forward(x, res, gain, checkpoint=parts == "all")
    v = h * f32(gain) if gain is not None else h                   # binary32
    want_q, want_s = ref.padded_codes(v)
    assert np.array_equal(o.codes.cpu().numpy(), want_q)
    h64 = h.astype(np.float64)
    rstd = ((h64 ** 2).mean(axis=1) + np.float64(np.float32(1e-5))) ** -0.5
    within(f64(o.rstd), rstd, 68 * U * rstd, "rstd")
    within(f64(o.scales), want_s * rstd, 72 * U * want_s * rstd, "scales")
    if parts == "all":
        assert torch.equal(o.h.cpu(), torch.from_numpy(h).to(x.dtype))
        cq, cs = ref.checkpoint(h)
        assert np.array_equal(o.saved_codes.cpu().numpy(), cq)
        assert np.array_equal(o.saved_scales.cpu().numpy(), cs)
        if cols > 32768:                                           # (refused: the next test)
            return
        again = n.forward(x, res, gain, inplace=True)              # h over the residual
        assert again.h is res and torch.equal(res, o.h) and torch.equal(again.codes, o.codes)
        assert torch.equal(again.rstd, o.rstd) and again.saved_codes is None
    else:
        assert o.h is x and o.saved_codes is None


def test_norm_inplace_is_refused_where_rows_are_read_twice(torch, q8):
    from paper_2609_26077_amd import FMM_ERR_UNSUPPORTED, FmmError
    x = randn(torch, 1, 2, 40000)
    with pytest.raises(FmmError) as e:
        q8.RMSNormQ8(2, 40000, x.dtype).forward(x, x.clone(), inplace=True)
    assert e.value.status == FMM_ERR_UNSUPPORTED


@pytest.mark.parametrize("t", TYPES)
def test_norm_rows_that_cannot_be_normalized(torch, q8, t):
    """A zero row stays zero under eps; NaN and infinity give NaN rows and NaN groups, and leave the other rows alone."""
    rows, cols = 5, 300
    x = randn(torch, 2, rows, cols, t=t)
    x[1] = 0
    x[2, 299] = float("nan")
    x[3, 130] = float("inf")
    o = q8.RMSNormQ8(rows, cols, x.dtype).forward(x, checkpoint=True)
    y = f64(q8.dequantize(o.codes, o.scales, cols))
    assert (y[1] == 0).all() and np.isnan(y[2]).all() and np.isnan(y[3]).all()
    alone = q8.RMSNormQ8(1, cols, x.dtype)
    for r in (0, 4):
        p = alone.forward(x[r:r + 1])
        assert torch.equal(p.codes[0], o.codes[r]) and torch.equal(p.scales[0], o.scales[r])
    s = f64(o.saved_scales)
    assert np.isnan(s[2]).tolist() == [False, False, True] and np.isnan(s[3]).tolist() == [False, True, False]
    assert np.isfinite(s[[0, 1, 4]]).all()


def norm_case(torch, q8, t, rows, cols, gain=True, dh=True):
    x = randn(torch, rows + cols, rows, cols, t=t, scale=2.0)
    g = 1 + randn(torch, 21, cols, t=t, scale=0.3) if gain else None
    if gain:
        g[cols // 2] = 0
    n = q8.RMSNormQ8(rows, cols, x.dtype, eps=1e-5)
    o = n.forward(x, None, g, checkpoint=True)
    dy = randn(torch, 22, rows, cols, t=t, scale=0.1)
    d = randn(torch, 23, rows, cols, t=t, scale=0.1) if dh else None
    return n, x, g, o, dy, d


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("source", ["h", "saved"])
@pytest.mark.parametrize("rows,cols", NORMS + [(2100, 320), (1100, 1000)])
def test_norm_gradient(torch, q8, t, source, rows, cols):
    more = (rows + cols) % 2 == 0                        # with gain and dh, or without
    n, x, g, o, dy, dh = norm_case(torch, q8, t, rows, cols, more, more)
    if source == "h":
        h, given = f64(x), {"h": x}
    else:
        h, given = ref.values(o.saved_codes.cpu().numpy(), o.saved_scales.cpu().numpy(), cols), \
            {"saved": (o.saved_codes, o.saved_scales)}
    dx, dgain = n.backward(dy, o.rstd, g, dh=dh, **given)
    want, want_g, terms, terms_g = ref.norm_gradient(h, f64(o.rstd), f64(dy), f64(g) if more else 1.0,
                                                     f64(dh) if more else 0.0)
    within(f64(dx), want, 80 * U * terms + ref.HALF_ULP[t] * np.abs(want) + ref.SMALLEST[t], "dx")
    within(f64(dgain), want_g, (rows + 16) * U * terms_g, "dgain")
    again, again_g = n.backward(dy, o.rstd, g, dh=dh, **given)
    assert torch.equal(again, dx) and torch.equal(again_g, dgain)
    bare, none = n.backward(dy, o.rstd, g, dh=dh, need_gain=False, **given)
    assert none is None and torch.equal(bare, dx)


def test_norm_gradient_against_differences(torch, q8):
    """L(h, g) = sum dy y(h, g) + sum dh h in binary64, differenced along random
    directions: a central difference of step e is off by e^2 of third
    derivatives, here under 1e-6 of the sum of magnitudes."""
    rows, cols = 7, 200
    n, x, g, o, dy, dh = norm_case(torch, q8, "fp32", rows, cols)
    dx, dgain = n.backward(dy, o.rstd, g, h=x, dh=dh)
    rng = np.random.default_rng(0)
    h0, g0, DY, DH = f64(x), f64(g), f64(dy), f64(dh)

    def loss(h, gain):
        rstd = ((h ** 2).mean(axis=1, keepdims=True) + np.float64(np.float32(1e-5))) ** -0.5
        return (DY * h * rstd * gain).sum() + (DH * h).sum()

    e = 1e-4
    for _ in range(8):
        d, dg = rng.standard_normal((rows, cols)), rng.standard_normal(cols)
        num = (loss(h0 + e * d, g0) - loss(h0 - e * d, g0)) / (2 * e)
        assert abs(num - (f64(dx) * d).sum()) <= 1e-5 * np.abs(f64(dx) * d).sum()
        num = (loss(h0, g0 + e * dg) - loss(h0, g0 - e * dg)) / (2 * e)
        assert abs(num - (f64(dgain) * dg).sum()) <= 1e-5 * np.abs(f64(dgain) * dg).sum()


def test_norm_gradient_of_no_rows(torch, q8):
    n = q8.RMSNormQ8(0, 50, torch.float32)
    e = torch.empty((0, 50), device="cuda")
    dx, dgain = n.backward(e, torch.empty(0, device="cuda"), h=e)
    assert dx.shape == (0, 50) and (dgain == 0).all()


# ---- the product ---------------------------------------------------------------------
def check_matmul(torch, q8, t, M, N, K, bias, seed=1):
    a, sa = codes(torch, seed, M, K)
    w, sw = codes(torch, seed + 1, N, K)
    b = randn(torch, seed + 2, N, scale=5.0) if bias else None
    C = q8.LinearQ8(M, N, K, dtype_of(torch, t)).matmul(a, sa, w, sw, b)
    acc = a.cpu().numpy().astype(np.int64) @ w.cpu().numpy().astype(np.int64).T
    p = acc * f64(sa)[:, None] * f64(sw)
    want = p + (f64(b) if bias else 0.0)
    assert tuple(C.shape) == (M, N)
    within(f64(C), want, 4 * U * np.abs(p) + (2 * U * np.abs(f64(b)) if bias else 0.0)
           + ref.HALF_ULP[t] * np.abs(want) + ref.SMALLEST[t], "C")


MATMULS = [(1, 1, 1), (1, 16, 128), (1, 1000, 4096), (2, 33, 129), (3, 64, 1000), (4, 130, 640), (5, 257, 2049),
           (8, 48, 8192), (15, 17, 100), (16, 512, 512), (17, 1, 127), (31, 300, 384), (33, 96, 2000), (48, 1031, 256),
           (64, 2048, 1024), (65, 65, 65), (100, 4100, 300), (127, 129, 128), (128, 128, 4096), (129, 200, 1301),
           (255, 257, 256), (300, 4097, 640), (1000, 1302, 1472), (513, 8200, 130), (2049, 2050, 200), (4096, 4096, 256)]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("M,N,K", MATMULS)
def test_matmul(torch, q8, t, M, N, K):
    check_matmul(torch, q8, t, M, N, K, bias=(M + N + K) % 2 == 0)


@pytest.mark.parametrize("M,N,K", [(0, 5, 7), (5, 0, 7), (4, 6, 0), (40, 70, 0)])
def test_matmul_of_nothing(torch, q8, M, N, K):
    check_matmul(torch, q8, "fp32", M, N, K, bias=True)


@pytest.mark.parametrize("M", [1, 3, 20, 70, 200])
def test_matmul_longest_sum(torch, q8, M):
    """Every code -128 over the longest contracted axis: the largest int32 sum, 131071 2^14."""
    K, N = 131071, 40
    a = torch.zeros((M, ref.pitch(K)), dtype=torch.int8, device="cuda")
    w = torch.zeros((N, ref.pitch(K)), dtype=torch.int8, device="cuda")
    a[:, :K] = -128
    w[:, :K] = -128
    C = q8.LinearQ8(M, N, K, torch.float32).matmul(a, torch.ones(M, device="cuda"), w, torch.ones(N, device="cuda"))
    assert (f64(C) == 131071.0 * 2 ** 14).all()


def test_matmul_propagates_rows_without_a_scale(torch, q8):
    M, N, K = 5, 70, 300
    x, v = randn(torch, 1, M, K), randn(torch, 2, N, K)
    x[3, 7] = float("inf")
    v[11, 0] = float("nan")
    C = f64(q8.LinearQ8(M, N, K, torch.float32).matmul(*q8.quantize(x), *q8.quantize(v)))
    nan = np.zeros((M, N), bool)
    nan[3] = True
    nan[:, 11] = True
    assert np.array_equal(np.isnan(C), nan)


@pytest.mark.parametrize("M,N,K", [(1, 100, 300), (20, 33, 500), (70, 130, 256), (300, 257, 384)])
def test_matmul_writes_only_its_output(torch, q8, M, N, K):
    a, sa = codes(torch, 1, M, K)
    w, sw = codes(torch, 2, N, K)
    for t in TYPES:
        buf = torch.full((M * N + 64,), 3.0, dtype=dtype_of(torch, t), device="cuda")
        C = buf[7:7 + M * N].view(M, N)
        lin = q8.LinearQ8(M, N, K, C.dtype)
        lin.matmul(a, sa, w, sw, C=C)
        assert (buf[:7] == 3).all() and (buf[7 + M * N:] == 3).all()
        assert torch.equal(C, lin.matmul(a, sa, w, sw))


# ---- the linear gradients --------------------------------------------------------------
GRADS = [(1, 1, 1), (1, 100, 300), (2, 64, 64), (7, 130, 65), (33, 1, 200), (64, 64, 128), (65, 63, 1), (100, 257, 129),
         (128, 512, 256), (256, 2048, 2048), (300, 200, 1000), (1000, 1302, 1472), (2050, 130, 260), (130, 4100, 520),
         (640, 4096, 4160)]


def check_grad(torch, q8, t, M, N, K, need_x=True, need_w=True, bias=True):
    a, sa = codes(torch, 1, M, K)
    w, sw = codes(torch, 2, N, K)
    dy = randn(torch, 3, M, N, t=t, scale=0.1)
    lin = q8.LinearQ8(M, N, K, dy.dtype)
    dx, dw, db = lin.backward(dy, a, sa, w, sw, need_x=need_x, need_w=need_w, bias=bias)
    DY, A, W = f64(dy), ref.values(a.cpu().numpy(), f64(sa), K), ref.values(w.cpu().numpy(), f64(sw), K)
    r = ROUNDING[t] + 2.0 ** -19
    for got, P, Q, name in ((dx, DY, W, "dX"), (dw, DY.T, A, "dW")):
        if got is None:
            continue
        want, S = P @ Q, np.abs(P) @ np.abs(Q)
        within(f64(got), want, (r + P.shape[1] * U) * S + ref.HALF_ULP[t] * np.abs(want) + ref.SMALLEST[t], name)
    if bias:
        within(f64(db), DY.sum(axis=0), (M + 4) * U * np.abs(DY).sum(axis=0), "dbias")
    assert (dx is not None) == need_x and (dw is not None) == need_w and (db is not None) == bias
    return lin, (dy, a, sa, w, sw), (dx, dw, db)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("M,N,K", GRADS)
def test_linear_gradient(torch, q8, t, M, N, K):
    lin, args, first = check_grad(torch, q8, t, M, N, K)
    for got, again in zip(first, lin.backward(*args, bias=True)):
        assert torch.equal(got, again)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("x,w,b", [(True, False, False), (False, True, False), (False, False, True), (True, False, True),
                                   (False, True, True), (False, False, False)])
def test_linear_gradient_of_what_is_wanted(torch, q8, t, x, w, b):
    check_grad(torch, q8, t, 70, 130, 200, need_x=x, need_w=w, bias=b)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("x,w", [(True, True), (True, False), (False, True)])
@pytest.mark.parametrize("M,N,K", [(4096, 4100, 17), (4100, 130, 70), (70, 4100, 130)])
def test_linear_gradient_in_runs(torch, q8, t, x, w, M, N, K):
    """Few outputs and long sums, whose contracted axes are split: of both products, and of each where only it is wanted."""
    check_grad(torch, q8, t, M, N, K, need_x=x, need_w=w)


@pytest.mark.parametrize("M,N,K", [(0, 5, 7), (5, 0, 7), (4, 6, 0)])
def test_linear_gradient_of_nothing(torch, q8, M, N, K):
    check_grad(torch, q8, "bf16", M, N, K)


def test_linear_gradient_against_differences(torch, q8):
    """The layer is bilinear in the values its operands stand for, so a central difference of its loss is exact."""
    M, N, K = 40, 33, 50
    lin, (dy, a, sa, w, sw), (dx, dw, db) = check_grad(torch, q8, "fp32", M, N, K)
    DY, A, W = f64(dy), ref.values(a.cpu().numpy(), f64(sa), K), ref.values(w.cpu().numpy(), f64(sw), K)
    rng = np.random.default_rng(0)

    def loss(A, W, b):
        return (DY * (A @ W.T + b)).sum()

    b0, e = np.zeros(N), 1e-2
    for _ in range(4):
        d = rng.standard_normal((M, K))
        num = (loss(A + e * d, W, b0) - loss(A - e * d, W, b0)) / (2 * e)
        assert abs(num - (f64(dx) * d).sum()) <= 1e-5 * np.abs(f64(dx) * d).sum()
        d = rng.standard_normal((N, K))
        num = (loss(A, W + e * d, b0) - loss(A, W - e * d, b0)) / (2 * e)
        assert abs(num - (f64(dw) * d).sum()) <= 1e-5 * np.abs(f64(dw) * d).sum()
        d = rng.standard_normal(N)
        num = (loss(A, W, b0 + e * d) - loss(A, W, b0 - e * d)) / (2 * e)
        assert abs(num - (f64(db) * d).sum()) <= 1e-5 * np.abs(f64(db) * d).sum()


@pytest.mark.parametrize("t", TYPES)
def test_linear_gradient_propagates_what_is_not_finite(torch, q8, t):
    """An infinity of dY reaches its row of dX, its column's row of dW and its bias entry, and nothing else."""
    M, N, K = 70, 66, 100
    a, sa = codes(torch, 1, M, K)
    w, sw = codes(torch, 2, N, K)
    a[:, :K].clamp_(min=1)     # no 0 x infinity among the terms
    w[:, :K].clamp_(min=1)
    dy = randn(torch, 3, M, N, t=t)
    dy[5, 9] = float("inf")
    dy[64, 65] = float("nan")
    dx, dw, db = (f64(v) for v in q8.LinearQ8(M, N, K, dy.dtype).backward(dy, a, sa, w, sw, bias=True))
    assert (dx[5] == np.inf).all() and np.isnan(dx[64]).all() and np.isfinite(np.delete(dx, [5, 64], axis=0)).all()
    assert (dw[9] == np.inf).all() and np.isnan(dw[65]).all() and np.isfinite(np.delete(dw, [9, 65], axis=0)).all()
    assert db[9] == np.inf and np.isnan(db[65]) and np.isfinite(np.delete(db, [9, 65])).all()


# ---- streams and graphs ------------------------------------------------------------------
def layer(torch, q8, M, N, K):
    norm, lin = q8.RMSNormQ8(M, K, torch.bfloat16), q8.LinearQ8(M, N, K, torch.bfloat16)
    w, sw = q8.quantize(randn(torch, 5, N, K, t="bf16"))
    gain = 1 + randn(torch, 6, K, t="bf16", scale=0.1)

    def step(x, res, dc, stream=None):
        o = norm.forward(x, res, gain, checkpoint=True, stream=stream)
        c = lin.matmul(o.codes, o.scales, w, sw, stream=stream)
        dy, dw, db = lin.backward(dc, o.codes, o.scales, w, sw, bias=True, stream=stream)
        dx, dgain = norm.backward(dy, o.rstd, gain, saved=(o.saved_codes, o.saved_scales), dh=res, stream=stream)
        return o.h, c, dw, db, dx, dgain

    return step


@pytest.mark.parametrize("M,N,K", [(1, 300, 520), (200, 300, 520)])
def test_streams(torch, q8, M, N, K):
    """The same results on a stream other than the inputs' own, given by name or made current."""
    step = layer(torch, q8, M, N, K)
    args = [randn(torch, s, M, K, t="bf16") for s in (1, 2)] + [randn(torch, 3, M, N, t="bf16")]
    want = step(*args)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    named = step(*args, stream=side)
    side.synchronize()
    by_handle = step(*args, stream=side.cuda_stream)
    side.synchronize()
    with torch.cuda.stream(side):
        current = step(*args)
    side.synchronize()
    for got in (named, by_handle, current):
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("M,N,K", [(1, 300, 520), (200, 300, 520)])
def test_graph_replays(torch, q8, M, N, K):
    """Captured once, replayed on new inputs with eager work between, each replay against the eager result."""
    step = layer(torch, q8, M, N, K)
    args = [randn(torch, s, M, K, t="bf16") for s in (1, 2)] + [randn(torch, 3, M, N, t="bf16")]
    step(*args)               # (the workspaces come with the first call)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(*args)
    for k in range(4):
        for i, x in enumerate(args):
            x.copy_(randn(torch, 100 * k + i, *x.shape, t="bf16"))
        graph.replay()
        torch.cuda.synchronize()
        got = [v.clone() for v in out]
        want = step(*args)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), k


# ---- offsets beyond 32 bits ----------------------------------------------------------------
def test_rows_beyond_32_bit_offsets(torch, q8):
    """More than 2^31 elements, and more than 2^32 bytes: the last rows are as if they were alone."""
    rows, cols = 70000, 32768
    x = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
    tail = randn(torch, 4, 3, cols, t="bf16")
    x[-3:] = tail
    q, s = q8.quantize(x)
    want_q, want_s = q8.quantize(tail)
    assert torch.equal(q[-3:], want_q) and torch.equal(s[-3:], want_s)
    assert not q[:-3].any() and (s[:-3] == s[0]).all()
    del q, s
    n, alone = q8.RMSNormQ8(rows, cols, x.dtype), q8.RMSNormQ8(3, cols, x.dtype)
    o, w = n.forward(x, checkpoint=True), alone.forward(tail, checkpoint=True)
    for got, want in zip(o[1:], w[1:]):
        assert torch.equal(got[-3:], want)
    dx, dgain = n.backward(x, o.rstd, saved=(o.saved_codes, o.saved_scales))
    want_dx, want_g = alone.backward(tail, w.rstd, saved=(w.saved_codes, w.saved_scales))
    assert torch.equal(dx[-3:], want_dx) and not dx[:-3].any()
    within(f64(dgain), f64(want_g), 8 * U * np.abs(f64(want_g)) + 1e-6, "dgain")
    v = q8.dequantize(o.codes, o.scales, cols, torch.bfloat16)
    assert torch.equal(v[-3:], q8.dequantize(w.codes, w.scales, cols, torch.bfloat16))


@pytest.mark.parametrize("M,N,K", [(300000, 8192, 130), (8193, 270000, 64)])
def test_matmul_beyond_32_bit_offsets(torch, q8, M, N, K):
    a, sa = torch.zeros((M, ref.pitch(K)), dtype=torch.int8, device="cuda"), torch.ones(M, device="cuda")
    w, sw = torch.zeros((N, ref.pitch(K)), dtype=torch.int8, device="cuda"), torch.ones(N, device="cuda")
    ta, _ = codes(torch, 1, 300, K)
    tw, _ = codes(torch, 2, 300, K)
    a[-300:], w[-300:] = ta, tw
    C = q8.LinearQ8(M, N, K, torch.bfloat16).matmul(a, sa, w, sw)
    want = q8.LinearQ8(300, 300, K, torch.bfloat16).matmul(ta, sa[:300].clone(), tw, sw[:300].clone())
    assert torch.equal(C[-300:, -300:], want)
    assert not C[:-300].any() and not C[:, :-300].any()


# ---- the example -----------------------------------------------------------------------------
def test_feedforward_example(torch, q8):
    """It learns, and a token's output is that of the same layer evaluated in
    binary64 on the values its codes stand for, but for the roundings of u and
    silu(u): silu's slope is at most 1.1 and a code's half step 1/254 of its row's
    largest magnitude."""
    from examples.q8_feedforward import FeedForward, train
    width, hidden = 256, 520
    layer = FeedForward(width, hidden)
    losses, x = train(layer, 300, 25)
    assert losses[-1] < 0.5 * losses[0] and np.isfinite(losses).all()
    token = x[:1]
    out, h, kept = layer.forward(token, torch.zeros_like(token))
    assert kept is None and torch.equal(h, token)
    o = q8.RMSNormQ8(1, width).forward(token, None, layer.gain_in)
    y = ref.values(o.codes.cpu().numpy(), o.scales.cpu().numpy(), width)
    W1 = ref.values(layer.q1[0].cpu().numpy(), layer.q1[1].cpu().numpy(), width)
    W2 = ref.values(layer.q2[0].cpu().numpy(), layer.q2[1].cpu().numpy(), hidden)
    u = y @ W1.T + f64(layer.b1)
    s = u / (1 + np.exp(-u))
    du = 2.0 ** -8 * np.abs(u) * 1.1 + 2.0 ** -8 * np.abs(s)          # u and silu(u) in bf16
    ds = du + np.abs(s).max() * (1 + 2.0 ** -8) / 254 + 2.0 ** -8 * np.abs(s)
    want = s @ W2.T + f64(layer.b2)
    within(f64(out), want, ds @ np.abs(W2).T + 2.0 ** -8 * np.abs(want) + 1e-6, "out")


# ---- the binding under the wrappers ------------------------------------------------------------
@pytest.mark.parametrize("t", TYPES)
def test_binding_calls_are_what_the_wrappers_call(torch, q8, t):
    """The functions named after the C entry points, on tensors, and outputs that the caller provides."""
    import paper_2609_26077_amd as fm
    M, N, K = 9, 70, 200
    dt, P = dtype_of(torch, t), ref.pitch(K)
    ty = q8.TYPES[dt]
    x, res, dy = randn(torch, 1, M, K, t=t), randn(torch, 2, M, K, t=t), randn(torch, 3, M, N, t=t)
    gain = 1 + randn(torch, 4, K, t=t, scale=0.1)
    new = lambda *s, d=dt: torch.empty(s, dtype=d, device="cuda")
    i8, f4 = torch.int8, torch.float32

    want_q, want_s = q8.quantize(x)
    q, s = new(M, P, d=i8), new(M, d=f4)
    a, b = q8.quantize(x, codes=q, scales=s)
    assert a is q and b is s and torch.equal(q, want_q) and torch.equal(s, want_s)
    q2, s2 = new(M, P, d=i8), new(M, d=f4)
    fm.fmm_q8_quantize(ty, M, K, x, q2, s2)
    assert torch.equal(q2, want_q) and torch.equal(s2, want_s)
    v = new(M, K)
    fm.fmm_q8_dequantize(ty, M, K, 0, q2, s2, v)
    assert torch.equal(v, q8.dequantize(want_q, want_s, K, dt))

    norm = q8.RMSNormQ8(M, K, dt)
    o = norm.forward(x, res, gain, checkpoint=True)
    h, rstd, saved, saved_s = new(M, K), new(M, d=f4), new(M, P, d=i8), new(M, P // 128, d=f4)
    fm.fmm_rmsnorm_q8(norm.desc, x, res, gain, h, q2, s2, saved, saved_s, rstd)
    for got, want in zip((h, q2, s2, rstd, saved, saved_s), o):
        assert torch.equal(got, want)
    dx, dg = new(M, K), new(K, d=f4)
    n = fm.fmm_rmsnorm_q8_backward_scratch_size(norm.desc)
    fm.fmm_rmsnorm_q8_backward(norm.desc, x, res, None, saved, saved_s, rstd, gain, dx, dg, new(max(n, 16), d=torch.uint8), n)
    for got, want in zip((dx, dg), norm.backward(x, o.rstd, gain, saved=(o.saved_codes, o.saved_scales), dh=res)):
        assert torch.equal(got, want)

    lin = q8.LinearQ8(M, N, K, dt)
    w, sw = codes(torch, 5, N, K)
    bias = randn(torch, 6, N)
    C = new(M, N)
    fm.fmm_q8_matmul(lin.desc, q2, s2, w, sw, bias, C)
    assert torch.equal(C, lin.matmul(q2, s2, w, sw, bias))
    n = fm.fmm_q8_linear_backward_scratch_size(lin.desc)
    gx, gw, gb = new(M, K), new(N, K), new(N, d=f4)
    fm.fmm_q8_linear_backward(lin.desc, dy, q2, s2, w, sw, gx, gw, gb, new(n, d=torch.uint8), n)
    for got, want in zip((gx, gw, gb), lin.backward(dy, q2, s2, w, sw, bias=True)):
        assert torch.equal(got, want)


@pytest.mark.parametrize("t,M,N,K", [("fp32", 1500, 1700, 100), ("bf16", 2047, 1999, 128), ("fp16", 2040, 1900, 129),
                                     ("bf16", 1900, 2000, 300), ("fp32", 1800, 2010, 500), ("fp16", 1283, 1411, 1030),
                                     ("bf16", 127, 30001, 520)])
def test_matmul_of_about_a_tile_a_unit(torch, q8, t, M, N, K):
    """Tiles enough for most compute units and no more, one step of the contracted axis to nine."""
    check_matmul(torch, q8, t, M, N, K, bias=K > 300)


@pytest.mark.parametrize("t,M,N,K", [("bf16", 1030, 1100, 1300), ("fp16", 900, 700, 1500), ("fp32", 300, 2000, 900),
                                     ("fp32", 1283, 200, 1411), ("bf16", 1900, 33, 2000), ("bf16", 33, 1900, 2000)])
@pytest.mark.parametrize("x,w", [(True, True), (True, False), (False, True)])
def test_linear_gradient_of_about_a_tile_a_unit(torch, q8, t, x, w, M, N, K):
    check_grad(torch, q8, t, M, N, K, need_x=x, need_w=w)


# ---- the default stream by its handle -------------------------------------------------------------
def test_default_stream_by_handle(torch, q8):
    """Handle 0 is torch's default stream: calls on it come after what writes their
    inputs there, and before what reads their outputs."""
    M, N, K = 64, 96, 1024
    assert torch.cuda.current_stream().cuda_stream == 0
    lin = q8.LinearQ8(M, N, K, torch.float32)
    w, sw = q8.quantize(randn(torch, 2, N, K))
    x, late = torch.zeros((M, K), device="cuda"), randn(torch, 1, M, K)
    want = lin.matmul(*q8.quantize(late), w, sw)
    torch.cuda.synchronize()
    torch.cuda._sleep(20_000_000)                 # some ms: the write of x is still to come when the calls are made
    x.copy_(late)
    got = lin.matmul(*q8.quantize(x, stream=0), w, sw, stream=0).clone()
    assert torch.equal(got, want)


def test_one_object_on_two_streams(torch, q8):
    """Gradients of the same objects, under way on two streams at once."""
    M, N, K = 4100, 130, 520
    norm, lin = q8.RMSNormQ8(M, K, torch.bfloat16), q8.LinearQ8(M, N, K, torch.bfloat16)
    w, sw = codes(torch, 5, N, K)
    sides = [torch.cuda.Stream(), torch.cuda.Stream()]
    inputs = []
    for s in (10, 20):
        a, sa = codes(torch, s, M, K)
        h, dh = randn(torch, s + 1, M, K, t="bf16"), randn(torch, s + 2, M, K, t="bf16")
        inputs.append((randn(torch, s + 3, M, N, t="bf16", scale=0.1), a, sa, h, dh, randn(torch, s + 4, M).abs() + 0.5))

    def both(dy, a, sa, h, dh, rstd, stream=None):
        return (*norm.backward(dh, rstd, h=h, stream=stream), *lin.backward(dy, a, sa, w, sw, bias=True, stream=stream))

    want = [both(*i) for i in inputs]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(8):
        for k in (0, 1):
            got[k].append(both(*inputs[k], stream=sides[k]))
    torch.cuda.synchronize()
    for k in (0, 1):
        for out in got[k]:
            assert all(torch.equal(a, b) for a, b in zip(out, want[k]))


@pytest.mark.parametrize("t", TYPES)
def test_linear_gradient_near_the_largest_float(torch, q8, t):
    """Finite products with a scale, past what bfloat16 rounds to infinity: a sum with
    one term of 1 or -1 times such a value is that value, and one of zeros is zero."""
    M, N, K = 70, 66, 100
    big = float(np.finfo(np.float32).max)
    a, sa = codes(torch, 1, M, K)
    w, sw = codes(torch, 2, N, K)
    a[:, :K] = torch.sign(a[:, :K])
    w[:, :K] = torch.sign(w[:, :K])
    sa[:], sw[:] = 1, 1
    dy = torch.zeros((M, N), dtype=dtype_of(torch, t), device="cuda")
    if t == "fp32":
        dy[5, 9], dy[64, 65], dy[6, 10] = big, -big, 3.397e38
    elif t == "fp16":
        dy[5, 9], dy[64, 65], dy[6, 10] = 65504.0, -65504.0, 65504.0
        sa[[5, 64, 6]] = sw[[9, 65, 10]] = 5.19e33          # (times 65504: 3.39966e38)
    else:
        dy[5, 9], dy[64, 65], dy[6, 10] = 1.0, -1.0, 1.0
        a[5, :K] = w[9, :K] = 127
        a[64, :K] = w[65, :K] = -127
        sa[[5, 64, 6]] = sw[[9, 65, 10]] = big / 127
    lin = q8.LinearQ8(M, N, K, dy.dtype)
    dx, dw, _ = lin.backward(dy, a, sa, w, sw)
    for got, P, Q, name in ((dx, f64(dy) * f64(sw), f64(w)[:, :K], "dX"), (dw, (f64(dy) * f64(sa)[:, None]).T, f64(a)[:, :K], "dW")):
        want = P @ Q
        r = ROUNDING[t] + 2.0 ** -19 + 2.0 ** -7 * (t == "bf16")       # (bfloat16's largest number is 2^-8 below its power of two)
        if t == "fp16":                                                # what fp16 holds of it
            want = np.where(np.abs(want) > 65520, np.copysign(np.inf, want), want)
            assert np.array_equal(f64(got), want), name
        else:
            within(f64(got), want, r * np.abs(want) + ref.HALF_ULP[t] * np.abs(want), name)


# ---- every kernel that the rules choose --------------------------------------------------------------
# The shapes are chosen for a device of 256 compute units; each test first asserts which
# kernel its sizes take (and a CPU test that the lists hold every kernel).  The references are products in binary64 on the GPU: sums of
# integers, exact in any order, for the int8 product.
def check_product(torch, q8, t, kernel, M, N, K):
    import paper_2609_26077_amd as fm
    lin = q8.LinearQ8(M, N, K, dtype_of(torch, t))
    assert fm.fmm_q8_matmul_kernel(lin.desc) == kernel
    a, sa = codes(torch, M, M, K)
    w, sw = codes(torch, N + 1, N, K)
    b = randn(torch, 3, N, scale=5.0)
    C = lin.matmul(a, sa, w, sw, b)
    wt, b64 = w[:, :K].double().t().contiguous(), b.double()
    for m in range(0, M, 2048):
        rows = slice(m, m + 2048)
        p = torch.mm(a[rows, :K].double(), wt) * sa[rows, None].double() * sw.double()
        want = p + b64
        bound = 4 * U * p.abs() + 2 * U * b64.abs() + ref.HALF_ULP[t] * want.abs() + ref.SMALLEST[t]
        err = (C[rows].double() - want).abs()
        assert bool((err <= bound).all()), f"rows from {m}: {float((err / bound).max()):.3g} of the bound"


PRODUCTS = (
    # (pieces of a wave: from none to enough that each slot is filled again)
    [("few_tokens_kernel 16x16", 13, 333, K) for K in (100, 1100, 2100, 4300)]
    + [("few_tokens_kernel 32x32", *s) for s in ((2140, 33, 430), (23, 4651, 560), (23, 4651, 1100), (2237, 33, 2700))]
    + [("few_tokens_kernel 48x32", *s) for s in ((37, 6201, 100), (36, 4651, 560), (48, 7168, 2048), (47, 4651, 1500),
                                                 (4177, 33, 2700))]
    + [("matmul_kernel 64x64", *s) for s in ((49, 8200, 100), (49, 9300, 200), (101, 6201, 300), (101, 6201, 430),
                                             (49, 7203, 560), (49, 7200, 700), (49, 8200, 800), (51, 6203, 2700))]
    + [("matmul_kernel 128x128 ahead", *s) for s in ((200, 8200, 100), (200, 8200, 200), (199, 7201, 300), (153, 9301, 430),
                                                     (140, 9300, 560), (141, 9303, 700), (140, 9300, 2700))]
    + [("matmul_kernel 128x128", *s) for s in ((782, 4651, 100), (394, 8200, 200), (395, 8201, 300), (394, 8203, 430),
                                               (394, 8200, 560), (391, 8207, 700), (394, 8200, 2700))]
    + [("matmul_kernel 256x256", *s) for s in ((20001, 9003, 100), (9001, 9003, 200), (9001, 9003, 300), (9001, 8963, 430),
                                               (5001, 5003, 560), (3498, 6203, 700), (4096, 4096, 1000), (1946, 4651, 2700))])


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("kernel,M,N,K", PRODUCTS)
def test_each_product_kernel(torch, q8, t, kernel, M, N, K):
    """Each workgroup shape over one step of the contracted axis and many, with ragged edges."""
    check_product(torch, q8, t, kernel, M, N, K)


# kernel, runs of dX and dW (None: whatever they are), sizes, what is wanted; each for the types named
GRADIENTS = (
    [("grad_kernel 64x64 64x64", *r) for r in (
        ((1, 1), (33, 35, 17), (1, 1), TYPES), ((8, 2), (200, 700, 17), (1, 1), ["fp32"]),
        ((4, 2), (200, 700, 17), (1, 1), ["fp16"]), ((1, 16), (1700, 33, 17), (0, 1), ["fp32"]),
        ((1, 8), (1700, 33, 17), (0, 1), ["fp16"]), ((1, 4), (1700, 33, 17), (0, 1), ["bf16"]),
        ((16, 1), (33, 1700, 17), (1, 0), ["fp32"]), ((8, 1), (33, 1700, 17), (1, 0), ["fp16"]),
        ((4, 1), (33, 1700, 17), (1, 0), ["bf16"]))]
    + [("grad_kernel 64x64 128x128", *r) for r in (
        ((1, 1), (130, 333, 3000), (1, 1), ["fp32"]), ((8, 1), (33, 2600, 1302), (1, 1), ["fp32"]),
        ((1, 8), (5200, 2050, 130), (0, 1), ["fp32"]), ((1, 1), (70, 1700, 3000), (1, 1), ["bf16"]),
        ((4, 1), (33, 5200, 2100), (1, 1), ["bf16"]), ((1, 4), (4100, 4100, 130), (0, 1), ["fp16"]),
        ((2, 1), (33, 1700, 3000), (1, 1), ["fp16"]))]
    + [("grad_kernel 128x128 64x64", *r) for r in (
        ((1, 1), (333, 130, 3000), (1, 1), ["fp32"]), ((1, 8), (2600, 33, 1302), (1, 1), ["fp32"]),
        ((1, 4), (5200, 33, 2100), (1, 1), ["bf16"]), ((1, 2), (1700, 33, 3000), (1, 1), ["fp16"]),
        ((8, 1), (2050, 5200, 130), (1, 0), ["fp32"]), ((4, 1), (4100, 4100, 130), (1, 0), ["fp16"]))]
    + [("grad_kernel 128x128 128x128", runs, s, (1, 1), t) for runs, s, t in (
        ((1, 1), (333, 520, 4160), TYPES), ((1, 8), (2050, 70, 1302), ["fp32"]), ((8, 1), (70, 2050, 1302), ["fp32"]),
        ((4, 2), (2050, 4100, 130), ["fp32"]), ((4, 4), (4100, 4100, 70), ["fp16"]), ((8, 1), (70, 5200, 1302), ["bf16"]))]
    + [("grad_kernel 128x128 128x128 ahead", *r) for r in (
        ((1, 1), (200, 201, 4160), (1, 1), TYPES), ((16, 1), (70, 2050, 520), (1, 1), ["fp32"]),
        ((8, 8), (1700, 2050, 17), (1, 1), ["fp32"]), ((8, 4), (1700, 4100, 17), (1, 1), ["fp16"]),
        ((8, 2), (1290, 5200, 70), (1, 1), ["bf16"]), ((1, 16), (4100, 1700, 17), (0, 1), ["fp32"]),
        ((1, 1), (2050, 33, 1302), (1, 0), ["fp16", "fp32"]))]
    + [("grad_kernel 256x256 256x256", *r) for r in (
        ((1, 1), (1000, 1290, 4161), (1, 1), ["fp32"]), ((1, 1), (640, 4096, 4160), (0, 1), TYPES),
        ((1, 1), (4100, 333, 3001), (1, 0), ["fp16", "fp32"]), ((1, 8), (5200, 130, 3000), (1, 1), ["fp32"]),
        ((8, 1), (130, 5200, 3000), (1, 1), ["fp32"]), ((1, 1), (4096, 4096, 4096), (1, 1), TYPES),
        ((1, 1), (4033, 4031, 3903), (1, 1), TYPES))])
GRADIENTS = [(t, kernel, runs, s, w) for kernel, runs, s, w, types in GRADIENTS for t in types]


def gradient_plan(torch, q8, t, kernel, runs, sizes, wanted):
    import paper_2609_26077_amd as fm
    lin = q8.LinearQ8(*sizes, dtype_of(torch, t))
    assert fm.fmm_q8_linear_backward_kernel(lin.desc, *wanted) == (kernel, runs)
    return lin


@pytest.mark.parametrize("t,kernel,runs,sizes,wanted", GRADIENTS)
def test_each_gradient_kernel(torch, q8, t, kernel, runs, sizes, wanted):
    """Dense codes, to the bound of the module's head."""
    lin = gradient_plan(torch, q8, t, kernel, runs, sizes, wanted)
    M, N, K = sizes
    a, sa = codes(torch, 1, M, K)
    w, sw = codes(torch, 2, N, K)
    dy = randn(torch, 3, M, N, t=t, scale=0.1)
    dx, dw, db = lin.backward(dy, a, sa, w, sw, need_x=bool(wanted[0]), need_w=bool(wanted[1]), bias=True)
    D, A, W = dy.double(), a[:, :K].double() * sa[:, None].double(), w[:, :K].double() * sw[:, None].double()
    r = ROUNDING[t] + 2.0 ** -19
    for got, P, Q, name in ((dx, D, W, "dX"), (dw, D.t().contiguous(), A, "dW")):
        if got is None:
            continue
        want, S = torch.mm(P, Q), torch.mm(P.abs(), Q.abs())
        bound = (r + P.shape[1] * U) * S + ref.HALF_ULP[t] * want.abs() + ref.SMALLEST[t]
        err = (got.double() - want).abs()
        assert bool((err <= bound).all()), f"{name}: {float((err / bound).max()):.3g} of the bound"
    within(f64(db), f64(D.sum(dim=0)), (M + 4) * U * f64(D.abs().sum(dim=0)), "dbias")


@pytest.mark.parametrize("t,kernel,runs,sizes,wanted", GRADIENTS)
def test_each_part_of_a_gradient_counts(torch, q8, t, kernel, runs, sizes, wanted):
    """Codes with one entry a column: an output is one term, dY s q, which every part of
    dY s has to reach, wherever along the contracted axis it is.  The factors are such
    that the parts hold all of dY s (24 bits for fp32, 16 for fp16; bf16's q s has 8) and
    that the term is exact in fp32: outputs are equal to it, rounded once."""
    lin = gradient_plan(torch, q8, t, kernel, runs, sizes, wanted)
    M, N, K = sizes
    g = torch.Generator().manual_seed(7)

    def pick(values, *shape):
        return torch.tensor(values, dtype=torch.float64)[torch.randint(0, len(values), shape, generator=g)]

    def one_hot(rows):
        at, q = torch.randint(0, rows, (K,), generator=g), pick([-128, -64, -4, -2, -1, 1, 2, 8, 32, 64], K)
        full = torch.zeros((rows, ref.pitch(K)), dtype=torch.int8)
        full[at, torch.arange(K)] = q.to(torch.int8)
        return full.cuda(), at.cuda(), q.cuda()

    powers = [2.0 ** e for e in range(-3, 4)]
    scales = powers if t != "fp16" else [m / 32 for m in range(17, 32, 2)]     # (fp16: 11 bits of dY, 5 of s)
    if t == "fp32":
        dy = (torch.randint(-2 ** 24 + 1, 2 ** 24, (M, N), generator=g) | 1).double() * 2.0 ** -20
    else:
        bits = 11 if t == "fp16" else 8
        dy = (torch.randint(2 ** (bits - 1), 2 ** bits, (M, N), generator=g) | 1).double() * 2.0 ** -bits * pick([-1, 1], M, N)
    dy, sa, sw = dy.cuda(), pick(scales, M).cuda(), pick(scales, N).cuda()
    a, m, qa = one_hot(M)
    w, n, qw = one_hot(N)
    dt = dtype_of(torch, t)
    dx, dw, _ = lin.backward(dy.to(dt), a, sa.float(), w, sw.float(), need_x=bool(wanted[0]), need_w=bool(wanted[1]))
    if dx is not None:
        assert torch.equal(dx, ((dy * sw)[:, n] * qw).float().to(dt))
    if dw is not None:
        assert torch.equal(dw, ((dy * sa[:, None])[m].t() * qa).float().to(dt))


# ---- the norm over many rows ------------------------------------------------------------------------
@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("source", ["h", "saved"])
@pytest.mark.parametrize("rows,cols", [
    # 768 workgroups of 256 threads (16-bit types; 512 for fp32), 8 rows and more for each, the last ones fewer
    (8192, 1300), (6500, 4095), (6144, 2049),
    # 512 workgroups, three rows for each and more; 512 and 1024 threads a row: 256 and 128 workgroups
    (1700, 3001), (2011, 1500), (1000, 6001), (700, 12001),
    # four rows a workgroup at once, 512 and 768 workgroups
    (9003, 700), (26001, 300), (25001, 520)])
def test_norm_gradient_of_many_rows(torch, q8, t, source, rows, cols):
    """Workgroups that walk many rows, to the bounds of the module's head; the reference in binary64 on the GPU."""
    n, x, g, o, dy, dh = norm_case(torch, q8, t, rows, cols)
    if source == "h":
        h, given = x.double(), {"h": x}
    else:
        h = (o.saved_codes.view(rows, -1, 128).double() * o.saved_scales[:, :, None].double()).view(rows, -1)[:, :cols]
        given = {"saved": (o.saved_codes, o.saved_scales)}
    dx, dgain = n.backward(dy, o.rstd, g, dh=dh, **given)
    r = o.rstd[:, None].double()
    xh, d = h * r, dy.double()
    w = d * g.double()
    c = (w * xh).mean(dim=1, keepdim=True)
    want = r * (w - xh * c) + dh.double()
    terms = r * (w.abs() + xh.abs() * (w * xh).abs().mean(dim=1, keepdim=True)) + dh.double().abs()
    err, bound = (dx.double() - want).abs(), 80 * U * terms + ref.HALF_ULP[t] * want.abs() + ref.SMALLEST[t]
    assert bool((err <= bound).all()), f"dx: {float((err / bound).max()):.3g} of the bound"
    within(f64(dgain), f64((d * xh).sum(dim=0)), (rows + 16) * U * f64((d * xh).abs().sum(dim=0)), "dgain")
    again, again_g = n.backward(dy, o.rstd, g, dh=dh, **given)
    assert torch.equal(again, dx) and torch.equal(again_g, dgain)


@pytest.mark.parametrize("rows,cols", [((1 << 20) + 5, 1100), ((1 << 22) + 7, 72)])
def test_rows_beyond_a_launch(torch, q8, rows, cols):
    """More rows than a launch has places for: workgroups go on to further rows, whose
    results are those of the same rows in calls of their own."""
    x = torch.randn((rows, cols), generator=torch.Generator("cuda").manual_seed(1), device="cuda", dtype=torch.bfloat16)
    gain = 1 + randn(torch, 2, cols, t="bf16", scale=0.1)
    q, s = q8.quantize(x)
    o = q8.RMSNormQ8(rows, cols, x.dtype).forward(x, x, gain, checkpoint=True)
    for r0 in range(0, rows, 1 << 19):
        part = x[r0:r0 + (1 << 19)]
        want_q, want_s = q8.quantize(part)
        assert torch.equal(q[r0:r0 + len(part)], want_q) and torch.equal(s[r0:r0 + len(part)], want_s)
        want = q8.RMSNormQ8(len(part), cols, x.dtype).forward(part, part, gain, checkpoint=True)
        for got, v in zip(o, want):
            assert torch.equal(got[r0:r0 + len(part)], v)


@pytest.mark.parametrize("t", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(5, 300), (600, 4096), (3, 33000)])
def test_norm_of_small_rows(torch, q8, t, rows, cols):
    """Rows far below 1e-12, eps 0: y is of order 1 and its codes, and the checkpoint's of h, are the nearest
    multiples of a 127th of the largest magnitude, to the bar of the codes' rule; so is a gradient from them."""
    size = 10.0 ** torch.linspace(-10, -17, rows)
    x = (randn(torch, 1, rows, cols).cpu() * size[:, None]).to(dtype_of(torch, t)).cuda()
    g = 1 + randn(torch, 2, cols, t=t, scale=0.2)
    n = q8.RMSNormQ8(rows, cols, x.dtype, eps=0.0)
    o = n.forward(x, None, g, checkpoint=True)
    h = f64(x)
    rstd = (h ** 2).mean(axis=1) ** -0.5
    within(f64(o.rstd), rstd, 68 * U * rstd, "rstd")
    y = h * rstd[:, None] * f64(g)
    amax = np.abs(y).max(axis=1)
    within(f64(o.scales), amax / 127, 76 * U * amax / 127, "scales")
    got = ref.values(o.codes.cpu().numpy(), f64(o.scales), cols)
    within(got, y, ((0.5 + 2.0 ** -15) * f64(o.scales) + 80 * U * amax)[:, None], "half a step of y")
    P = ref.pitch(cols)
    groups = np.pad(h, ((0, 0), (0, P - cols))).reshape(rows, -1, 128)
    want = np.abs(groups).max(axis=2) / 127
    within(f64(o.saved_scales), want, 2 * U * want, "the checkpoint's scales")
    kept = ref.values(o.saved_codes.cpu().numpy(), f64(o.saved_scales), cols)
    within(kept, h, np.repeat((0.5 + 2.0 ** -15) * f64(o.saved_scales), 128, axis=1)[:, :cols], "half a step of h")
