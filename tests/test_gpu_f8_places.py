"""Where the kernels of the e4m3 layers' products take their codes and scales from: each kernel, by
name, with scales that differ from block to block, from row to row and from expert to expert.

One code a row or column of an operand: every result is then one product of two codes and powers
of two, whose digits are one code's (the other being a power of two), so a code, a scale or an expert taken from
another place shows, and results are compared for equality.  Results of whole operands have the bars of test_gpu_f8."""
from __future__ import annotations

import pytest

from test_gpu_f8_kernels import GRADIENTS, PRODUCTS, TYPE, U, bound, dtype_of, product, within

pytestmark = pytest.mark.gpu

# more experts than a wave has lanes, under each of the tiles
PRODUCTS_OF_MANY = [
    ("few_tokens_kernel 16x16", "bf16", 64, 200, 40, 300),
    ("few_tokens_kernel 32x32", "fp32", 3000, 100, 140, 260),
    ("matmul_kernel 64x64", "bf16", 4000, 130, 257, 300),
    ("matmul_kernel 128x128", "fp16", 9000, 130, 520, 260),
    ("matmul_kernel 128x128", "fp32", 12000, 100, 1000, 300),
    ("matmul_kernel 256x256", "bf16", 33500, 66, 1000, 900),
]
GRADIENTS_OF_MANY = [
    ("grad_kernel 64x64 64x64", "fp32", 3000, 100, 140, 260, (1, 0)),
    ("grad_kernel 64x64 128x128", "fp16", 9000, 130, 520, 260, (0, 1)),
    ("grad_kernel 128x128 64x64", "bf16", 9000, 130, 520, 260, (1, 0)),
    ("grad_kernel 128x128 128x128", "fp32", 2000, 70, 1030, 520, (1, 1)),
    ("grad_kernel 256x256 256x256", "bf16", 33500, 66, 1000, 900, (1, 1)),
]
SOME_PRODUCTS, SOME_GRADIENTS = PRODUCTS + PRODUCTS_OF_MANY, GRADIENTS + GRADIENTS_OF_MANY


@pytest.fixture(scope="module")
def torch():
    import torch
    return torch


@pytest.fixture(scope="module")
def f8():
    from paper_2609_26077_amd import f8
    return f8


class Make:
    """Operands from a seed, on the device."""

    def __init__(self, torch, f8, seed):
        self.torch, self.f8 = torch, f8
        self.g = torch.Generator(device="cuda").manual_seed(seed)

    def ints(self, lo, hi, *shape):
        return self.torch.randint(lo, hi, shape, generator=self.g, device="cuda", dtype=self.torch.int64)

    def some(self, n, count):
        """`count` of n places, in any order."""
        return self.torch.randperm(n, generator=self.g, device="cuda")[:count]

    def powers(self, *shape):
        """Powers of two of either sign."""
        torch = self.torch
        return torch.exp2(self.ints(-3, 4, *shape).double()) * (1 - 2 * self.ints(0, 2, *shape))

    def scales(self, *shape):
        return (127 + self.ints(-3, 4, *shape)).to(self.torch.uint8).view(self.f8.SCALES)

    def dense(self, rows, cols):
        q = self.ints(0, 256, rows, self.f8.pitch(cols))
        q[(q & 0x7f) == 0x7f] = 0
        q[:, cols:] = 0
        return q.to(self.torch.uint8).view(self.f8.CODES)

    def ones(self, rows, cols, r, c):
        """Codes of +-1 at (r, c) and 0 elsewhere."""
        q = self.torch.zeros(rows, self.f8.pitch(cols), dtype=self.torch.uint8, device="cuda")
        q[r, c] = (0x38 + 0x80 * self.ints(0, 2, len(r))).to(self.torch.uint8)
        return q.view(self.f8.CODES)


def cuts(rows, experts):
    """First rows of the experts and the end: uneven, one without rows, the first and the last rows nobody's."""
    if not experts:
        return [0, rows]
    E = experts
    cut = sorted([rows // 9] + [rows * (3 * e * e + 1) // (3 * E * E + 2) for e in range(1, E)] + [max(rows - 3, rows // 9)])
    if E > 2:
        cut[2] = cut[1]
    return cut


def values(f8, q, s, cols):
    return f8.dequantize(q, s, cols).double()


def rounded(f8, v):
    """The values of the codes of v's rows (compared with the rule's in test_gpu_f8)."""
    return f8.dequantize(*f8.quantize(v.float().contiguous()), v.shape[1]).double()


def off_border(torch, dtype, *shape):
    """(a tensor that begins one element off a 16-byte border, what it is part of)."""
    n = 1
    for s in shape:
        n *= s
    buf = torch.full((n + 17,), 7.0, dtype=dtype, device="cuda")
    return buf[1:n + 1].view(*shape), buf


def untouched(buf, n):
    return bool((buf[:1] == 7).all()) and bool((buf[n + 1:] == 7).all())


@pytest.mark.parametrize("sparse", ["a", "w"])
@pytest.mark.parametrize("kernel,t,rows,experts,N,K", SOME_PRODUCTS)
def test_product(torch, f8, kernel, t, rows, experts, N, K, sparse):
    import paper_2609_26077_amd as fm
    E = max(1, experts)
    assert fm.fmm_f8_matmul_kernel(fm.fmm_f8_desc(rows, E, N, K, TYPE[t])) == kernel
    m = Make(torch, f8, rows + N + K)
    far = K - 1 if K <= 16384 else 16384           # (half of the codes in what follows the first 128 steps, where there is more)

    def places(n):
        at = m.ints(0, K, n)
        at[::2] = m.ints(min(far, K - 1), K, len(at[::2])) if K > 16384 else at[::2]
        return at

    at_a, at_w = places(rows), places(E * N)
    every = torch.arange(max(rows, E * N), device="cuda")
    a = m.ones(rows, K, every[:rows], at_a) if sparse == "a" else m.dense(rows, K)
    w = (m.ones(E * N, K, every[:E * N], at_w) if sparse == "w" else m.dense(E * N, K)).view(E, N, -1)
    sa, sw = m.scales(rows, f8.scale_pitch(K)), m.scales(E, -(-N // 128), f8.scale_pitch(K))
    cut = cuts(rows, experts)
    dtype = dtype_of(torch, t)
    out, buf = off_border(torch, dtype, rows, N) if sparse == "w" else (torch.full((rows, N), 7.0, dtype=dtype, device="cuda"), None)
    if experts:
        off = torch.tensor(cut, dtype=torch.int32).cuda()
        f8.GroupedLinearF8(rows, E, N, K, dtype).matmul(a, sa, w, sw, off, C=out)
    else:
        f8.LinearF8(rows, N, K, dtype).matmul(a, sa, w[0], sw[0], C=out)
    va, vw = values(f8, a, sa, K), values(f8, w, sw, K)
    want = torch.full((rows, N), 7.0, dtype=torch.float64, device="cuda")
    for e, (lo, hi) in enumerate(zip(cut, cut[1:])):
        if sparse == "a":
            k = at_a[lo:hi]
            want[lo:hi] = va[lo:hi].gather(1, k[:, None]) * vw[e][:, k].t()
        else:
            k = at_w[e * N:(e + 1) * N]
            want[lo:hi] = va[lo:hi][:, k] * vw[e].gather(1, k[:, None]).t()
    assert torch.equal(out, want.to(dtype))
    assert buf is None or untouched(buf, rows * N)


@pytest.mark.parametrize("kernel,t,rows,experts,N,K", SOME_PRODUCTS)
def test_product_of_whole_operands(torch, f8, kernel, t, rows, experts, N, K):
    E = max(1, experts)
    m = Make(torch, f8, rows + N + K)
    a, w = m.dense(rows, K), m.dense(E * N, K).view(E, N, -1)
    sa, sw = m.scales(rows, f8.scale_pitch(K)), m.scales(E, -(-N // 128), f8.scale_pitch(K))
    # (a factor of 2^-24 keeps fp16's results in its range)
    sa, sw = ((s.view(torch.uint8) - 12).view(f8.SCALES) for s in (sa, sw))
    cut = cuts(rows, experts)
    if experts:
        C = f8.GroupedLinearF8(rows, E, N, K, dtype_of(torch, t)).matmul(a, sa, w, sw, torch.tensor(cut, dtype=torch.int32).cuda())
    else:
        C = f8.LinearF8(rows, N, K, dtype_of(torch, t)).matmul(a, sa, w[0], sw[0])
    va, vw = values(f8, a, sa, K), values(f8, w, sw, K)
    for e, (lo, hi) in enumerate(zip(cut, cut[1:])):
        want, S = product(va[lo:hi], vw[e]), product(va[lo:hi].abs(), vw[e].abs())
        within(torch, C[lo:hi], want, bound(t, S, want, K), f"expert {e}")


@pytest.mark.parametrize("sparse", ["dy", "operands"])
@pytest.mark.parametrize("kernel,t,rows,experts,N,K,want", SOME_GRADIENTS)
def test_gradients(torch, f8, kernel, t, rows, experts, N, K, want, sparse):
    import paper_2609_26077_amd as fm
    E, dtype = max(1, experts), dtype_of(torch, t)
    desc = fm.fmm_f8_desc(rows, E, N, K, TYPE[t])
    assert fm.fmm_f8_linear_backward_kernel(desc, *want) == kernel
    m = Make(torch, f8, rows + N + K)
    cut = cuts(rows, experts)
    span = list(zip(cut, cut[1:]))
    sa, sw = m.scales(rows, f8.scale_pitch(K)), m.scales(E, -(-N // 128), f8.scale_pitch(K))
    pairs = []               # of each expert: rows of it with columns, no row and no column twice
    if sparse == "dy":
        a, w = m.dense(rows, K), m.dense(E * N, K).view(E, N, -1)
        dy = torch.zeros(rows, N, dtype=torch.float64, device="cuda")
        for lo, hi in span:
            n = min(hi - lo, N)
            r, c = m.some(hi - lo, n), m.some(N, n)
            dy[lo + r, c] = m.powers(n)
            pairs.append((r, c))
    else:
        dy = m.powers(rows, 1) * torch.randn(rows, N, generator=m.g, device="cuda")
        r_all, c_all, blocks = [], [], []
        for lo, hi in span:
            n = min(hi - lo, K)
            r, c = m.some(hi - lo, n), m.some(K, n)
            j, k = m.some(N, min(N, K)), m.some(K, min(N, K))
            pairs.append((r, c, j, k))
            r_all.append(lo + r)
            c_all.append(c)
            blocks.append(m.ones(N, K, j, k).view(torch.uint8))
        a, w = m.ones(rows, K, torch.cat(r_all), torch.cat(c_all)), torch.stack(blocks).view(f8.CODES)
    dy = dy.to(dtype)
    off = torch.tensor(cut, dtype=torch.int32).cuda() if experts else None
    dx, x_buf = off_border(torch, dtype, rows, K) if want[0] else (None, None)
    dw, w_buf = off_border(torch, dtype, E, N, K) if want[1] else (None, None)
    db = torch.empty(E, N, device="cuda")
    n = fm.fmm_f8_linear_backward_scratch_size(desc)
    fm.fmm_f8_linear_backward(desc, dy, a, sa, w, sw, off, dx, dw, db, torch.empty(n, dtype=torch.uint8, device="cuda"), n)
    va, vw = values(f8, a, sa, K), values(f8, w, sw, K)
    for e, (lo, hi) in enumerate(span):
        y = dy[lo:hi].double()
        want_x = torch.zeros(hi - lo, K, dtype=torch.float64, device="cuda")
        want_w = torch.zeros(N, K, dtype=torch.float64, device="cuda")
        if hi > lo:
            yr, yc, xc = rounded(f8, y), rounded(f8, y.t()).t(), rounded(f8, va[lo:hi].t()).t()
            if sparse == "dy":
                r, c = pairs[e]
                v = y[r, c][:, None]
                want_x[r], want_w[c] = v * vw[e][c], v * xc[r]
                assert torch.equal(db[e].double(), y.sum(0))
            else:
                r, c, j, k = pairs[e]
                want_x[:, k] = yr[:, j] * vw[e][j, k]
                want_w[:, c] = yc[r].t() * va[lo + r, c]
        if want[0]:
            assert torch.equal(dx[lo:hi], want_x.to(dtype)), f"dX of expert {e}"
        if want[1]:
            assert torch.equal(dw[e], want_w.to(dtype)), f"dW of expert {e}"
    assert x_buf is None or untouched(x_buf, rows * K)
    assert w_buf is None or untouched(w_buf, E * N * K)


@pytest.mark.parametrize("kernel,t,rows,experts,N,K,want", SOME_GRADIENTS)
def test_gradients_of_whole_operands(torch, f8, kernel, t, rows, experts, N, K, want):
    E, dtype = max(1, experts), dtype_of(torch, t)
    m = Make(torch, f8, rows + N + K)
    a, w = m.dense(rows, K), m.dense(E * N, K).view(E, N, -1)
    sa, sw = m.scales(rows, f8.scale_pitch(K)), m.scales(E, -(-N // 128), f8.scale_pitch(K))
    sa, sw = ((s.view(torch.uint8) - 12).view(f8.SCALES) for s in (sa, sw))
    cut = cuts(rows, experts)
    dy = (m.powers(rows, 1) * torch.randn(rows, N, generator=m.g, device="cuda")).to(dtype)
    kw = dict(need_x=bool(want[0]), need_w=bool(want[1]), bias=True)
    if experts:
        off = torch.tensor(cut, dtype=torch.int32).cuda()
        dx, dw, db = f8.GroupedLinearF8(rows, E, N, K, dtype).backward(dy, a, sa, w, sw, off, **kw)
    else:
        dx, dw, db = f8.LinearF8(rows, N, K, dtype).backward(dy, a, sa, w[0], sw[0], **kw)
        dw, db = dw if dw is None else dw[None], db[None]
    va, vw, yr = values(f8, a, sa, K), values(f8, w, sw, K), rounded(f8, dy)
    for e, (lo, hi) in enumerate(zip(cut, cut[1:])):
        y = dy[lo:hi].double()
        if want[0]:
            C, S = product(yr[lo:hi], vw[e].t()), product(yr[lo:hi].abs(), vw[e].abs().t())
            within(torch, dx[lo:hi], C, bound(t, S, C, N), f"dX of expert {e}")
        if want[1] and hi > lo:
            yc, xc = rounded(f8, y.t()), rounded(f8, va[lo:hi].t())
            C, S = product(yc, xc), product(yc.abs(), xc.abs())
            within(torch, dw[e], C, bound(t, S, C, hi - lo), f"dW of expert {e}")
        within(torch, db[e], y.sum(0), 2 * (hi - lo + 1) * U * y.abs().sum(0) + 1e-30, f"dbias of expert {e}")


@pytest.mark.parametrize("t", ["bf16", "fp16"])
@pytest.mark.parametrize("K", [512, 4096, 33000])
def test_16_bit_sums_keep_their_digits(torch, f8, t, K):
    """Root mean square errors, relative to the results', of products and of dW over K normal values.  Of each eight
    products the fp8 cores cut at most seven, toward zero, by less than 2^-13 of the largest, whose square is on average
    at most eight products' squares; with signs of either kind the cuts add up as the products do, so 7 K / 8 cuts of
    mean square 8 2^-26 p^2 make 7 2^-26 of K p^2.  The rounding's own error is that of the exact results rounded; a
    twentieth of either for the draw."""
    n, dtype = 300, dtype_of(torch, t)
    g = torch.Generator(device="cuda").manual_seed(K)
    x, v, dy = (torch.randn(*s, generator=g, device="cuda") for s in ((n, K), (n, K), (K, n)))
    a, sa = f8.quantize(x)
    w, sw = f8.quantize_weight(v * K ** -0.5)
    b, sb = f8.quantize(x.t().contiguous())
    wb, swb = f8.quantize_weight(v[:, :n].contiguous())
    dy = (dy * K ** -0.5).to(dtype)
    _, dw, _ = f8.LinearF8(K, n, n, dtype).backward(dy, b, sb, wb, swb, need_x=False)
    yc, xc = rounded(f8, dy.t()), rounded(f8, values(f8, b, sb, n).t())
    for got, want in ((f8.LinearF8(n, n, K, dtype).matmul(a, sa, w, sw), product(values(f8, a, sa, K), values(f8, w, sw, K))),
                      (dw, product(yc, xc))):
        own, half = ((y.double() - want).square().mean() / want.square().mean() for y in (got, want.to(dtype)))
        assert float(own) <= 1.05 * (float(half) + 7 * 2.0 ** -26)
