"""The operators of an 8-bit linear layer whose speed is watched: the RMS norm
with the residual's addition and an 8-bit output, its gradient from an 8-bit
checkpoint, the int8 product with a scale for each token and channel, and the
linear layer's gradients from its 8-bit operands.

Rows of 8 bits are int8 codes q and one float scale s, the values being q s:
a = max(amax |x|, 1e-12) over the row, q = rne(x (127 / a)), s = a / 127.  Code
rows are padded with zeros to a multiple of 128.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
_BYTES = {"bf16": 2, "fp16": 2, "fp32": 4}
_EPS = 1e-6
_GROUP = 128


# ---- the cases ---------------------------------------------------------------
def _norm(name, rows, cols, dtype, residual=True, checkpoint=True):
    c = {"op": "norm", "rows": rows, "cols": cols, "dtype": dtype, "residual": residual, "checkpoint": checkpoint}
    return c if name is None else dict(c, name=name)


def _norm_grad(name, rows, cols, dtype, source="codes", residual=True):
    c = {"op": "norm_grad", "rows": rows, "cols": cols, "dtype": dtype, "source": source, "residual": residual}
    return c if name is None else dict(c, name=name)


def _matmul(name, M, N, K, dtype, bias=False, source="codes"):
    c = {"op": "matmul", "M": M, "N": N, "K": K, "dtype": dtype, "bias": bias, "source": source}
    return c if name is None else dict(c, name=name)


def _linear_grad(name, M, N, K, dtype, bias=True):
    c = {"op": "linear_grad", "M": M, "N": N, "K": K, "dtype": dtype, "bias": bias}
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # serving, one token: the norm in front of a projection, where the call's latency is all
        _norm("norm_1x4096", 1, 4096, "bf16", checkpoint=False),
        # a training step's norm over 8192 tokens, with the 8-bit checkpoint of the residual stream
        _norm("norm_8192x4096", 8192, 4096, "bf16"),
        # rows that fit no vector: an odd width, in fp32
        _norm("norm_1000x1301_fp32", 1000, 1301, "fp32"),
        # that training step's norm gradient, from the checkpoint
        _norm_grad("norm_grad_8192x4096", 8192, 4096, "bf16"),
        # a small ragged gradient from the stored residual stream
        _norm_grad("norm_grad_1000x1302_fp16", 1000, 1302, "fp16", source="h", residual=False),
        # serving, one token: every weight is read once
        _matmul("matmul_1x8192x8192", 1, 8192, 8192, "bf16"),
        # serving, a batch of tokens against a wide projection
        _matmul("matmul_48x7168x2048", 48, 7168, 2048, "bf16"),
        # a ragged prompt: activations quantized on the way, a bias, fp16
        _matmul("matmul_1000x1302x1472_fp16", 1000, 1302, 1472, "fp16", bias=True, source="values"),
        # a training step's forward product
        _matmul("matmul_8192x8192x8192", 8192, 8192, 8192, "bf16"),
        # a small micro-batch's gradients
        _linear_grad("linear_grad_256x2048x2048", 256, 2048, 2048, "bf16"),
        # ragged gradients in fp32
        _linear_grad("linear_grad_1000x1302x1472_fp32", 1000, 1302, 1472, "fp32", bias=False),
        # a training step's gradients: the heaviest case
        _linear_grad("linear_grad_8192x8192x4096", 8192, 8192, 4096, "bf16"),
    ]


def _size(rng, lo, hi):
    """Spread over the logarithm; a third of the sizes on multiples of 128, the others wherever they fall."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if v >= 128 and rng.random() < 0.34:
        v -= v % 128
    return v + 1 if v == 3072 else v


def draw(rng):
    op = rng.choice(["norm", "norm_grad", "matmul", "linear_grad"])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    if op in ("norm", "norm_grad"):
        cols = _size(rng, 64, 16384)
        rows = _size(rng, 1, max(1, min(8192, 8192 * 4096 // cols)))
        if op == "norm":
            return _norm(None, rows, cols, dtype, rng.random() < 0.7, rng.random() < 0.5)
        return _norm_grad(None, rows, cols, dtype, rng.choice(["codes", "h"]), rng.random() < 0.7)
    if op == "matmul":
        M, N, K = _size(rng, 1, 8192), _size(rng, 64, 8192), _size(rng, 64, 8192)
        return _matmul(None, M, N, K, dtype, rng.random() < 0.5, rng.choice(["codes", "values"]))
    M, N, K = _size(rng, 16, 8192), _size(rng, 64, 8192), _size(rng, 64, 4096)
    return _linear_grad(None, M, N, K, dtype, rng.random() < 0.5)


# ---- 8-bit rows, plainly -------------------------------------------------------
def _codes(v):
    """(codes as floats, amax clamped) of each row of v (fp32)."""
    a = v.abs().amax(dim=-1, keepdim=True).clamp_min(1e-12)
    return torch.round(v * torch.div(torch.full_like(a, 127.0), a)), a


def _padded(v):
    return torch.nn.functional.pad(v, (0, -v.shape[-1] % _GROUP))


def _quantized(v):
    q, a = _codes(v)
    return _padded(q).to(torch.int8), (a / 127.0).squeeze(-1)


# ---- inputs --------------------------------------------------------------------
def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    op, dtype = case["op"], _TYPES[case["dtype"]]
    s = {"case": case}
    if op in ("norm", "norm_grad"):
        R, K = case["rows"], case["cols"]
        # a residual stream: a few channels an order of magnitude above the others
        loud = torch.where(torch.rand(K, generator=g, device="cuda") < 0.004, 12.0, 1.0)
        x = (normal(R, K) * loud).to(dtype)
        s["gain"] = (1.0 + 0.2 * normal(K)).to(dtype)
        if op == "norm":
            s["x"] = x
            s["residual"] = normal(R, K).to(dtype) if case["residual"] else None
        else:
            h = x.float()
            s["rstd"] = torch.rsqrt(h.square().mean(dim=1) + _EPS)
            s["dy"] = (0.05 * normal(R, K)).to(dtype)
            s["dh"] = (0.05 * normal(R, K)).to(dtype) if case["residual"] else None
            if case["source"] == "h":
                s["h"] = x
            else:
                q, a = _codes(_padded(h).view(R, -1, _GROUP))
                s["saved_codes"], s["saved_scales"] = q.to(torch.int8).view(R, -1), (a / 127.0).squeeze(-1)
    else:
        M, N, K = case["M"], case["N"], case["K"]
        a = normal(M, K).to(dtype)
        if case.get("source") == "values":
            s["x"] = a
        else:
            s["a"], s["sa"] = _quantized(a.float())
        s["w"], s["sw"] = _quantized((normal(N, K) / math.sqrt(K)).to(dtype).float())
        if op == "matmul":
            s["bias"] = 0.1 * normal(N) if case["bias"] else None
        else:
            s["dy"] = (0.05 * normal(M, N)).to(dtype)
    if own:
        from paper_2609_26077_amd import q8
        s["plan"] = (q8.RMSNormQ8(case["rows"], case["cols"], dtype, eps=_EPS) if op in ("norm", "norm_grad")
                     else q8.LinearQ8(case["M"], case["N"], case["K"], dtype))
    return s


# ---- one pass --------------------------------------------------------------------
def run(s):
    return (_own if own else _plain)(s)


def _group_values(codes, scales, cols):
    return (codes.view(codes.shape[0], -1, _GROUP).float() * scales[:, :, None]).view(codes.shape[0], -1)[:, :cols]


def _own(s):
    from paper_2609_26077_amd import q8
    case, plan = s["case"], s["plan"]
    if case["op"] == "norm":
        o = plan.forward(s["x"], s["residual"], s["gain"], checkpoint=case["checkpoint"])
        K, dtype = case["cols"], _TYPES[case["dtype"]]
        out = {"h": o.h, "y": q8.dequantize(o.codes, o.scales, K, dtype), "scales": o.scales, "rstd": o.rstd}
        if case["checkpoint"]:
            out["saved"] = q8.dequantize(o.saved_codes, o.saved_scales, K, dtype)
        return out
    if case["op"] == "norm_grad":
        saved = (s["saved_codes"], s["saved_scales"]) if case["source"] == "codes" else None
        dx, dgain = plan.backward(s["dy"], s["rstd"], s["gain"], h=s.get("h"), saved=saved, dh=s["dh"])
        return {"dx": dx, "dgain": dgain}
    if case["op"] == "matmul":
        a, sa = q8.quantize(s["x"]) if case["source"] == "values" else (s["a"], s["sa"])
        return plan.matmul(a, sa, s["w"], s["sw"], s["bias"])
    dx, dw, dbias = plan.backward(s["dy"], s["a"], s["sa"], s["w"], s["sw"], bias=case["bias"])
    return {"dx": dx, "dw": dw, "dbias": dbias}


def _plain(s):
    case = s["case"]
    dtype = _TYPES[case["dtype"]]
    if case["op"] == "norm":
        K = case["cols"]
        h = s["x"].float()
        if s["residual"] is not None:
            h = h + s["residual"].float()
        rstd = torch.rsqrt(h.square().sum(dim=1) / K + _EPS)
        q, a = _codes(h * s["gain"].float())
        scales = (a / 127.0).squeeze(-1) * rstd
        out = {"h": h.to(dtype), "y": (q * scales[:, None]).to(dtype), "scales": scales, "rstd": rstd}
        if case["checkpoint"]:
            cq, ca = _codes(_padded(h).view(h.shape[0], -1, _GROUP))
            out["saved"] = (cq * (ca / 127.0)).view(h.shape[0], -1)[:, :K].to(dtype)
        return out
    if case["op"] == "norm_grad":
        K = case["cols"]
        h = s["h"].float() if case["source"] == "h" else _group_values(s["saved_codes"], s["saved_scales"], K)
        xh, dy = h * s["rstd"][:, None], s["dy"].float()
        w = dy * s["gain"].float()
        c = (w * xh).sum(dim=1, keepdim=True) / K
        dx = s["rstd"][:, None] * (w - xh * c)
        if s["dh"] is not None:
            dx = dx + s["dh"].float()
        return {"dx": dx.to(dtype), "dgain": (dy * xh).sum(dim=0)}
    K = case["K"]
    w = s["w"][:, :K].float()
    if case["op"] == "matmul":
        if case["source"] == "values":
            a, amax = _codes(s["x"].float())
            sa = amax / 127.0
        else:
            a, sa = s["a"][:, :K].float(), s["sa"][:, None]
        c = (a @ w.t()) * sa * s["sw"]
        if s["bias"] is not None:
            c = c + s["bias"]
        return c.to(dtype)
    dy = s["dy"].float()
    return {"dx": ((dy * s["sw"]) @ w).to(dtype), "dw": ((dy * s["sa"][:, None]).t() @ s["a"][:, :K].float()).to(dtype),
            "dbias": dy.sum(dim=0) if case["bias"] else None}


# ---- what a pass cannot do without ---------------------------------------------------
def work(case):
    t = _BYTES[case["dtype"]]
    if case["op"] in ("norm", "norm_grad"):
        R, K = case["rows"], case["cols"]
        groups = -(-K // _GROUP)
        if case["op"] == "norm":
            # the input [, the residual and their sum], the gain, codes and the values they stand for, scales and 1 / rms
            b = R * K * t * (3 if case["residual"] else 1) + K * t + R * K * (1 + t) + 8 * R
            b += R * (K * (1 + t) + 4 * groups) if case["checkpoint"] else 0
            return {"bytes": b, "flops": 8 * R * K}
        b = 2 * R * K * t + K * t + 4 * R + 4 * K + (R * K * t if case["residual"] else 0)
        b += R * K * t if case["source"] == "h" else R * (K + 4 * groups)
        return {"bytes": b, "flops": 10 * R * K}
    M, N, K = case["M"], case["N"], case["K"]
    if case["op"] == "matmul":
        a = M * K * t if case["source"] == "values" else M * K + 4 * M
        return {"bytes": a + N * K + 4 * N + M * N * t + (4 * N if case["bias"] else 0), "flops": 2 * M * N * K}
    return {"bytes": M * N * t + M * K + N * K + 4 * M + 4 * N + M * K * t + N * K * t + (4 * N if case["bias"] else 0),
            "flops": 4 * M * N * K}


# ---- the definition in 64 bits ------------------------------------------------------
def _row64(v):
    """Nearest multiples of a 127th of each row's largest magnitude: (integers, step)."""
    step = torch.clamp(torch.amax(torch.abs(v), -1), min=float(np.float32(1e-12))) / 127
    return torch.round(v / step.unsqueeze(-1)), step


def _product64(x, y):
    """x y in fp64, in bands of rows (a band's temporary stays small)."""
    return torch.cat([torch.mm(b, y) for b in torch.split(x, 2048)])


def exact(case, seed):
    s, f64 = prepare(case, seed), torch.float64
    up = {k: v.to(f64) for k, v in s.items() if isinstance(v, torch.Tensor)}
    if case["op"] == "norm":
        R, K = case["rows"], case["cols"]
        h = up["x"] + up["residual"] if "residual" in up else up["x"]
        rstd = (torch.einsum("rk,rk->r", h, h) / K + _EPS) ** -0.5
        q, step = _row64(h * up["gain"])
        out = {"h": h, "y": q * (step * rstd).unsqueeze(1), "scales": step * rstd, "rstd": rstd}
        if case["checkpoint"]:
            parts = [_row64(p) for p in torch.split(h, _GROUP, dim=1)]
            out["saved"] = torch.cat([q * d.unsqueeze(1) for q, d in parts], dim=1)
        return out
    if case["op"] == "norm_grad":
        R, K = case["rows"], case["cols"]
        if case["source"] == "h":
            h = up["h"]
        else:
            h = (up["saved_codes"] * torch.repeat_interleave(up["saved_scales"], _GROUP, dim=1))[:, :K]
        r = up["rstd"].unsqueeze(1)
        t = up["dy"] * up["gain"]
        # d/dh of the sum of t h (mean h^2 + eps)^(-1/2)
        dx = r * t - r ** 3 * h * (torch.einsum("rk,rk->r", t, h) / K).unsqueeze(1)
        if "dh" in up:
            dx = dx + up["dh"]
        return {"dx": dx, "dgain": torch.einsum("rk,rk,r->k", up["dy"], h, up["rstd"])}
    K = case["K"]
    wv = up["w"][:, :K] * up["sw"].unsqueeze(1)
    if case["op"] == "matmul":
        if case["source"] == "values":
            q, step = _row64(up["x"])
            av = q * step.unsqueeze(1)
        else:
            av = up["a"][:, :K] * up["sa"].unsqueeze(1)
        c = _product64(av, wv.t().contiguous())
        return c + up["bias"] if "bias" in up else c
    av = up["a"][:, :K] * up["sa"].unsqueeze(1)
    return {"dx": _product64(up["dy"], wv), "dw": _product64(up["dy"].t().contiguous(), av),
            "dbias": torch.einsum("mn->n", up["dy"]) if case["bias"] else None}
