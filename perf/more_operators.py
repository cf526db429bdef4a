"""More operators whose speed is watched: those of a linear layer, or of many
experts' layers, on e4m3 operands with a power-of-two scale for each block of
128, and the global norm of many gradients with clipping.

A block's scale is 2^e, e the least integer with amax |x| <= 448 2^e (e >= -126; 0
for a block of zeros), held as the byte e + 127; a code is the e4m3 number
nearest x 2^-e, ties to even.  Blocks are 128 columns of a row (activations,
gradients) or 128 x 128 (weights).  Code rows are padded with zeros to a multiple
of 128, rows of scales to a multiple of 16.
"""
from __future__ import annotations

import math
import random

import torch
import torch.nn.functional as F

own = False

_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
_BYTES = {"bf16": 2, "fp16": 2, "fp32": 4}
_B = 128


# ---- the cases ---------------------------------------------------------------
def _quantize(rows, cols, dtype, blocks=False, experts=1):
    return {"op": "quantize", "rows": rows, "cols": cols, "dtype": dtype, "blocks": blocks, "experts": experts}


def _matmul(rows, N, K, dtype, bias=False, experts=0):
    return {"op": "matmul", "rows": rows, "N": N, "K": K, "dtype": dtype, "bias": bias, "experts": experts}


def _grad(rows, N, K, dtype, bias=False, experts=0):
    return {"op": "grad", "rows": rows, "N": N, "K": K, "dtype": dtype, "bias": bias, "experts": experts}


def _clip(tensors, least, most, dtype):
    return {"op": "clip", "tensors": tensors, "least": least, "most": most, "dtype": dtype}


def listed():
    return [dict(c, name=name) for name, c in [
        # serving, one token: the activations in front of a projection, where the call's latency is all
        ("quantize_1x4096", _quantize(1, 4096, "bf16")),
        # master weights of a few experts after a step, odd widths
        ("quantize_weights_8x1301x2050_fp32", _quantize(1301, 2050, "fp32", blocks=True, experts=8)),
        # serving, one token: every weight is read once
        ("matmul_1x8192x8192", _matmul(1, 8192, 8192, "bf16")),
        # a ragged prompt in full output precision, with a bias
        ("matmul_1000x1302x1472_fp32", _matmul(1000, 1302, 1472, "fp32", bias=True)),
        # a training step's forward product
        ("matmul_8192x8192x8192", _matmul(8192, 8192, 8192, "bf16")),
        # serving: 16 tokens at 4 of 32 experts each
        ("grouped_64x2048x4096_of_32", _matmul(64, 2048, 4096, "bf16", experts=32)),
        # a prompt's tokens over a few experts, odd sizes
        ("grouped_2001x1030x1472_of_7_fp16", _matmul(2001, 1030, 1472, "fp16", bias=True, experts=7)),
        # a training step's tokens over the experts
        ("grouped_16384x4096x4096_of_16", _matmul(16384, 4096, 4096, "bf16", experts=16)),
        # gradients of a small ragged micro-batch in fp32
        ("grad_1000x1302x1472_fp32", _grad(1000, 1302, 1472, "fp32", bias=True)),
        # gradients of a training step over the experts
        ("grouped_grad_16384x4096x2048_of_16", _grad(16384, 4096, 2048, "bf16", experts=16)),
        # the many small tensors of a narrow network
        ("clip_300_small_fp32", _clip(300, 64, 65536, "fp32")),
        # the gradients of a few wide layers
        ("clip_40_large", _clip(40, 1 << 20, 1 << 24, "bf16")),
    ]]


def _size(rng, lo, hi):
    """Spread over the logarithm; a third of the sizes on multiples of 128, the others wherever they fall."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return v - v % _B if v >= _B and rng.random() < 0.34 else v


def draw(rng):
    op = rng.choice(["quantize", "matmul", "matmul", "grouped", "grouped", "grad", "grouped_grad", "clip"])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    if op == "quantize":
        cols, blocks = _size(rng, 64, 16384), rng.random() < 0.4
        rows = _size(rng, 1, max(1, min(16384, (1 << 25) // cols)))
        experts = rng.randint(1, 8) if blocks else 1
        return _quantize(max(1, rows // experts), cols, dtype, blocks, experts)
    if op == "clip":
        least = _size(rng, 1, 1 << 16)
        most = _size(rng, least + 1, 1 << 22)
        return _clip(_size(rng, 1, 400), least, most, dtype)
    experts = int(round(math.exp(rng.uniform(0.0, math.log(64))))) if op.startswith("grouped") else 0
    top = 4096 if experts else 8192
    if op.endswith("grad"):
        rows, N, K = _size(rng, 16, 8192), _size(rng, 64, 4096), _size(rng, 64, 2048)
    else:
        rows, N, K = _size(rng, 1, top), _size(rng, 64, top), _size(rng, 64, top)
    while experts * N * K > 16 * 4096 * 4096:
        experts //= 2
    return (_grad if op.endswith("grad") else _matmul)(rows, N, K, dtype, rng.random() < 0.4, experts)


# ---- 8-bit blocks, plainly -----------------------------------------------------
def _exponents(a):
    """The least e with a <= 448 2^e = 7/8 2^(e + 9), as integers."""
    m, x = torch.frexp(a)
    e = torch.where(m <= 0.875, x - 9, x - 8).clamp_min(-126)
    return torch.where(a > 0, e, torch.zeros_like(e))


def _two(e):
    """2^e, exactly (-126 <= e <= 127)."""
    return ((e + 127).to(torch.int32) << 23).view(torch.float32)


def _coded(v, axes):
    """(codes, exponents) of v, its blocks spanning `axes`."""
    e = _exponents(v.abs().amax(dim=axes, keepdim=True))
    return (v * _two(-e)).clamp(-448.0, 448.0).to(torch.float8_e4m3fn), e


def _rounded(v, axes):
    """The values that the codes of v stand for."""
    q, e = _coded(v, axes)
    return q.float() * _two(e)


def _scale_rows(e):
    """Exponents [..., blocks] as bytes, rows padded to 16."""
    return F.pad((e + 127).to(torch.uint8), (0, -e.shape[-1] % 16), value=127).contiguous().view(torch.float8_e8m0fnu)


def _activations(x):
    """Codes [rows, pitch] and scales [rows, scale pitch] of x."""
    R, K = x.shape
    q, e = _coded(F.pad(x.float(), (0, -K % _B)).view(R, -1, _B), 2)
    return q.view(R, -1), _scale_rows(e.view(R, -1))


def _weights(w):
    """Codes [experts, N, pitch] and scales [experts, N / 128, scale pitch] of w."""
    E, N, K = w.shape
    v = F.pad(w.float(), (0, -K % _B, 0, -N % _B))
    q, e = _coded(v.view(E, v.shape[1] // _B, _B, v.shape[2] // _B, _B), (2, 4))
    return (q.view(torch.uint8).view(E, v.shape[1], v.shape[2])[:, :N].contiguous().view(torch.float8_e4m3fn),
            _scale_rows(e.view(E, v.shape[1] // _B, v.shape[2] // _B)))


def _steps(scales):
    return scales.view(torch.uint8).to(torch.int32) - 127


def _values(q, s, K):
    """The values of codes with a scale for each row and 128 columns."""
    P = q.shape[1]
    return (q.float().view(-1, P // _B, _B) * _two(_steps(s)[:, :P // _B, None])).view(-1, P)[:, :K]


def _weight_values(q, s, K):
    E, N, P = q.shape
    e = _steps(s)[:, :, :P // _B].repeat_interleave(_B, dim=1)[:, :N]
    return (q.float().view(E, N, P // _B, _B) * _two(e)[..., None]).view(E, N, P)[:, :, :K]


# ---- inputs --------------------------------------------------------------------
def _loads(rows, experts, seed):
    """Rows of each expert: some have many, some have none."""
    r = random.Random(seed)
    p = [math.exp(r.gauss(0.0, 0.7)) if r.random() < 0.92 else 0.0 for _ in range(experts)]
    p = p if sum(p) else [1.0] * experts
    loads = [int(rows * v / sum(p)) for v in p]
    for e in r.choices(range(experts), weights=p, k=rows - sum(loads)):
        loads[e] += 1
    return loads


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    op, dtype = case["op"], _TYPES[case["dtype"]]
    s = {"case": case}
    if op == "clip":
        # gradients of layers whose magnitudes lie orders apart
        r = random.Random(case["tensors"])
        sizes = [int(math.exp(r.uniform(math.log(case["least"]), math.log(case["most"])))) for _ in range(case["tensors"])]
        r = random.Random(int(seed))
        s["grads"] = [(normal(n) * 10.0 ** r.uniform(-4, -1)).to(dtype) for n in sizes]
        # clipped into one buffer, each tensor on a border of its own
        s["at"] = [0]
        for n in sizes:
            s["at"].append(s["at"][-1] - (-n // _B) * _B)
        s["flat"] = torch.zeros(s["at"][-1], dtype=dtype, device="cuda")
        s["out"] = [s["flat"][i:i + n] for i, n in zip(s["at"], sizes)]
        s["max_norm"] = 1.0
        return s
    if op == "quantize":
        # a few channels an order of magnitude above the others
        K = case["cols"]
        loud = torch.where(torch.rand(K, generator=g, device="cuda") < 0.004, 12.0, 1.0)
        shape = (case["experts"], case["rows"], K) if case["blocks"] else (case["rows"], K)
        s["x"] = (normal(*shape) * (0.02 if case["blocks"] else loud)).to(dtype)
        return s
    R, N, K, E = case["rows"], case["N"], case["K"], max(1, case["experts"])
    s["a"], s["sa"] = _activations(normal(R, K).to(dtype))
    s["w"], s["sw"] = _weights(normal(E, N, K) / math.sqrt(K))
    loads = _loads(R, E, int(seed)) if case["experts"] else [R]
    s["offsets"] = torch.tensor([sum(loads[:e]) for e in range(E + 1)], dtype=torch.int32).cuda()
    s["most"] = max(loads)          # rows of the fullest expert
    if op == "matmul":
        s["bias"] = 0.1 * normal(E, N) if case["bias"] else None
    else:
        s["dy"] = (normal(R, N) * torch.exp(normal(R, 1)) * 1e-3).to(dtype)
    if own:
        from paper_2609_26077_amd import f8
        s["plan"] = (f8.GroupedLinearF8(R, E, N, K, dtype) if case["experts"] else f8.LinearF8(R, N, K, dtype))
    return s


# ---- one pass --------------------------------------------------------------------
def run(s):
    return (_own if own else _plain)(s)


def _own(s):
    case = s["case"]
    if case["op"] == "clip":
        from paper_2609_26077_amd import grads
        return {"norm": grads.clip(s["grads"], s["max_norm"], out=s["out"]), "out": s["flat"]}
    from paper_2609_26077_amd import f8
    if case["op"] == "quantize":
        q, sc = (f8.quantize_weight if case["blocks"] else f8.quantize)(s["x"])
        return f8.dequantize(q, sc, case["cols"], _TYPES[case["dtype"]])
    plan, bias = s["plan"], case["bias"]
    if case["experts"]:
        if case["op"] == "matmul":
            return plan.matmul(s["a"], s["sa"], s["w"], s["sw"], s["offsets"], s["bias"])
        dx, dw, dbias = plan.backward(s["dy"], s["a"], s["sa"], s["w"], s["sw"], s["offsets"], bias=bias)
    else:
        w, sw = s["w"][0], s["sw"][0]
        if case["op"] == "matmul":
            return plan.matmul(s["a"], s["sa"], w, sw, s["bias"][0] if bias else None)
        dx, dw, dbias = plan.backward(s["dy"], s["a"], s["sa"], w, sw, bias=bias)
    return {"dx": dx, "dw": dw, "dbias": dbias}


def _by_expert(s):
    """Places of the rows in a batch of [experts, rows of the fullest, to 128]."""
    off = s["offsets"].long()
    rows = torch.arange(s["case"]["rows"], device="cuda")
    e = torch.searchsorted(off[1:].contiguous(), rows, right=True)
    L = -(-s["most"] // _B) * _B
    return e * L + rows - off[e], L


def _padded(v, at, L, E):
    return torch.zeros(E * L, v.shape[1], device="cuda").index_copy_(0, at, v).view(E, L, v.shape[1])


def _plain(s):
    case = s["case"]
    dtype = _TYPES[case["dtype"]]
    if case["op"] == "clip":
        squares = torch.stack([t.double().square().sum() for t in s["grads"]])
        norm = squares.sum().sqrt()
        c = (s["max_norm"] / (norm + 1e-6)).clamp_max(1.0).float()
        for t, o in zip(s["grads"], s["out"]):
            o.copy_(t.float() * c)
        return {"norm": norm.float(), "out": s["flat"]}
    if case["op"] == "quantize":
        x = s["x"]
        if case["blocks"]:
            return _weight_values(*_weights(x), case["cols"]).to(dtype)
        return _values(*_activations(x), case["cols"]).to(dtype)
    K, E = case["K"], max(1, case["experts"])
    x, w = _values(s["a"], s["sa"], K), _weight_values(s["w"], s["sw"], K)
    at, L = _by_expert(s)
    if case["op"] == "matmul":
        c = torch.bmm(_padded(x, at, L, E), w.transpose(1, 2))
        if s["bias"] is not None:
            c = c + s["bias"][:, None]
        return c.view(E * L, -1)[at].to(dtype)
    N = case["N"]
    dy = s["dy"].float()
    rows = _rounded(F.pad(dy, (0, -N % _B)).view(len(dy), -1, _B), 2).view(len(dy), -1)[:, :N]
    dx = torch.bmm(_padded(rows, at, L, E), w).view(E * L, K)[at]
    # along the rows of each expert
    dyp = _padded(dy, at, L, E)
    dyc = _rounded(dyp.view(E, L // _B, _B, N), 2).view(E, L, N)
    xc = _rounded(_padded(x, at, L, E).view(E, L // _B, _B, K), 2).view(E, L, K)
    dw = torch.bmm(dyc.transpose(1, 2), xc)
    dbias = dyp.sum(dim=1) if case["bias"] else None
    if not case["experts"]:
        dw, dbias = dw[0], None if dbias is None else dbias[0]
    return {"dx": dx.to(dtype), "dw": dw.to(dtype), "dbias": dbias}


# ---- what a pass cannot do without ---------------------------------------------------
def work(case):
    t = _BYTES[case["dtype"]]
    if case["op"] == "clip":
        n = case["tensors"] * (case["most"] - case["least"]) / math.log(case["most"] / case["least"])
        return {"bytes": 2 * n * t, "flops": 3 * n}
    if case["op"] == "quantize":
        n = case["experts"] * case["rows"] * case["cols"]
        return {"bytes": n * (2 * t + 1), "flops": 4 * n}
    R, N, K, E = case["rows"], case["N"], case["K"], max(1, case["experts"])
    read = R * K + min(E, R) * N * K + (min(E, R) * N * 4 if case["bias"] else 0)
    if case["op"] == "matmul":
        return {"bytes": read + R * N * t, "flops": 2 * R * N * K}
    return {"bytes": read + R * (N + K) * t + E * N * K * t, "flops": 4 * R * N * K}


# ---- the definition in 64 bits ------------------------------------------------------
def _near64(v, top):
    """The multiples that 4 significant bits allow, below a block's largest magnitude `top`."""
    s = torch.exp2(torch.ceil(torch.log2(torch.where(top > 0, top, 448.0) / 448.0)).clamp_min(-126.0))
    s = torch.where(top > 448.0 * s, s * 2, torch.where((top <= 224.0 * s) & (s > 2.0 ** -126) & (top > 0), s / 2, s))
    u = v / s
    grid = torch.exp2(torch.floor(torch.log2(u.abs().clamp_min(2.0 ** -6))) - 3)
    return torch.round(u / grid) * grid * s


def _bands64(v, dim, starts=(0,)):
    """v with blocks of 128 along `dim`, counted from each of `starts`."""
    cuts = list(starts) + [v.shape[dim]]
    parts = [p for a, b in zip(cuts, cuts[1:]) if b > a for p in torch.split(v.narrow(dim, a, b - a), _B, dim=dim)]
    return torch.cat([_near64(p, p.abs().amax(dim=dim, keepdim=True)) for p in parts], dim=dim)


def exact(case, seed):
    s, f64 = prepare(case, seed), torch.float64
    if case["op"] == "clip":
        norm = sum(float(torch.linalg.vector_norm(t.to(f64))) ** 2 for t in s["grads"]) ** 0.5
        c = min(1.0, s["max_norm"] / (norm + 1e-6))
        out = torch.zeros(s["at"][-1], dtype=f64, device="cuda")
        for t, i in zip(s["grads"], s["at"]):
            out[i:i + t.numel()] = t.to(f64) * c
        return {"norm": torch.tensor(norm, dtype=f64), "out": out}
    if case["op"] == "quantize":
        x = s["x"].to(f64)
        if not case["blocks"]:
            return _bands64(x, 1)
        return torch.cat([torch.cat([_near64(p, p.abs().amax(dim=(1, 2), keepdim=True)) for p in torch.split(r, _B, dim=2)], dim=2)
                          for r in torch.split(x, _B, dim=1)], dim=1)
    K, N, E = case["K"], case["N"], max(1, case["experts"])
    grow = lambda b, n: torch.exp2(b.view(torch.uint8).to(f64) - 127).repeat_interleave(_B, -1)[..., :n]  # noqa: E731
    x = s["a"].to(f64)[:, :K] * grow(s["sa"], K)
    off = s["offsets"].tolist()
    span = [slice(a, b) for a, b in zip(off, off[1:])]

    def weight(e):
        return s["w"][e].to(f64)[:, :K] * grow(s["sw"][e], K).repeat_interleave(_B, 0)[:N]

    if case["op"] == "matmul":
        return torch.cat([x[r] @ weight(e).t().contiguous() + (s["bias"][e].to(f64) if s["bias"] is not None else 0.0)
                          for e, r in enumerate(span)])
    dy = s["dy"].to(f64)
    rows = _bands64(dy, 1)
    dyc, xc = _bands64(dy, 0, off[:-1]), _bands64(x, 0, off[:-1])
    dw = torch.stack([dyc[r].t().contiguous() @ xc[r] for r in span])
    db = torch.stack([dy[r].sum(dim=0) for r in span]) if case["bias"] else None
    if not case["experts"]:
        dw, db = dw[0], None if db is None else db[0]
    return {"dx": torch.cat([rows[r] @ weight(e) for e, r in enumerate(span)]), "dw": dw, "dbias": db}
