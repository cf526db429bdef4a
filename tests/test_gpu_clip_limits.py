"""Clipping at the ends of its arguments' range, many tensors, and what autograd sees of it.  Bars as in test_gpu_clip."""
from __future__ import annotations

import numpy as np
import pytest

from test_gpu_clip import HALF_ULP, SMALLEST, check, tensors

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    return torch


@pytest.fixture(scope="module")
def grads():
    from paper_2609_26077_amd import grads
    return grads


def test_autograd_sees_the_write(torch, grads):
    """A tensor that a graph has kept for its backward pass is clipped: the pass is refused, as after torch's own writes."""
    for out in (False, True):
        g = torch.randn(100, device="cuda")
        x = torch.randn(100, device="cuda", requires_grad=True)
        y = (x * g).sum()
        if out:
            grads.clip([torch.randn_like(g)], 0.5, out=[g])
        else:
            grads.clip([g], 0.5)
        assert g._version == 1
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()
    # inputs that are only read, and tensors that keep no version
    a, b = torch.randn(10, device="cuda"), torch.empty(10, device="cuda")
    grads.clip([a], 0.5, out=[b])
    assert (a._version, b._version) == (0, 1)
    with torch.inference_mode():
        c = torch.randn(10, device="cuda")
    grads.clip([c], 0.0)
    assert bool((c == 0).all())


def test_an_infinite_norm_gives_zeros(torch, grads):
    """Whatever the limit, an infinite one too: the factor is 0 (infinity times 0 is NaN)."""
    for most in (0.0, 1.0, float("inf")):
        ts = [torch.ones(100, device="cuda"), torch.ones(33, device="cuda", dtype=torch.bfloat16)]
        ts[1][5] = -float("inf")
        norm = grads.clip(ts, most)
        assert float(norm) == float("inf")
        assert bool((ts[0] == 0).all()) and bool(torch.isnan(ts[1][5])) and int((ts[1] == 0).sum()) == 32
    # a limit that nothing reaches
    ts = [torch.full((100,), 3e38, device="cuda")]
    grads.clip(ts, float("inf"))
    assert bool((ts[0] == 3e38).all())


@pytest.mark.parametrize("types", ["float32", "bfloat16", "mixed"])
@pytest.mark.parametrize("scale,most", [(1e38, 1.0), (3e38, 1e-3), (1e30, 1e-12), (1e37, 1e-38), (3e38, 1e-42)])
def test_factors_below_fp32s_normal_numbers(torch, grads, types, scale, most):
    """The factor keeps its digits: its bar is that of any other, 2^-24 relative (in binary64 less), of the limit as fp32 holds it."""
    dtypes = [torch.float32, torch.bfloat16] if types == "mixed" else [getattr(torch, types)]
    g = torch.Generator().manual_seed(3)
    ts = [(scale * (torch.rand(n, generator=g, dtype=torch.float64) * 2 - 1)).to(dtypes[i % len(dtypes)]).cuda()
          for i, n in enumerate((3000, 1, 700))]
    most = float(np.float32(most))
    up = [t.double().cpu().numpy() for t in ts]
    want = np.sqrt(sum((u ** 2).sum() for u in up))
    c = most / (want + 1e-6)
    assert 0 < c < 2.0 ** -126
    out = [torch.empty_like(t) for t in ts]
    grads.clip(ts, most, out=out)
    for u, o in zip(up, out):
        n = str(o.dtype).split(".")[1]
        assert (np.abs(o.double().cpu().numpy() - u * c) <= (HALF_ULP[n] + 2.5 * 2.0 ** -24) * np.abs(u * c) + SMALLEST[n]).all()


@pytest.mark.parametrize("count,size", [(1000, 1301), (5000, 77), (122880, 5)])
def test_many_tensors(torch, grads, count, size):
    """More than a few launches of 120 tensors, to the most that a call takes; one tensor more is refused."""
    g = torch.Generator(device="cuda").manual_seed(count)
    buf = torch.randn(count, size, generator=g, device="cuda") * torch.exp(torch.randn(count, 1, generator=g, device="cuda"))
    out = torch.full_like(buf, 7.0)
    norm = grads.clip(buf.unbind(), 0.5, out=out.unbind())
    again = torch.empty_like(buf)
    assert torch.equal(grads.clip(buf.unbind(), 0.5, out=again.unbind()), norm) and torch.equal(again, out)
    x = buf.double()
    want = float(x.square().sum().sqrt())
    assert abs(float(norm) - want) <= 2.0 ** -23 * want
    c = min(1.0, 0.5 / (want + 1e-6))
    assert bool(((out.double() - c * x).abs() <= 3.5 * 2.0 ** -24 * c * x.abs()).all())
    if count == 122880:
        with pytest.raises(RuntimeError):
            grads.clip([*buf.unbind(), torch.zeros(1, device="cuda")], 0.5)
