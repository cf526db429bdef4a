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
