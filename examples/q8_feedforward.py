"""A pre-norm feed-forward layer on 8-bit operands: trained with 8-bit
checkpoints, then run for single tokens.

    h = x + residual;  y = norm(h) gain;  u = y W1^T + b1;  out = silu(u) W2^T + b2

Forward, the norm writes y as int8 codes with a scale per token, the products
take those against int8 weights with a scale per output channel, and silu(u) is
quantized in between.  What the backward pass keeps is 8 bits an element: the
norm's checkpoint of h, the products' operands as they are, and u's codes.  The
master weights are float32 and are quantized after every step.

    python examples/q8_feedforward.py [--tokens 4096] [--width 1024] [--hidden 4096] [--steps 30] [--max-norm 1]
"""
from __future__ import annotations

import argparse
import os
import sys
import time

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch  # noqa: E402

from paper_2609_26077_amd import q8  # noqa: E402
from paper_2609_26077_amd.grads import clip  # noqa: E402


KEPT_PLANS = 8


class FeedForward:
    """The layer's weights, and its forward and backward passes for any number of tokens."""

    def __init__(self, width, hidden, dtype=torch.bfloat16, device="cuda:0", seed=0):
        g = torch.Generator(device=device).manual_seed(seed)
        self.width, self.hidden, self.dtype, self.device = width, hidden, dtype, device
        self.gain = torch.ones(width, device=device)
        self.w1 = torch.randn(hidden, width, generator=g, device=device) / width ** 0.5
        self.w2 = torch.randn(width, hidden, generator=g, device=device) / hidden ** 0.5
        self.b1, self.b2 = torch.zeros(hidden, device=device), torch.zeros(width, device=device)
        self.plans = {}
        self.quantize_weights()

    def quantize_weights(self):
        self.q1, self.q2 = q8.quantize(self.w1), q8.quantize(self.w2)
        self.gain_in = self.gain.to(self.dtype)

    def _plan(self, tokens):
        """The operators for this many tokens.  Those of the last few counts are kept, as
        each that a backward pass came to holds a workspace."""
        plan = self.plans.pop(tokens, None)
        if plan is None:
            plan = (q8.RMSNormQ8(tokens, self.width, self.dtype, device=self.device),
                    q8.LinearQ8(tokens, self.hidden, self.width, self.dtype, device=self.device),
                    q8.LinearQ8(tokens, self.width, self.hidden, self.dtype, device=self.device))
            if len(self.plans) == KEPT_PLANS:
                del self.plans[next(iter(self.plans))]      # the one that was used longest ago
        self.plans[tokens] = plan
        return plan

    def forward(self, x, residual, train=False):
        """(out, h, what backward needs or None)"""
        norm, up, down = self._plan(x.shape[0])
        o = norm.forward(x, residual, self.gain_in, checkpoint=train)
        u = up.matmul(o.codes, o.scales, *self.q1, bias=self.b1)
        s = q8.quantize(torch.nn.functional.silu(u))
        out = down.matmul(*s, *self.q2, bias=self.b2)
        kept = (o.codes, o.scales, o.rstd, (o.saved_codes, o.saved_scales), s, q8.quantize(u)) if train else None
        return out, o.h, kept

    def backward(self, dout, dh, kept):
        """Gradients of (x and residual), w1, b1, w2, b2, gain; dh: the gradient of h from its other uses."""
        y, ys, rstd, saved, s, (uq, us) = kept
        norm, up, down = self._plan(dout.shape[0])
        ds, dw2, db2 = down.backward(dout, *s, *self.q2, bias=True)
        u = q8.dequantize(uq, us, self.hidden, self.dtype)
        sig = torch.sigmoid(u)
        du = ds * (sig * (1 + u * (1 - sig)))
        dy, dw1, db1 = up.backward(du, y, ys, *self.q1, bias=True)
        dx, dgain = norm.backward(dy, rstd, self.gain_in, saved=saved, dh=dh)
        return dx, dw1, db1, dw2, db2, dgain

    def step(self, grads, rate, max_norm=None):
        """max_norm: the gradients are scaled down to this norm, of all of them together, first."""
        if max_norm is not None:
            clip(grads, max_norm)
        for p, g in zip((self.w1, self.b1, self.w2, self.b2, self.gain), grads):
            p.add_(g, alpha=-rate)
        self.quantize_weights()


def train(layer, tokens, steps, seed=1, max_norm=None):
    """Fits out + h to a fixed random map of x by gradient descent; the losses of the steps."""
    rate = 5.0 / layer.width
    g = torch.Generator(device=layer.device).manual_seed(seed)
    x = torch.randn(tokens, layer.width, generator=g, device=layer.device)
    m = torch.randn(layer.width, layer.width, generator=g, device=layer.device) / layer.width ** 0.5
    x, residual = x.to(layer.dtype), torch.zeros_like(x, dtype=layer.dtype)
    target = (x.float() @ m).to(layer.dtype) + x
    losses = []
    for _ in range(steps):
        out, h, kept = layer.forward(x, residual, train=True)
        err = (out + h - target).float()
        losses.append(err.square().mean())
        d = (err * (2.0 / tokens)).to(layer.dtype)
        _, *grads = layer.backward(d, d, kept)
        layer.step(grads, rate, max_norm)
    return [float(v) for v in losses], x


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--tokens", type=int, default=4096)
    ap.add_argument("--width", type=int, default=1024)
    ap.add_argument("--hidden", type=int, default=4096)
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--max-norm", type=float, default=None, help="clip each step's gradients to this norm")
    a = ap.parse_args(argv)
    layer = FeedForward(a.width, a.hidden)
    losses, x = train(layer, a.tokens, 2, max_norm=a.max_norm)          # (first launches)
    torch.cuda.synchronize()
    t = time.perf_counter()
    more, x = train(layer, a.tokens, a.steps, max_norm=a.max_norm)
    torch.cuda.synchronize()
    print(f"training: loss {losses[0]:.4f} -> {more[-1]:.4f} in {a.steps + 2} steps, "
          f"{1e3 * (time.perf_counter() - t) / a.steps:.2f} ms a step of {a.tokens} tokens")
    zero = torch.zeros_like(x[:1])
    for _ in range(3):
        layer.forward(x[:1], zero)
    torch.cuda.synchronize()
    t = time.perf_counter()
    for i in range(100):
        layer.forward(x[i:i + 1], zero)
    torch.cuda.synchronize()
    print(f"serving: {1e4 * (time.perf_counter() - t):.1f} us a token")
    return losses + more


if __name__ == "__main__":
    main()
