#!/usr/bin/env python3
"""One MLP block of a decoder with 8-bit gate, up and down projections: forwards for a prompt and a single token, and one
fine-tuning step back through it. The weights stay as they are in 8 bits; what learns is the norm's weight and a factorised
adapter (a Tucker layer beside the down projection), as compressed models are healed.

    python examples/fp8_mlp_block.py [--hidden 5120] [--width 25600] [--tokens 777]

Every step runs through the public entry points, and the results are compared with the same block in 64 bits on the CPU at a
small size (run without arguments on an MI355X: prints the relative errors and the times).
"""
from __future__ import annotations

import argparse
import math
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2602_01613_amd as tn  # noqa: E402

EPS = 1e-6


class MlpBlock:
    """y = s + down(silu(gate(n)) * up(n)) + adapter(n), s = x + residual, n = norm(s)."""

    def __init__(self, w_gate, w_up, w_down, norm_weight, adapter, modes, ranks, max_tokens, train=False):
        self.block = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")      # partial sums, shared by the layers
        self.norm_weight = norm_weight
        self.gate_up = tn.Fp8Linear([w_gate, w_up], max_tokens, workspace=self.block)
        self.down = tn.Fp8Linear([w_down], max_tokens, workspace=self.block)
        make = lambda flags: tn.TNLinear(tn.TN_FORMAT_TUCKER, tn.TN_DTYPE_BF16, modes, modes, ranks, adapter, max_tokens, flags=flags)      # noqa: E731
        self.adapter = make(tn.TN_FLAG_TRAINABLE if train else 0)
        if train:
            self.gate_up_back = tn.Fp8Linear([w_gate, w_up], max_tokens, transpose=True, workspace=self.block)
            self.down_back = tn.Fp8Linear([w_down], max_tokens, transpose=True, workspace=self.block)
            self.adapter_back = make(tn.TN_FLAG_TRANSPOSE)

    def forward(self, x, residual):
        n = tn.rms_norm(x, self.norm_weight, EPS, residual=residual, outputs="both")      # 8 bits for gate and up, bf16 for the factors
        h = self.gate_up.gated(n.fp8)
        return n.sum + self.down(h) + self.adapter(n.y)

    def step(self, x, residual, dy):
        """(y, gradient of x and residual, gradient of the norm's weight, gradients of the adapter's tensors) for dL/dy = dy."""
        n = tn.rms_norm(x, self.norm_weight, EPS, residual=residual, outputs="both")
        gate_up = self.gate_up(n.fp8)                                                       # kept for the way back
        h = tn.silu_gate(gate_up, outputs="fp8").fp8
        y = n.sum + self.down(h) + self.adapter(n.y)
        dh = self.down_back(dy)
        d_gate_up = tn.silu_gate_gradients(gate_up, dh, outputs="fp8").fp8
        dn = self.gate_up_back(d_gate_up) + self.adapter_back(dy)
        dx, d_weight = tn.rms_norm_gradients(dn, n.sum, self.norm_weight, EPS, dsum=dy)
        return y, dx, d_weight, self.adapter.param_gradients(n.y, dy)


def make_block(hidden, width, max_tokens, train=False, seed=0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    normal = lambda *shape: torch.randn(shape, generator=gen, device="cuda")      # noqa: E731
    m1 = max(d for d in range(1, int(math.isqrt(hidden)) + 1) if hidden % d == 0)
    modes, r = (m1, hidden // m1), min(8, m1)
    ranks = (r, r, r, r)
    weights = {"gate": (normal(width, hidden) / hidden ** 0.5).bfloat16(), "up": (normal(width, hidden) / hidden ** 0.5).bfloat16(),
               "down": (normal(hidden, width) / width ** 0.5).bfloat16(), "norm": (1 + 0.1 * normal(hidden)).bfloat16()}
    adapter = [(normal(*ranks) / r).bfloat16()] + [(normal(m, r) / m ** 0.5).bfloat16() for m in modes + modes]
    block = MlpBlock(weights["gate"], weights["up"], weights["down"], weights["norm"], adapter, modes, ranks, max_tokens, train)
    return block, weights, adapter, normal


def in_64_bits(weights, adapter, x, residual, dy):
    """The block on the CPU with the weights as they are, unquantised, and the gradients by differentiation."""
    d = lambda t: t.detach().double().cpu()      # noqa: E731
    s = d(x + residual).requires_grad_()
    norm = d(weights["norm"]).requires_grad_()
    factors = [d(t).requires_grad_() for t in adapter]
    n = s / torch.sqrt((s * s).mean(dim=1, keepdim=True) + EPS) * norm
    gate, up = n @ d(weights["gate"]).T, n @ d(weights["up"]).T
    h = gate * torch.sigmoid(gate) * up
    core, u1, u2, v1, v2 = factors
    w = torch.kron(u1, u2) @ core.reshape(core.shape[0] * core.shape[1], -1) @ torch.kron(v1, v2).T
    y = s + h @ d(weights["down"]).T + n @ w.T
    (y * d(dy)).sum().backward()
    return y.detach(), s.grad, norm.grad, [f.grad for f in factors]


def relative_error(got, ref):
    ref = ref.double().cpu()
    return float((got.detach().double().cpu() - ref).norm() / ref.norm())


def check(hidden=640, width=1300, tokens=77):
    block, weights, adapter, normal = make_block(hidden, width, tokens, train=True)
    x, residual, dy = (normal(tokens, hidden).bfloat16() for _ in range(3))
    ref = in_64_bits(weights, adapter, x, residual, dy)
    y, dx, d_weight, d_adapter = block.step(x, residual, dy)
    return {"forward": relative_error(block.forward(x, residual), ref[0]), "step y": relative_error(y, ref[0]), "dx": relative_error(dx, ref[1]),
            "norm weight": relative_error(d_weight, ref[2]),
            "adapter": max(relative_error(g, r) for g, r in zip(d_adapter, ref[3]))}


def timed(fn, reps=20):
    for _ in range(3):
        fn()
    torch.cuda.synchronize()
    start = time.perf_counter()
    for _ in range(reps):
        fn()
    torch.cuda.synchronize()
    return (time.perf_counter() - start) / reps * 1e6


def main():
    p = argparse.ArgumentParser()
    p.add_argument("--hidden", type=int, default=5120)
    p.add_argument("--width", type=int, default=25600)
    p.add_argument("--tokens", type=int, default=777)
    a = p.parse_args()
    print("relative errors against unquantised weights in 64 bits:", {k: f"{v:.1e}" for k, v in check().items()})
    block, _, _, normal = make_block(a.hidden, a.width, a.tokens, train=True)
    for tokens in (1, a.tokens):
        x, residual, dy = (normal(tokens, a.hidden).bfloat16() for _ in range(3))
        print(f"{tokens} tokens: forward {timed(lambda: block.forward(x, residual)):.0f} us, "
              f"fine-tuning step {timed(lambda: block.step(x, residual, dy)):.0f} us")


if __name__ == "__main__":
    main()
