#!/usr/bin/env python3
"""Fine-tuning beside frozen 4-bit projections: one MLP block of a decoder whose gate, up and down weights stay in 4 bits while a factorised adapter
(a Tucker layer beside them), held as bf16 tensors with fp32 masters, learns by AdamW with its states in 8 bits.

    python examples/int4_finetune.py [--hidden 5120] [--width 25600] [--tokens 777]

Every step runs through the public entry points; outputs and gradients are compared with the same block in 64 bits on the CPU, with the weights that
the 4-bit layers hold, at a small size (run without arguments on an MI355X: prints the relative errors and the times).
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


class Block:
    """y = x + down(silu(gate(x)) * up(x)) + adapter(x)."""

    def __init__(self, w_gate, w_up, w_down, adapter, modes, ranks, max_tokens, group=128, state_bits=8):
        self.gate_up, self.down = tn.Int4Linear([w_gate, w_up], max_tokens, group=group), tn.Int4Linear([w_down], max_tokens, group=group)
        self.gate_up_back, self.down_back = self._transposed(self.gate_up), self._transposed(self.down)
        self.adapter, self.modes, self.ranks, self.max_tokens = adapter, modes, ranks, max_tokens
        self.optimizer = tn.AdamW(adapter, lr=1e-3, weight_decay=0.0, state_bits=state_bits)
        self._make_adapter()

    @staticmethod
    def _transposed(layer):
        """The gradients' layer with the same codes: groups lie along the inputs in both."""
        codes, scales, zeros = zip(*(layer.quantized_tensor(i) for i in range(layer.n_tensors)))
        return tn.Int4Linear(codes, layer.max_tokens, transpose=True, group=layer.group, scales=[s.to(layer.scale_dtype) for s in scales], zeros=zeros,
                             in_features=layer.shape[1])

    def _make_adapter(self):
        """A factorised layer lays its tensors out when it is made: after each step of the optimizer it is made again."""
        make = lambda flags: tn.TNLinear(tn.TN_FORMAT_TUCKER, tn.TN_DTYPE_BF16, self.modes, self.modes, self.ranks, self.adapter, self.max_tokens, flags=flags)      # noqa: E731
        self.factors, self.factors_back = make(tn.TN_FLAG_TRAINABLE), make(tn.TN_FLAG_TRANSPOSE)

    def forward(self, x):
        return x + self.down(self.gate_up.gated(x)) + self.factors(x)

    def gradients(self, x, dy):
        """(y, gradient of x, gradients of the adapter's tensors) for dL/dy = dy."""
        gate_up = self.gate_up(x)                                                # kept for the way back
        y = x + self.down(tn.silu_gate(gate_up).y) + self.factors(x)
        d_gate_up = tn.silu_gate_gradients(gate_up, self.down_back(dy)).y
        dx = dy + self.gate_up_back(d_gate_up) + self.factors_back(dy)
        return y, dx, self.factors.param_gradients(x, dy)

    def step(self, x, dy, max_norm=1.0):
        """One step of the optimizer; returns (y, gradient of x, norm of the adapter's gradients)."""
        y, dx, grads = self.gradients(x, dy)
        norm = self.optimizer.gradient_norm(grads)                               # (over several ranks: their squares' sum, here)
        self.optimizer.step(grads, max_norm=max_norm, norm=norm)
        self._make_adapter()
        return y, dx, norm


def make_block(hidden, width, max_tokens, group=128, seed=0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    normal = lambda *shape: torch.randn(shape, generator=gen, device="cuda")      # noqa: E731
    m1 = max(d for d in range(1, int(math.isqrt(hidden)) + 1) if hidden % d == 0)
    modes, r = (m1, hidden // m1), min(8, m1)
    ranks = (r, r, r, r)
    weights = [(normal(rows, cols) / cols ** 0.5).bfloat16() for rows, cols in ((width, hidden), (width, hidden), (hidden, width))]
    adapter = [(normal(*ranks) / r).bfloat16()] + [(normal(m, r) / m ** 0.5).bfloat16() for m in modes + modes]
    return Block(*weights, adapter, modes, ranks, max_tokens, group), normal


def held(layer, slot):
    """The weight a 4-bit layer holds, in 64 bits on the CPU."""
    codes, scales, zeros = (t.double().cpu() for t in layer.quantized_tensor(slot))
    n, group = layer.shape[1], layer.group
    values = torch.stack([codes % 16, torch.floor(codes / 16)], dim=2).flatten(1)[:, :n]
    of = torch.arange(n) // group
    return (values - zeros[:, of]) * scales[:, of]


def in_64_bits(block, x, dy):
    """The block and its gradients on the CPU by differentiation."""
    d = lambda t: t.detach().double().cpu()      # noqa: E731
    s = d(x).requires_grad_()
    core, u1, u2, v1, v2 = factors = [d(t).requires_grad_() for t in block.adapter]
    gate, up = (s @ held(block.gate_up, i).T for i in (0, 1))
    w = torch.kron(u1, u2) @ core.reshape(core.shape[0] * core.shape[1], -1) @ torch.kron(v1, v2).T
    y = s + (gate * torch.sigmoid(gate) * up) @ held(block.down, 0).T + s @ w.T
    (y * d(dy)).sum().backward()
    return y.detach(), s.grad, [f.grad for f in factors]


def relative_error(got, ref):
    return float((got.detach().double().cpu() - ref).norm() / ref.norm())


def check(hidden=640, width=1300, tokens=77, group=128):
    """Relative errors of the block, its gradients, their norm and the parameters' first moves (of lr each, where the gradient is not near zero)."""
    block, normal = make_block(hidden, width, tokens, group)
    x, dy = (normal(tokens, hidden).bfloat16() for _ in range(2))
    ref = in_64_bits(block, x, dy)
    y, dx, grads = block.gradients(x, dy)
    before = [t.double() for t in block.optimizer.params]
    errors = {"forward": relative_error(block.forward(x), ref[0]), "y": relative_error(y, ref[0]), "dx": relative_error(dx, ref[1]),
              "adapter": max(relative_error(g, r) for g, r in zip(grads, ref[2]))}
    _, _, norm = block.step(x, dy)
    exact = math.sqrt(sum(float((g * g).sum()) for g in ref[2]))
    errors["norm"] = abs(float(norm) / exact - 1)
    masters, at = block.optimizer.state_dict()["master"], 0
    moves = []
    for b, g in zip(before, grads):
        move = (masters[at:at + b.numel()].double() - b.flatten()) / block.optimizer.lr
        at += -(-b.numel() // 128) * 128
        scaled = g.double().flatten() * min(1.0, 1.0 / float(norm))
        moves.append(float((move + scaled / (scaled.abs() + block.optimizer.eps)).abs().max()))
    errors["move"] = max(moves)
    return errors


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
    print("relative errors against 64 bits:", {k: f"{v:.1e}" for k, v in check().items()})
    block, normal = make_block(a.hidden, a.width, a.tokens)
    for tokens in (1, a.tokens):
        x, dy = normal(tokens, a.hidden).bfloat16(), (1e-3 * normal(tokens, a.hidden)).bfloat16()
        print(f"{tokens} tokens: forward {timed(lambda: block.forward(x)):.0f} us, gradients {timed(lambda: block.gradients(x, dy)):.0f} us, "
              f"whole step {timed(lambda: block.step(x, dy), 5):.0f} us")


if __name__ == "__main__":
    main()
