"""The AdamW step over one buffer of values in 64 bits, on the CPU, from its definition (numpy only): states as they are, or in 8 bits
with rounding to either neighbour by a hash of the seed, the step and the place."""
from __future__ import annotations

import numpy as np

from .fp8_oracle import BLOCK, block_exponent


def mix(x):
    x = np.asarray(x, dtype=np.uint64) & np.uint64(0xFFFFFFFF)
    for shift, factor in ((16, 0x9E3779B1), (15, 0xB7E15163)):
        x = ((x ^ (x >> np.uint64(shift))) * np.uint64(factor)) & np.uint64(0xFFFFFFFF)
    return x ^ (x >> np.uint64(16))


def hash_of(seed: int, step: int, places: np.ndarray) -> np.ndarray:
    places = np.asarray(places, dtype=np.uint64)
    key = mix(mix(seed) ^ np.uint64(step & 0xFFFFFFFF))
    return mix((places & np.uint64(0xFFFFFFFF)) ^ mix(key ^ (places >> np.uint64(32))))


def neighbours(v: np.ndarray):
    """Of v in whole blocks: (exponents of the blocks, |v| / 2^e, the e4m3 value below it, the part of the way to the one above, the step)."""
    v = np.asarray(v, dtype=np.float64).reshape(-1, BLOCK)
    e = block_exponent(np.abs(v).max(axis=1))
    y = np.abs(v) / np.exp2(e.astype(np.float64))[:, None]
    _, ex = np.frexp(np.where(y == 0, 1.0, y))
    step = np.exp2(np.maximum(ex - 1, -6) - 3.0)
    below = np.floor(y / step) * step
    return e, y, below, (y - below) / step, step


def quantize(v: np.ndarray, h16: np.ndarray):
    """(values of the codes, exponents of the blocks); v is finite and has whole blocks."""
    e, _, below, part, step = neighbours(v)
    up = part + (h16.reshape(-1, BLOCK).astype(np.float64) + 0.5) / 65536 >= 1
    return (np.sign(np.asarray(v).reshape(-1, BLOCK)) * (below + up * step)).reshape(-1), e


def least_root(beta1: float, beta2: float) -> float:
    """sqrt(v) / |m| at the least, over all pasts: m is a sum of (1 - beta1) beta1^i g_i, v one of (1 - beta2) beta2^i g_i^2."""
    return ((1 - beta2) * (1 - beta1 ** 2 / beta2)) ** 0.5 / (1 - beta1) if beta1 ** 2 < beta2 else 0.0


def step(p, g, m, v, t, lr, beta1, beta2, eps, decay, clip=1.0, least=0.0):
    """(p, m, v) after step t; least: the root's least part of |m| (least_root, for states in 8 bits)."""
    g = g * clip
    m, v = beta1 * m + (1 - beta1) * g, beta2 * v + (1 - beta2) * g * g
    root = np.maximum(np.sqrt(v), least * np.abs(m))
    return p * (1 - lr * decay) - lr * (m / (1 - beta1 ** t)) / (root / (1 - beta2 ** t) ** 0.5 + eps), m, v
