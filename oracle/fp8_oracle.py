"""The operators around 8-bit projections in 64 bits, on the CPU, from their definitions (numpy only).

8-bit format: e4m3 values under power-of-two scales, one for each 128 consecutive elements of a row, or 128 x 128 of a weight:
2^e with the least e >= -127 for which the largest finite magnitude of the block is at most 448 * 2^e (-127 for zeros). What is
not finite is stored as NaN.
"""
from __future__ import annotations

import numpy as np

BLOCK = 128
E4M3_MAX = 448.0


def e4m3_round(v: np.ndarray) -> np.ndarray:
    """The e4m3 value nearest to v (|v| <= 448), ties to the even code: 3 mantissa bits, least exponent -6."""
    v = np.asarray(v, dtype=np.float64)
    _, ex = np.frexp(np.where(v == 0, 1.0, v))           # |v| = m * 2^ex, m in [0.5, 1)
    step = np.exp2(np.maximum(ex - 1, -6) - 3.0)
    return np.round(v / step) * step


def block_exponent(most: np.ndarray) -> np.ndarray:
    """e of blocks whose largest finite magnitude is `most`."""
    most = np.asarray(most, dtype=np.float64)
    m, ex = np.frexp(most)                               # 448 = 0.875 * 2^9
    return np.where(most > 0, np.maximum(ex - 9 + (m > 0.875), -127), -127).astype(np.int64)


def quantize(v: np.ndarray, rows: int = 1):
    """(values of the codes, exponents) of v [n, k] in blocks of `rows` x 128; codes are float64, NaN where v is not finite."""
    v = np.asarray(v, dtype=np.float64)
    n, k = v.shape
    nb, kb = -(-n // rows), -(-k // BLOCK)
    codes, exps = np.zeros((n, k)), np.zeros((nb, kb), dtype=np.int64)
    for i in range(nb):
        for j in range(kb):
            part = v[i * rows:(i + 1) * rows, j * BLOCK:(j + 1) * BLOCK]
            fine = np.isfinite(part)
            exps[i, j] = block_exponent(np.abs(part[fine]).max() if fine.any() else 0.0)
            scaled = np.where(fine, part, 0.0) / 2.0 ** float(exps[i, j])
            codes[i * rows:(i + 1) * rows, j * BLOCK:(j + 1) * BLOCK] = np.where(fine, e4m3_round(scaled), np.nan)
    return codes, exps


def dequantize(codes: np.ndarray, exps: np.ndarray, rows: int = 1) -> np.ndarray:
    n, k = codes.shape
    scale = np.exp2(exps.astype(np.float64))
    return codes * np.repeat(np.repeat(scale, rows, axis=0)[:n], BLOCK, axis=1)[:, :k]


def rms_norm(s: np.ndarray, weight, eps: float) -> np.ndarray:
    return s / np.sqrt((s * s).mean(axis=1, keepdims=True) + eps) * (1.0 if weight is None else weight)


def rms_norm_gradients(dy: np.ndarray, s: np.ndarray, weight, eps: float, dsum=None):
    """(dx, dweight)."""
    r = 1 / np.sqrt((s * s).mean(axis=1, keepdims=True) + eps)
    u, g = s * r, dy * (1.0 if weight is None else weight)
    dx = r * (g - u * (g * u).mean(axis=1, keepdims=True))
    return dx if dsum is None else dx + dsum, (dy * u).sum(axis=0)


def silu_gate(gate: np.ndarray, up: np.ndarray) -> np.ndarray:
    with np.errstate(over="ignore"):
        return gate / (1 + np.exp(-gate)) * up


def silu_gate_gradients(gate: np.ndarray, up: np.ndarray, dh: np.ndarray):
    """(dgate, dup)."""
    with np.errstate(over="ignore"):
        sig = 1 / (1 + np.exp(-gate))
    return dh * up * sig * (1 + gate * (1 - sig)), dh * gate * sig
