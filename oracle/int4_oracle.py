"""Projections with 4-bit weights in 64 bits, on the CPU, from their definitions (numpy only).

W[f][k] = (code[f][k] - zero[f][k // group]) * scale[f][k // group], codes and zeros from 0 to 15, two codes to a byte with the even k
in the low half.
"""
from __future__ import annotations

import numpy as np


def pack(codes: np.ndarray) -> np.ndarray:
    """codes [m, n] of 0 .. 15 as bytes [m, ceil(n / 2)]."""
    m, n = codes.shape
    even = np.zeros((m, n + n % 2), dtype=np.uint8)
    even[:, :n] = codes
    return even[:, 0::2] | (even[:, 1::2] << 4)


def unpack(packed: np.ndarray, n: int) -> np.ndarray:
    codes = np.empty((packed.shape[0], 2 * packed.shape[1]), dtype=np.uint8)
    codes[:, 0::2], codes[:, 1::2] = packed & 15, packed >> 4
    return codes[:, :n]


def weight(codes: np.ndarray, scales: np.ndarray, zeros, group: int) -> np.ndarray:
    """codes [m, n], scales and zeros [m, ceil(n / group)] (zeros None: 8)."""
    of = np.arange(codes.shape[1]) // group
    zeros = np.full(scales.shape, 8.0) if zeros is None else zeros.astype(np.float64)
    return (codes.astype(np.float64) - zeros[:, of]) * scales.astype(np.float64)[:, of]


def bf16(v: np.ndarray) -> np.ndarray:
    """fp32 values rounded to bf16, ties to even."""
    u = np.ascontiguousarray(v, dtype=np.float32).view(np.uint32).astype(np.uint64)
    return ((u + 0x7FFF + ((u >> 16) & 1)) & 0xFFFF0000).astype(np.uint32).view(np.float32)


def quantize(w: np.ndarray, group: int):
    """(codes, scales, zeros) of fp32 w [m, n] as the library quantises: every operation is one of fp32's, rounded once."""
    w = np.asarray(w, dtype=np.float32)
    m, n = w.shape
    groups = -(-n // group)
    codes, scales, zeros = np.full((m, n), 8, dtype=np.uint8), np.zeros((m, groups), dtype=np.float32), np.full((m, groups), 8, dtype=np.uint8)
    f15 = np.float32(15)
    for g in range(groups):
        part = w[:, g * group:(g + 1) * group]
        fine = np.isfinite(part).all(axis=1)
        safe = np.where(fine[:, None], part, np.float32(0))
        lo, hi = np.minimum(safe.min(axis=1), np.float32(0)), np.maximum(safe.max(axis=1), np.float32(0))
        s = bf16(hi / f15 - lo / f15)
        some = fine & (s > 0)
        div = np.where(some, s, np.float32(1))
        z = np.where(some, np.clip(np.rint(-lo / div), 0, 15), 8)
        q = np.clip(np.rint(safe / div[:, None]) + z[:, None], 0, 15)
        scales[:, g], zeros[:, g] = np.where(fine, s, np.nan), z
        codes[:, g * group:(g + 1) * group] = np.where(some[:, None], q, 8)
    return codes, scales, zeros


def silu_gate(gate: np.ndarray, up: np.ndarray) -> np.ndarray:
    with np.errstate(over="ignore"):
        return gate / (1 + np.exp(-gate)) * up
