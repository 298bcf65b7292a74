"""CPU oracle of the rotary position embedding: rows normalised and rotated, in float64.

TEST INFRASTRUCTURE ONLY, numpy, written from the definition; it shares no code with the library."""
from __future__ import annotations

from typing import Optional

import numpy as np

from .paged_attention import bf16_bits_to_f64


def positions(ctx_lens: np.ndarray, cu_q_lens: Optional[np.ndarray], total: int) -> np.ndarray:
    """The position of every row; -1 for rows of no sequence and of sequences with a negative length."""
    pos = np.full(total, -1, np.int64)
    for b, c in enumerate(np.asarray(ctx_lens, np.int64)):
        lo, hi = (b, b + 1) if cu_q_lens is None else (int(cu_q_lens[b]), int(cu_q_lens[b + 1]))
        if c >= 0:
            pos[lo:hi] = c + np.arange(hi - lo)
    return pos


def norm_rows(x: np.ndarray, weight: Optional[np.ndarray], eps: float) -> np.ndarray:
    """float64 rows [..., d] over their root mean square, times a weight; without one as they are."""
    if weight is None:
        return x
    return x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * weight


def rotate(x: np.ndarray, pos: np.ndarray, inv_freq: np.ndarray, interleaved: bool, factor: float = 1.0) -> np.ndarray:
    """float64 rows [tokens][heads][d], the first 2 len(inv_freq) channels turned by pos * inv_freq."""
    n = len(inv_freq)
    a = pos.astype(np.float64)[:, None] * inv_freq.astype(np.float32).astype(np.float64)
    turn = (factor * np.exp(1j * a))[:, None, :]
    y = x.copy()
    i, j = (np.arange(n) * 2, np.arange(n) * 2 + 1) if interleaved else (np.arange(n), np.arange(n) + n)
    z = (x[..., i] + 1j * x[..., j]) * turn
    y[..., i], y[..., j] = z.real, z.imag
    return y


def rope_rows(bits: np.ndarray, pos: np.ndarray, inv_freq: np.ndarray, interleaved: bool, factor: float = 1.0,
              weight_bits: Optional[np.ndarray] = None, eps: float = 1e-6) -> np.ndarray:
    """bf16 bit patterns [tokens][heads][d] -> float64 rows, normalised (with a weight) and rotated."""
    w = None if weight_bits is None else bf16_bits_to_f64(weight_bits)
    return rotate(norm_rows(bf16_bits_to_f64(bits), w, eps), pos, inv_freq, interleaved, factor)
