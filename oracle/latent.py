"""CPU oracle of attention over a paged cache of latent rows, in float64.

TEST INFRASTRUCTURE ONLY, numpy, written from the definition; it shares no code with the library.  A cached row is (c, r): all
of it is the key of every head, c the value."""
from __future__ import annotations

from typing import Optional, Tuple

import numpy as np

from .paged_attention import PAGE, bf16_bits_to_f64
from .rotary import norm_rows, positions, rotate


def latent_rows(rows_bits: np.ndarray, pos: np.ndarray, dc: int, inv_freq: np.ndarray, interleaved: bool, factor: float = 1.0,
                weight_bits: Optional[np.ndarray] = None, eps: float = 1e-6) -> np.ndarray:
    """bf16 bit patterns [tokens][dc + dr] -> the float64 rows that the cache takes: c normalised, r rotated."""
    x = bf16_bits_to_f64(rows_bits)
    w = None if weight_bits is None else bf16_bits_to_f64(weight_bits)
    r = rotate(x[:, None, dc:], pos, inv_freq, interleaved, factor)[:, 0]
    return np.concatenate([norm_rows(x[:, :dc], w, eps), r], -1)


def latent_attention(q_bits: np.ndarray, cache_bits: np.ndarray, block_table: np.ndarray, ctx_lens: np.ndarray,
                     cu_q_lens: Optional[np.ndarray], dc: int, scale: float) -> Tuple[np.ndarray, np.ndarray, np.ndarray]:
    """(out [rows][H][dc], lse [rows][H], size: out with |c| for c); NaN in rows of no sequence."""
    total, heads, width = q_bits.shape
    out = np.full((total, heads, dc), np.nan)
    size, lse = out.copy(), np.full((total, heads), np.nan)
    pos = positions(ctx_lens, cu_q_lens, total)
    for b in range(len(ctx_lens)):
        lo, hi = (b, b + 1) if cu_q_lens is None else (int(cu_q_lens[b]), int(cu_q_lens[b + 1]))
        if lo == hi:
            continue
        n = int(pos[hi - 1]) + 1
        pages = np.asarray(block_table[b][:(n + PAGE - 1) // PAGE], np.int64)
        k = bf16_bits_to_f64(cache_bits[pages]).reshape(-1, width)[:n]
        for i in range(lo, hi):
            seen = k[:pos[i] + 1]
            s = bf16_bits_to_f64(q_bits[i]) @ seen.T * float(np.float32(scale))
            top = s.max(-1, keepdims=True)
            with np.errstate(invalid="ignore"):                # infinities among the scores or the values
                p = np.exp(s - top)
                z = p.sum(-1, keepdims=True)
                out[i], size[i] = p / z @ seen[:, :dc], p / z @ np.abs(seen[:, :dc])
            lse[i] = (top + np.log(z))[:, 0]
    return out, lse, size
