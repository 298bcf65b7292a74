"""CPU oracle for a KV cache in MX blocks (quantised append, read-back).

TEST INFRASTRUCTURE ONLY, numpy and float64, written from the format's definition; it shares no code
with the library.  32 neighbouring channels of a token and kv-head share a scale 2^(s - 127); elements
are E2M1 (4 bits) or E4M3 (8 bits).  Attention over such a cache is `oracle.attention` over the pools that
`mx_pools` reads back: every value is exact in bf16.
"""
from __future__ import annotations

from typing import Optional, Tuple

import numpy as np

from .paged_attention import PAGE, _q_lens, _q_starts, bf16_bits_to_f64, f64_to_bf16_bits

# format -> (exponent of the largest binade, least exponent, bits after the leading one, largest value)
_ELEMENT = {4: (2, 0, 1, 6.0), 8: (8, -6, 3, 448.0)}


def mx_element_values(fmt: int) -> np.ndarray:
    """The value of every code: sign, exponent, mantissa, in 4 or 8 bits."""
    _, e_min, m_bits, _ = _ELEMENT[fmt]
    code = np.arange(1 << fmt)
    m = code & ((1 << m_bits) - 1)
    e = (code >> m_bits) & ((1 << (fmt - 1 - m_bits)) - 1)
    mag = np.where(e > 0, np.ldexp((1 << m_bits) + m, e - 1 + e_min - m_bits), np.ldexp(m, e_min - m_bits))
    v = np.where(code >> (fmt - 1), -mag, mag).astype(np.float64)
    if fmt == 8:
        v[[0x7f, 0xff]] = np.nan
    return v


def mx_quantise(bits: np.ndarray, fmt: int) -> Tuple[np.ndarray, np.ndarray]:
    """bf16 bit patterns [..., d] -> (codes uint8 [..., d], scales uint8 [..., d / 32])."""
    e_max, _, _, most = _ELEMENT[fmt]
    x = bf16_bits_to_f64(bits)
    x = x.reshape(x.shape[:-1] + (x.shape[-1] // 32, 32))
    bad = ~np.isfinite(x).all(-1)
    x = np.where(bad[..., None], 0.0, x)
    top = np.abs(x).max(-1)
    s = np.ones(top.shape, np.int64)
    while (short := top > np.ldexp(1.75, s - 127 + e_max)).any():   # the least that holds it
        s += short
    y = np.ldexp(x, 127 - s[..., None])
    values = mx_element_values(fmt)[:1 << (fmt - 1)]               # of the codes without sign, rising
    values = values[np.isfinite(values)]
    a = np.minimum(np.abs(y), most)
    hi = np.searchsorted(values, a)                                # the first value >= a
    lo = np.maximum(hi - 1, 0)
    up, down = values[hi] - a, a - values[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    code = code | (np.signbit(y).astype(np.int64) << (fmt - 1))
    code[bad] = 0
    return (code.reshape(bits.shape).astype(np.uint8), np.where(bad, 255, s).astype(np.uint8))


def mx_values(codes: np.ndarray, scales: np.ndarray, fmt: int) -> np.ndarray:
    """float64 values of codes [..., d] under scales [..., d / 32]."""
    v = mx_element_values(fmt)[codes].reshape(codes.shape[:-1] + (codes.shape[-1] // 32, 32))
    s = scales.astype(np.int64)[..., None]
    return np.where(s == 255, np.nan, np.ldexp(v, s - 127)).reshape(codes.shape)


def mx_block_bytes(d: int, fmt: int) -> int:
    return 2 * PAGE * (d * fmt // 8 + d // 32)


def _places(slot: int, d: int, fmt: int):
    """Byte offsets in a block of the token at `slot`: K code bytes [d fmt / 8] in channel order, V code bytes
    the same, K scales [d / 32], V scales [d / 32]."""
    row, nb = d * fmt // 8, d // 32
    i, blk = np.arange(row), np.arange(nb)
    if fmt == 4:                                                   # a byte is a pair of channels
        v = i * PAGE + slot
    else:                                                          # a byte is a channel
        v = ((slot // 8) * (d // 2) + i // 2) * 16 + 2 * (slot % 8) + i % 2
    codes = PAGE * row
    return (slot * row + i, codes + v, 2 * codes + ((slot % 4) * nb + blk) * 4 + slot // 4,
            2 * codes + PAGE * nb + blk * PAGE + slot)


def _pack_codes(codes: np.ndarray, fmt: int) -> np.ndarray:
    return codes if fmt == 8 else (codes[..., 0::2] | (codes[..., 1::2] << 4)).astype(np.uint8)


def _unpack_codes(b: np.ndarray, fmt: int) -> np.ndarray:
    return b if fmt == 8 else np.stack([b & 15, b >> 4], -1).reshape(b.shape[:-1] + (2 * b.shape[-1],))


def mx_append(cache: np.ndarray, fmt: int, k_new: np.ndarray, v_new: np.ndarray, block_table: np.ndarray,
              ctx_lens: np.ndarray, cu_q_lens: Optional[np.ndarray]) -> np.ndarray:
    """A copy of the cache uint8 [num_pages][H_kv][block] with the rows bf16 [total_q][H_kv][d] appended."""
    out = np.array(cache, copy=True)
    d = k_new.shape[-1]
    kc, ks = mx_quantise(k_new, fmt)
    vc, vs = mx_quantise(v_new, fmt)
    kc, vc = _pack_codes(kc, fmt), _pack_codes(vc, fmt)
    starts, lens = _q_starts(cu_q_lens, len(ctx_lens)), _q_lens(cu_q_lens, len(ctx_lens))
    for b in range(len(ctx_lens)):
        for t in range(int(lens[b])):
            pos, r = int(ctx_lens[b]) + t, int(starts[b]) + t
            page = int(block_table[b][pos // PAGE])
            for at, x in zip(_places(pos % PAGE, d, fmt), (kc, vc, ks, vs)):
                out[page][:, at] = x[r]
    return out


def mx_pools(cache: np.ndarray, d: int, fmt: int) -> Tuple[np.ndarray, np.ndarray]:
    """The K and V pools, bf16 bit patterns [num_pages][H_kv][16][d], that a cache stands for."""
    k = np.empty(cache.shape[:2] + (PAGE, d), np.uint16)
    v = np.empty_like(k)
    for slot in range(PAGE):
        kc, vc, ks, vs = (cache[..., at] for at in _places(slot, d, fmt))
        with np.errstate(over="ignore", invalid="ignore"):
            k[:, :, slot] = f64_to_bf16_bits(mx_values(_unpack_codes(kc, fmt), ks, fmt))
            v[:, :, slot] = f64_to_bf16_bits(mx_values(_unpack_codes(vc, fmt), vs, fmt))
    return k, v


def mx_pack(cache: np.ndarray, d: int, fmt: int, block_table: np.ndarray, ctx_lens: np.ndarray,
            cu_q_lens: Optional[np.ndarray]) -> np.ndarray:
    """Token ranges read back: bf16 bit patterns [2][total][H_kv][d]."""
    k, v = mx_pools(cache, d, fmt)
    starts, lens = _q_starts(cu_q_lens, len(ctx_lens)), _q_lens(cu_q_lens, len(ctx_lens))
    out = np.zeros((2, int(np.sum(lens)), cache.shape[1], d), np.uint16)
    for b in range(len(ctx_lens)):
        for t in range(int(lens[b])):
            pos = int(ctx_lens[b]) + t
            page = int(block_table[b][pos // PAGE])
            out[0, starts[b] + t], out[1, starts[b] + t] = k[page, :, pos % PAGE], v[page, :, pos % PAGE]
    return out
