"""Helpers of the tests of the rotary position embedding."""
import numpy as np
import torch

import oracle
from gpu_helpers import bits


def dev(x, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(x, dtype))).cuda()


def bf16(x):
    return torch.from_numpy(np.asarray(x, np.float32)).to(torch.bfloat16)


def inv_freq(rotary, base=10000.0):
    return (float(base) ** (-np.arange(0, rotary, 2) / rotary)).astype(np.float32)


def rope_bound(rows_bits, want, rotary, interleaved, factor=1.0, weight_bits=None, eps=1e-6):
    """The error that the rotation's roundings allow for results `want` of bf16 rows [tokens][heads][d].

    Cosine and sine: the instructions are off by at most 2^-22.9 over the whole turn (measured at 2^22 arguments), the argument's rounding to 32
    bits by 2^-26 turns, 2^-23.3: together below 2^-22, times the pair's magnitudes.  The norm: a sum of d squares (8 in a row, then
    a tree) and a reciprocal root to 1.5 ulp, the products with the weight: below 2^-20 relative.  Three products and sums in 32
    bits: 2^-22 relative to the magnitudes.  The result is rounded to bf16: 2^-8 relative."""
    w = None if weight_bits is None else oracle.bf16_bits_to_f64(weight_bits)
    x = np.abs(oracle.norm_rows(oracle.bf16_bits_to_f64(rows_bits), w, eps))
    n = rotary // 2
    i, j = (np.arange(n) * 2, np.arange(n) * 2 + 1) if interleaved else (np.arange(n), np.arange(n) + n)
    size = x.copy()
    size[..., i] = size[..., j] = max(1.0, abs(factor)) * (x[..., i] + x[..., j])
    return 2.0 ** -8 * np.abs(want) + (2.0 ** -21 + (2.0 ** -20 if w is not None else 0.0)) * size + 1e-38


def check_rows(got_bits, rows_bits, pos, freq, interleaved, factor=1.0, weight_bits=None, eps=1e-6):
    want = oracle.rope_rows(rows_bits, pos, freq, interleaved, factor, weight_bits, eps)
    got = oracle.bf16_bits_to_f64(got_bits)
    off = np.abs(got - want)
    tol = rope_bound(rows_bits, want, 2 * len(freq), interleaved, factor, weight_bits, eps)
    bad = ~(off <= tol)
    assert not bad.any(), (np.argwhere(bad)[:4], float(off.max()))


class RopeCase:
    """New tokens of a batch: q, k, v as parts of one projection's output, pools with random pages, all on the GPU."""

    def __init__(self, hq, hkv, d, rotary, ctx, new, seed, interleaved=False, norm=False, factor=1.0, base=10000.0, spare=0,
                 bt_pad=2):
        rng = np.random.default_rng(seed)
        self.hq, self.hkv, self.d, self.interleaved, self.factor = hq, hkv, d, interleaved, factor
        self.ctx, self.new = np.asarray(ctx, np.int64), np.asarray(new, np.int64)
        self.cu = np.concatenate([[0], np.cumsum(self.new)])
        self.rows = int(self.cu[-1]) + spare                   # `spare` rows behind the last sequence
        self.pos = oracle.positions(self.ctx, self.cu, self.rows)
        pages = (self.ctx + self.new + 15) // 16
        self.num_pages = int(pages.sum()) + 3
        perm = rng.permutation(self.num_pages)
        self.bt = np.full((len(pages), int(pages.max()) + bt_pad), -5, np.int64)
        at = 0
        for b, n in enumerate(pages):
            self.bt[b, :n] = perm[at:at + n]
            at += n
        self.fused = bf16(rng.standard_normal((self.rows, hq + 2 * hkv + 1, d))).cuda()
        self.q, self.k, self.v = self.fused[:, :hq], self.fused[:, hq:hq + hkv], self.fused[:, hq + hkv:hq + 2 * hkv]
        self.freq = inv_freq(rotary, base)
        self.weights = [bf16(1 + 0.25 * rng.standard_normal(d)) if norm else None for _ in range(2)]
        self.pools = [bf16(rng.standard_normal((self.num_pages, hkv, 16, d))).cuda() for _ in range(2)]
        self.max_q, self.max_kv = max(1, int(self.new.max())), int((self.ctx + self.new).max())

    def rope(self):
        import paper_2609_35158_amd as pa
        w = [None if x is None else x.cuda() for x in self.weights]
        return pa.Rope(dev(self.freq, np.float32), interleaved=self.interleaved, factor=self.factor, q_weight=w[0], k_weight=w[1])

    def args(self):
        """block table, ctx, cu on the GPU."""
        return dev(self.bt), dev(self.ctx), dev(self.cu)

    def check(self, which, got, rows=None):
        """Rotated rows of q (0) or k (1) against the oracle's."""
        rows = self.pos >= 0 if rows is None else rows
        w = self.weights[which]
        check_rows(bits(got)[rows], bits((self.q, self.k)[which])[rows], self.pos[rows], self.freq, self.interleaved, self.factor,
                   None if w is None else bits(w))
