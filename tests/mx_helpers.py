"""Helpers of the tests on caches of MX blocks: caches whose unowned bytes are arbitrary, the oracle's results, and
error bounds by counting roundings."""
import numpy as np
import torch

import oracle
from gpu_helpers import bits


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def bf16(x):
    return torch.from_numpy(np.asarray(x, np.float32)).to(torch.bfloat16)


class MxCase:
    """Sequences of ctx cached tokens and new ones, the cache as it stands before the new tokens are appended: the
    cached tokens' blocks hold quantised rows, every other byte is random (NaN scales and codes among them)."""

    def __init__(self, fmt, d, hkv, G, ctx, new, seed, extra_pages=3, stride_pad=2, q_gain=1.5):
        rng = np.random.default_rng(seed)
        self.fmt, self.d, self.hkv, self.G, self.hq = fmt, d, hkv, G, hkv * G
        self.ctx, self.new = np.asarray(ctx, np.int32), np.asarray(new, np.int32)
        self.kv = self.ctx + self.new
        pages = (np.maximum(self.kv, 1) + 15) // 16
        self.num_pages = int(pages.sum()) + extra_pages
        perm = rng.permutation(self.num_pages).astype(np.int32)
        self.bt = np.full((len(pages), int(pages.max()) + stride_pad), -7, np.int32)
        at = 0
        for b, n in enumerate(pages):
            self.bt[b, :n] = perm[at:at + n]
            at += n
        self.cu = np.concatenate([[0], np.cumsum(self.new)]).astype(np.int32)
        self.total, self.max_q, self.max_kv = int(self.new.sum()), int(self.new.max()), int(self.kv.max())
        self.scale = float(np.float32(1.0 / np.sqrt(d)))
        cached = int(self.ctx.sum())
        old = [bits(bf16(rng.standard_normal((cached, hkv, d)) * np.exp2(rng.integers(-2, 3, size=(cached, hkv, 1)))))
               for _ in range(2)]
        cache = rng.integers(0, 256, size=(self.num_pages, hkv, oracle.mx_block_bytes(d, fmt)), dtype=np.uint8)
        self.cache = oracle.mx_append(cache, fmt, old[0], old[1], self.bt, np.zeros(len(pages), np.int64),
                                      np.concatenate([[0], np.cumsum(self.ctx)]))
        self.k_new, self.v_new = (bf16(rng.standard_normal((self.total, hkv, d))) for _ in range(2))
        self.q = bf16(q_gain * rng.standard_normal((self.total, self.hq, d)))
        self.after = oracle.mx_append(self.cache, fmt, bits(self.k_new), bits(self.v_new), self.bt, self.ctx, self.cu)

    def device(self, appended=True):
        """cache, block table, ctx, cu, q, k_new, v_new on the GPU."""
        return (dev(self.after if appended else self.cache), dev(self.bt), dev(self.ctx), dev(self.cu), self.q.cuda(),
                self.k_new.cuda(), self.v_new.cuda())

    def oracle(self):
        """(out, lse, bound of out, bound of lse), in float64."""
        k, v = oracle.mx_pools(self.after, self.d, self.fmt)
        args = (self.bt, self.ctx, self.cu, self.scale)
        out, lse = oracle.attention(bits(self.q), k, v, *args)
        size, _ = oracle.attention(bits(self.q), k, v & 0x7fff, *args)     # sum of weight times |v|
        # A score is D products summed in 32 bits: off by at most D 2^-24 scale sum |q k|, and by 2^-22 of
        # itself with its scaling and the exponential; scale sum |q k| <= scale |q| |k|.
        qn = np.linalg.norm(oracle.bf16_bits_to_f64(bits(self.q)), axis=-1)                # [total, hq]
        kn = 0.0
        for b in range(len(self.ctx)):
            pages = self.bt[b, :(self.kv[b] + 15) // 16]
            rows = oracle.bf16_bits_to_f64(k[pages]).transpose(0, 2, 1, 3).reshape(-1, self.hkv, self.d)[:self.kv[b]]
            if len(rows):
                kn = max(kn, float(np.nanmax(np.linalg.norm(rows, axis=-1))))
        score = self.scale * qn * kn
        off = self.d * 2.0 ** -24 * score + 2.0 ** -21 * score
        # sums over n keys in 32 bits, in lanes, units and runs of their own: at most n / 4 + 64 additions in a row
        sums = (self.max_kv / 4 + 64) * 2.0 ** -24
        # weights enter P.V in bf16 once (prefill: 2^-8) or in two parts (2^-16), the result is rounded to bf16
        weight = 2.0 ** -16 if self.max_q == 1 else 2.0 ** -8
        rel = (2 * off + 2 * sums + weight)[..., None]
        return out, lse, 2.0 ** -8 * np.abs(out) + rel * size + 1e-30, off + sums + 2.0 ** -21 * np.abs(lse) + 1e-6


def check(case, out, lse, rows=None):
    ref, ref_lse, tol, tol_lse = case.oracle()
    got = oracle.bf16_bits_to_f64(bits(out))
    rows = np.arange(case.total) if rows is None else rows
    bad = ~(np.abs(got - ref) <= tol)[rows]
    assert not bad.any(), (np.argwhere(bad)[:4], float(np.abs(got - ref)[rows].max()))
    if lse is not None:
        off = np.abs(lse.cpu().numpy().astype(np.float64) - ref_lse)
        assert (off <= tol_lse)[rows].all(), (float(off[rows].max()), float(tol_lse[rows].min()))
