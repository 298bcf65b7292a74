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


def torch_attention(q, k, v, scale):
    """One sequence in float64 on the GPU: q [n][hq][d], k and v [L][hkv][d], new token i at position L - n + i; (out, lse)."""
    n, hq, d = q.shape
    L, hkv, _ = k.shape
    G = hq // hkv
    q = q.double().view(n, hkv, G, d).permute(1, 2, 0, 3).reshape(hkv, G * n, d)
    s = torch.matmul(q, k.double().permute(1, 2, 0).contiguous()) * float(np.float32(scale))
    hidden = torch.arange(L, device=q.device)[None, :] > L - n + torch.arange(n, device=q.device)[:, None]
    s = s.view(hkv, G, n, L).masked_fill_(hidden, float("-inf"))
    lse = torch.logsumexp(s, -1)
    o = torch.matmul((s - lse[..., None]).exp_().view(hkv, G * n, L), v.double().transpose(0, 1).contiguous())
    return o.view(hkv, G, n, d).permute(2, 0, 1, 3).reshape(n, hq, d), lse.permute(2, 0, 1).reshape(n, hq)


class BigCase:
    """Sequences too large for the numpy oracle: a cache of quantised normal rows in random pages, on the GPU."""

    def __init__(self, fmt, d, hkv, G, ctx, new, seed):
        import paper_2609_35158_amd as pa
        rng = np.random.default_rng(seed)
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.d, self.hkv, self.hq, self.scale = d, hkv, hkv * G, float(np.float32(d ** -0.5))
        self.kv = np.asarray(ctx) + np.asarray(new)
        pages = (self.kv + 15) // 16
        num_pages = int(pages.sum()) + 5
        perm = rng.permutation(num_pages).astype(np.int32)
        bt = np.full((len(pages), int(pages.max())), -1, np.int32)
        at = 0
        for b, n in enumerate(pages):
            bt[b, :n] = perm[at:at + n]
            at += n
        # every page once, as pages of one long sequence
        self.cache = pa.mx_cache(num_pages, hkv, d, fmt)
        every, step = dev(np.arange(num_pages, dtype=np.int32)[None]), 4096
        for p in range(0, num_pages, step):
            n = 16 * min(step, num_pages - p)
            k, v = (torch.randn((n, hkv, d), generator=gen, device="cuda", dtype=torch.bfloat16) for _ in range(2))
            pa.kv_append_mx(k, v, self.cache, every, dev(np.array([16 * p], np.int32)), dev(np.array([0, n], np.int32)), n, 16 * num_pages)
        self.bt, self.ctx = dev(bt), dev(np.asarray(ctx, np.int32))
        self.cu = dev(np.concatenate([[0], np.cumsum(new)]).astype(np.int32))
        self.starts, self.new = np.concatenate([[0], np.cumsum(new)]), np.asarray(new)
        self.q = torch.randn((int(self.new.sum()), self.hq, d), generator=gen, device="cuda", dtype=torch.bfloat16)
        self.max_q, self.max_kv = int(self.new.max()), int(self.kv.max())

    def check(self, out, lse, seqs):
        """Sampled sequences: out within a rounding to bf16 and the weights' (2^-9 of a value of about 1), lse."""
        import paper_2609_35158_amd as pa
        zero = torch.zeros(1, dtype=torch.int32, device="cuda")
        for b in seqs:
            n, r = int(self.kv[b]), slice(int(self.starts[b]), int(self.starts[b] + self.new[b]))
            k, v = pa.kv_pack_mx(self.cache, self.bt[b:b + 1], zero, dev(np.array([0, n], np.int32)), n, n, n)
            ref, ref_lse = torch_attention(self.q[r], k, v, self.scale)
            off = (out[r].double() - ref).abs()
            assert bool((off <= 2.0 ** -8 * ref.abs() + 2.0 ** -9 * 4).all()), (b, float(off.max()))
            rel = float(off.norm() / ref.norm())
            assert rel < 2.6e-3, (b, rel)          # 2^-8 / sqrt(3) / 2 from either rounding, in the 2-norm
            assert float((lse[r].double() - ref_lse).abs().max()) < 2e-5, b
