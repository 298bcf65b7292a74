"""Helpers of the tests on caches of latent rows: batches whose unowned bytes are arbitrary, the oracle's results, and error
bounds by counting roundings."""
import numpy as np
import torch

import oracle
from gpu_helpers import bits
from rope_helpers import bf16, dev, inv_freq

DIMS = {512: 64, 256: 32}


def random_bits(rng, *shape):
    return rng.integers(0, 1 << 16, size=shape).astype(np.uint16)


def from_bits(x):
    return torch.from_numpy(np.ascontiguousarray(x).view(np.int16)).view(torch.bfloat16)


class LatentCase:
    """Sequences of ctx cached tokens and new ones, all of them in the cache; every byte of it that no token owns is random (NaN and
    infinities among them)."""

    def __init__(self, heads, dc, ctx, new, seed, gain=1.5, spread=False, spare=0, bt_pad=2):
        rng = np.random.default_rng(seed)
        self.heads, self.dc, self.dr = heads, dc, DIMS[dc]
        self.width = self.dc + self.dr
        self.ctx, self.new = np.asarray(ctx, np.int64), np.asarray(new, np.int64)
        self.kv = self.ctx + self.new
        self.cu = np.concatenate([[0], np.cumsum(self.new)])
        self.owned = int(self.cu[-1])
        self.total = self.owned + spare
        pages = (np.maximum(self.kv, 1) + 15) // 16
        self.num_pages = int(pages.sum()) + 3
        perm = rng.permutation(self.num_pages)
        self.bt = np.full((len(pages), int(pages.max()) + bt_pad), -7, np.int64)
        self.cache = random_bits(rng, self.num_pages, 16, self.width)
        at = 0
        for b, n in enumerate(pages):
            self.bt[b, :n] = perm[at:at + n]
            at += n
            rows = rng.standard_normal((int(self.kv[b]), self.width))
            if spread:                                         # tokens of very different sizes: the maximum keeps moving
                rows *= np.exp2(rng.integers(-3, 4, size=(len(rows), 1)))
            flat = np.zeros((16 * n, self.width), np.uint16)
            flat[:] = random_bits(rng, 16 * n, self.width)
            flat[:len(rows)] = bits(bf16(rows))
            self.cache[self.bt[b, :n]] = flat.reshape(n, 16, self.width)
        self.scale = float(np.float32(192.0 ** -0.5))
        q = rng.standard_normal((self.total, heads, self.width)) * gain
        self.q = bf16(q)
        self.max_q, self.max_kv = max(1, int(self.new.max())), int(max(1, self.kv.max()))

    def args(self):
        """q, cache, block table, ctx, cu on the GPU."""
        return self.q.cuda(), from_bits(self.cache).cuda(), dev(self.bt), dev(self.ctx), dev(self.cu)

    def prefill(self, **kw):
        import paper_2609_35158_amd as pa
        q, cache, bt, ctx, cu = self.args()
        return pa.latent_prefill_append(q, cache, bt, ctx, cu, self.max_q, self.max_kv, self.scale, return_lse=True, **kw)

    def decode(self, **kw):
        import paper_2609_35158_amd as pa
        q, cache, bt, ctx, _ = self.args()
        return pa.latent_decode(q, cache, bt, ctx, self.max_kv, self.scale, return_lse=True, **kw)

    def oracle(self):
        """(out, lse, bound of out, bound of lse), in float64."""
        out, lse, size = oracle.latent_attention(bits(self.q), self.cache, self.bt, self.ctx, self.cu, self.dc, self.scale)
        # A score is `width` products summed in 32 bits: off by at most width 2^-24 scale sum |q k|, and by 2^-21 of itself with
        # its scaling, the maximum taken off and the exponential; scale sum |q k| <= scale |q| |k|.
        qn = np.linalg.norm(oracle.bf16_bits_to_f64(bits(self.q)), axis=-1)
        kn = 0.0
        for b, n in enumerate(self.kv):
            rows = oracle.bf16_bits_to_f64(self.cache[self.bt[b, :(n + 15) // 16]]).reshape(-1, self.width)[:n]
            rows = rows[np.isfinite(rows).all(-1)]             # scores of the others have no bound
            if len(rows):
                kn = max(kn, float(np.linalg.norm(rows, axis=-1).max()))
        score = self.scale * qn * kn
        off = (self.width * 2.0 ** -24 + 2.0 ** -21) * score
        # sums over the keys in 32 bits: at most a quarter of them in a row, and joins
        sums = (self.max_kv / 4 + 300) * 2.0 ** -24
        # a weight enters the second product in bf16 (2^-8), the result is rounded to bf16
        rel = (2 * off + 2 * sums + 2.0 ** -8)[..., None]
        return out, lse, 2.0 ** -8 * np.abs(out) + rel * size + 1e-30, off + sums + 2.0 ** -21 * np.abs(lse) + 1e-6


def check(case, out, lse):
    ref, ref_lse, tol, tol_lse = case.oracle()
    n = case.owned
    got = oracle.bf16_bits_to_f64(bits(out))
    bad = ~(np.abs(got - ref) <= tol)[:n]
    assert not bad.any(), (np.argwhere(bad)[:4], float(np.nanmax(np.abs(got - ref)[:n])))
    off = np.abs(lse.cpu().numpy().astype(np.float64) - ref_lse)
    assert (off <= tol_lse)[:n].all(), float(off[:n].max())
    # the bounds let every element be off as far as the worst; together they average out: two roundings to bf16, each
    # 2^-8 / sqrt(3) / sqrt(2) relative in the mean of squares (uniform within half a step, values over a binade)
    rel = np.linalg.norm((got - ref)[:n]) / np.linalg.norm(ref[:n])
    assert rel < 2.0 ** -8, rel


def torch_latent(q, rows, dc, scale):
    """One sequence in float64 on the GPU: q [n][H][width], rows [L][width], new token i at position L - n + i; (out, lse, size: out
    with |c| for c)."""
    n, h, _ = q.shape
    L = rows.shape[0]
    k = rows.double()
    kt, v = k.T.contiguous(), k[:, :dc].contiguous()
    hidden = torch.arange(L, device=q.device)[None, :] > L - n + torch.arange(n, device=q.device)[:, None]
    out = torch.empty((n, h, dc), dtype=torch.float64, device=q.device)
    size, lse = torch.empty_like(out), torch.empty((n, h), dtype=torch.float64, device=q.device)
    for g in range(h):
        s = (torch.matmul(q[:, g].double().contiguous(), kt) * float(np.float32(scale))).masked_fill_(hidden, float("-inf"))
        z = torch.logsumexp(s, -1)
        p = (s - z[:, None]).exp_()
        out[:, g], size[:, g], lse[:, g] = torch.matmul(p, v), torch.matmul(p, v.abs()), z
    return out, lse, size
