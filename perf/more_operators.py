"""Performance cases of the rotary position operators and of attention over a paged cache of latent vectors.

Every case is one attention layer's share of a serving step on one GPU.  Before the call exist the pools or the cache, the
block table, the lengths, the rotation's frequencies and the output buffers, as an engine keeps them.

  op "rope"     rope_rows: queries and keys of the new tokens normalised per head and rotated (what goes into
                decode_append or a cache of MX blocks).
  op "append"   kv_append_rope: the same, with keys and values going into their pages.
  op "latent"   latent_append: a token's latent vector (normalised) and its shared rotated key part into the cache, the
                queries' rotated parts into the absorbed queries.
  op "decode"   latent_decode: one new token a sequence attends to its context, absorbed form.
  op "prefill"  latent_prefill_append: a turn's tokens, causal, absorbed form.

Fields: `batch` sequences with `new_lo`..`new_hi` new tokens each on `ctx_lo`..`ctx_hi` cached ones; `dist` is how contexts are
spread ("uniform", or "lognormal" around the geometric mean); `lengths` seeds the lengths; `heads` query heads.  Of the rotary
operators `kv_heads`, `dim`, `rotary` channels rotated, `pairs` ("halves": channel i with i + rotary / 2, "next": 2i with
2i + 1), `norm` whether heads are normalised.  Of the latent ones `dc` latent and `dr` rotated channels.

Values: projections of unit variance (rows are slices of the fused projections' outputs, hence strided); cached latent
vectors of unit variance, absorbed queries such that scores have a standard deviation of 2 under the scale 192^-1/2; every
slot of the pools and the cache holds data, also those no sequence owns.

A latent cache is bf16 [pages][16][dc + dr]: a token's latent vector, which is its value too, then its rotated key part.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

PAGE = 16
EPS = 1e-6
NOPE = 128                                                     # unrotated channels of a query head before absorption
LORA = 768                                                     # the queries' share of a fused down-projection


def _rope(name, op, heads, kv_heads, dim, rotary, pairs, norm, base, batch, ctx_lo, ctx_hi, new_lo=1, new_hi=1,
          dist="uniform", lengths=1):
    c = {"name": name, "op": op, "heads": heads, "kv_heads": kv_heads, "dim": dim, "rotary": rotary, "pairs": pairs,
         "norm": norm, "base": base, "batch": batch, "ctx_lo": ctx_lo, "ctx_hi": ctx_hi, "new_lo": new_lo, "new_hi": new_hi,
         "dist": dist, "lengths": lengths}
    if name is None:
        del c["name"]
    return c


def _latent(name, op, heads, dc, dr, batch, ctx_lo, ctx_hi, new_lo=1, new_hi=1, dist="uniform", lengths=1, pairs="next",
            base=10000.0):
    c = {"name": name, "op": op, "heads": heads, "dc": dc, "dr": dr, "pairs": pairs, "base": base, "batch": batch,
         "ctx_lo": ctx_lo, "ctx_hi": ctx_hi, "new_lo": new_lo, "new_hi": new_hi, "dist": dist, "lengths": lengths}
    if name is None:
        del c["name"]
    return c


def listed():
    return [
        # the rotation before one fused decode step: latency
        _rope("rope-step", "rope", 32, 8, 128, 128, "halves", True, 1e6, 64, 2048, 16384),
        # prompts of a small model on their way into a cache of MX blocks (head_dim 64, a part of it rotated, no norms)
        _rope("rope-prompts-d64", "rope", 16, 8, 64, 32, "next", False, 10000.0, 8, 0, 0, 500, 3001, lengths=5),
        # the append of one decode step
        _rope("append-step", "append", 32, 8, 128, 128, "halves", True, 1e6, 64, 2048, 16384, lengths=2),
        # tool outputs of odd lengths on top of long contexts
        _rope("append-turn", "append", 32, 4, 128, 128, "halves", True, 1e6, 16, 4096, 24576, 256, 2047, lengths=3),
        # the append of one step of latent rows, many heads
        _latent("latent-step", "latent", 128, 512, 64, 32, 1024, 32768, dist="lognormal", lengths=6),
        # a turn of latent rows, one shard's heads
        _latent("latent-turn", "latent", 16, 512, 64, 16, 4096, 24576, 256, 2047, lengths=7),
        # one trajectory left in the batch, one shard's heads: latency
        _latent("decode-1", "decode", 16, 512, 64, 1, 2731, 2731),
        # the ordinary decode step of a rollout, one shard's heads
        _latent("decode-64", "decode", 16, 512, 64, 64, 2048, 16384),
        # a decode worker that holds all heads, trajectories of very different lengths
        _latent("decode-32-lognormal-h128", "decode", 128, 512, 64, 32, 1024, 32768, dist="lognormal", lengths=42),
        # the ordinary turn: tool outputs of a few hundred tokens on top of long contexts
        _latent("prefill-turn", "prefill", 16, 512, 64, 4, 4096, 24576, 64, 400, lengths=4),
        # large turns of a few trajectories
        _latent("prefill-long", "prefill", 16, 512, 64, 6, 4096, 16384, 512, 2047, lengths=2),
        # the first turn of a small model: whole prompts, nothing cached, an odd number of heads
        _latent("prefill-prompts-dc256", "prefill", 20, 256, 32, 6, 0, 0, 300, 2000, lengths=9, pairs="halves"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "append", "latent", "decode", "decode", "prefill", "prefill"])
    while True:
        lengths, dist = rng.randrange(1, 1 << 20), rng.choice(["uniform", "lognormal"])
        pairs, base = rng.choice(["halves", "next"]), rng.choice([10000.0, 500000.0, 1e6])
        step = op == "decode" or (op != "prefill" and rng.random() < 0.4)
        batch = _log_int(rng, 1, 600 if step else 24)
        lo = _log_int(rng, 17, 8000) if step else rng.choice([0, _log_int(rng, 16, 8000)])
        hi = min(32000, _log_int(rng, lo, 4 * lo + 100)) if step else 2 * lo
        new = 1 if step else _log_int(rng, 2, 2048)
        new_hi = 1 if step else min(2048, new * rng.choice([1, 2, 4]))
        if op in ("rope", "append"):
            dim = rng.choice([64, 128, 128])
            kv_heads = rng.choice([1, 2, 4, 8])
            heads = kv_heads * rng.choice([1, 2, 4, 8])
            rotary = rng.choice([dim, dim, dim // 2, 16])
            c = _rope(None, op, heads, kv_heads, dim, rotary, pairs, rng.random() < 0.5, base, batch, lo, hi, new, new_hi, dist,
                      lengths)
        else:
            heads = rng.choice([1, 4, 8, 16, 16, 20, 32, 64, 128])
            dc, dr = rng.choice([(512, 64), (512, 64), (256, 32)])
            c = _latent(None, op, heads, dc, dr, batch, lo, hi, new, new_hi, dist, lengths, pairs, base)
        ctx, n = _lens(c)
        longest = int((ctx + n).max())
        room = batch * longest * 576 * 4 < 12e9                # what the plain form holds at once
        if op == "prefill":
            room = int(n.max()) * c["heads"] * longest * 4 < 6e9
        if room and _cost(c) <= _cost(_LARGEST):
            return c


def _lens(case):
    """(cached tokens, new tokens) of every sequence."""
    rng = np.random.default_rng(case["lengths"])
    n, lo, hi = case["batch"], case["ctx_lo"], case["ctx_hi"]
    if case["dist"] == "lognormal" and hi > lo > 0:
        x = rng.lognormal(0.5 * (math.log(lo) + math.log(hi)), 0.75, n)
        ctx = np.clip(np.rint(x), lo, hi).astype(np.int64)
    else:
        ctx = rng.integers(lo, hi, size=n, endpoint=True)
    return ctx, rng.integers(case["new_lo"], case["new_hi"], size=n, endpoint=True)


def work(case):
    ctx, new = _lens(case)
    rows, op, h = int(new.sum()), case["op"], case["heads"]
    pages = int(((ctx + new + PAGE - 1) // PAGE).sum())
    table = 4 * pages + 12 * len(ctx)
    new_table = 4 * int(((ctx + new + PAGE - 1) // PAGE - ctx // PAGE).sum()) + 12 * len(ctx)
    if op in ("rope", "append"):
        hkv, d, r = case["kv_heads"], case["dim"], case["rotary"]
        wide = (h + hkv * (1 if op == "rope" else 2)) * d
        return {"bytes": 4 * wide * rows + (new_table if op == "append" else 12 * len(ctx)) + 2 * r + (4 * d if case["norm"] else 0),
                "flops": rows * (h + hkv) * (3 * r + (4 * d if case["norm"] else 0))}
    dc, dr = case["dc"], case["dr"]
    if op == "latent":
        return {"bytes": 4 * (dc + dr + h * dr) * rows + new_table + 2 * dr + 2 * dc, "flops": rows * (4 * dc + 3 * dr * (h + 1))}
    keys, pairs = int((ctx + new).sum()), int((new * ctx + new * (new + 1) // 2).sum())
    return {"bytes": 2 * (dc + dr) * keys + rows * h * (2 * (2 * dc + dr) + 4) + table, "flops": 2 * h * (2 * dc + dr) * pairs}


def _cost(case):
    w = work(case)
    return w["bytes"] / 5e12 + w["flops"] / 1e15


_LARGEST = [c for c in listed() if c["name"] == "prefill-long"][0]


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16)


def prepare(case, seed):
    ctx, new = _lens(case)
    op, h = case["op"], case["heads"]
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    kv = ctx + new
    pages = (kv + PAGE - 1) // PAGE
    rows, num_pages = int(new.sum()), int(pages.sum()) + 7
    # pages of every sequence at random places; table entries past a sequence's end are 0
    perm = rng.permutation(num_pages).astype(np.int32)
    table = np.zeros((len(pages), int(pages.max())), np.int32)
    at = 0
    for b, n in enumerate(pages):
        table[b, :n] = perm[at:at + n]
        at += n
    st = {"op": op, "rows": rows, "max_q": int(new.max()), "max_kv": int(kv.max()), "num_pages": num_pages,
          "pairs": case["pairs"], "lens": list(zip(ctx.tolist(), new.tolist())), "workspace": None, "rope": None,
          "table": torch.from_numpy(table).cuda(), "ctx": torch.from_numpy(ctx.astype(np.int32)).cuda(),
          "cu": None if _single(new) else torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)).cuda()}
    if op in ("rope", "append"):
        hkv, d, r = case["kv_heads"], case["dim"], case["rotary"]
        fused = _normal(gen, rows, h + 2 * hkv, d)              # one projection's output: queries, keys, values
        st.update(q=fused[:, :h], k=fused[:, h:h + hkv], v=fused[:, h + hkv:],
                  q_out=torch.zeros((rows, h, d), dtype=torch.bfloat16, device="cuda"))
        if op == "append":
            st.update(k_pool=_normal(gen, num_pages, hkv, PAGE, d), v_pool=_normal(gen, num_pages, hkv, PAGE, d))
        else:
            st.update(k_out=torch.zeros((rows, hkv, d), dtype=torch.bfloat16, device="cuda"))
        w = [(1.0 + 0.25 * torch.randn(d, generator=gen, device="cuda")).to(torch.bfloat16) if case["norm"] else None
             for _ in range(2)]
        st.update(q_weight=w[0], k_weight=w[1])
    else:
        dc, dr = case["dc"], case["dr"]
        r = dr
        cache = torch.empty((num_pages, PAGE, dc + dr), dtype=torch.bfloat16, device="cuda")
        for p in range(0, num_pages, 1 << 14):                  # a part of the pages at a time
            cache[p:p + (1 << 14)].normal_(generator=gen)
        st.update(cache=cache, dc=dc, dr=dr, q=_normal(gen, rows, h, dc + dr).mul_(2.0 * math.sqrt(192.0 / (dc + dr))))
        if op == "latent":
            st.update(new=_normal(gen, rows, LORA + dc + dr)[:, LORA:], q_rope=_normal(gen, rows, h, NOPE + dr)[..., NOPE:],
                      k_weight=(1.0 + 0.25 * torch.randn(dc, generator=gen, device="cuda")).to(torch.bfloat16), q_weight=None)
        else:
            st.update(scale=192.0 ** -0.5, out=torch.zeros((rows, h, dc), dtype=torch.bfloat16, device="cuda"),
                      lse=torch.zeros((rows, h), dtype=torch.float32, device="cuda"))
    st["inv_freq"] = torch.from_numpy((case["base"] ** (-np.arange(0, r, 2) / r)).astype(np.float32)).cuda()
    return st


def _single(new):
    """Whether every sequence has one new token, which the calls take as no cu_q_lens."""
    return bool((new == 1).all())


def _run_own(st):
    import paper_2609_35158_amd as pa
    op, table, ctx, cu = st["op"], st["table"], st["ctx"], st["cu"]
    if op in ("rope", "append", "latent") and st["rope"] is None:   # a model's layer keeps it
        st["rope"] = pa.Rope(st["inv_freq"], interleaved=st["pairs"] == "next", q_weight=st["q_weight"],
                             k_weight=st["k_weight"], eps=EPS)
    if op == "rope":
        return list(pa.rope_rows(st["q"], st["k"], st["rope"], ctx, cu, st["max_q"], q_out=st["q_out"], k_out=st["k_out"]))
    if op == "append":
        q = pa.kv_append_rope(st["q"], st["k"], st["v"], st["rope"], st["k_pool"], st["v_pool"], table, ctx, cu, st["max_q"],
                              st["max_kv"], q_out=st["q_out"])
        return [q, st["k_pool"], st["v_pool"]]
    if op == "latent":
        pa.latent_append(st["q_rope"], st["new"], st["rope"], st["q"], st["cache"], table, ctx, cu, st["max_q"], st["max_kv"])
        return [st["q"], st["cache"]]
    if st["workspace"] is None:                                # an engine keeps one workspace for its calls
        desc = pa.binding.make_desc(table, ctx, cu, st["rows"], st["max_q"], st["max_kv"])
        st["workspace"] = torch.empty(pa.workspace_bytes_latent(st["q"].shape[1], st["cache"], desc), dtype=torch.uint8,
                                      device="cuda")
    kept = {"scale": st["scale"], "out": st["out"], "lse": st["lse"], "workspace": st["workspace"]}
    if op == "decode":
        return list(pa.latent_decode(st["q"], st["cache"], table, ctx, st["max_kv"], **kept))
    return list(pa.latent_prefill_append(st["q"], st["cache"], table, ctx, cu, st["max_q"], st["max_kv"], **kept))


def _places(st):
    """(sequence, position) of every new token's row."""
    dev = st["ctx"].device
    if st["cu"] is None:
        return torch.arange(st["rows"], device=dev), st["ctx"].long()
    seq = torch.repeat_interleave(torch.arange(st["ctx"].numel(), device=dev), st["cu"].diff(), output_size=st["rows"])
    return seq, st["ctx"].long()[seq] + torch.arange(st["rows"], device=dev) - st["cu"].long()[seq]


def _normed(x, weight):
    """Rows [..., d] in 32 bits, with a weight over their root mean square."""
    x = x.float()
    return x if weight is None else x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight.float()


def _rotated(x, st, pos):
    """The first channels of rows [tokens, heads, d] (32 bits) rotated by the tokens' positions."""
    angle = pos.double()[:, None, None] * st["inv_freq"].double()
    cos, sin = angle.cos().float(), angle.sin().float()
    r = 2 * cos.shape[-1]
    if st["pairs"] == "next":
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([y, x[..., r:]], -1)


def _attention(q, k, dc, scale, hidden):
    """Queries [..., rows, d] over keys [..., L, d] whose first dc channels are the values; hidden broadcasts to [..., rows, L]."""
    s = torch.matmul(q, k.transpose(-1, -2)).mul_(scale).masked_fill_(hidden, -math.inf)
    top = s.amax(-1, keepdim=True)
    s = s.sub_(top).exp_()
    total = s.sum(-1, keepdim=True)
    return torch.matmul(s, k[..., :dc]) / total, (top + total.log()).squeeze(-1)


def run(st):
    if own:
        return _run_own(st)
    op = st["op"]
    if op in ("rope", "append", "latent"):
        seq, pos = _places(st)
        page, slot = st["table"][seq, pos // PAGE].long(), pos % PAGE
    if op in ("rope", "append"):
        st["q_out"].copy_(_rotated(_normed(st["q"], st["q_weight"]), st, pos))
        k = _rotated(_normed(st["k"], st["k_weight"]), st, pos).to(torch.bfloat16)
        if op == "rope":
            st["k_out"].copy_(k)
            return [st["q_out"], st["k_out"]]
        st["k_pool"][page, :, slot], st["v_pool"][page, :, slot] = k, st["v"]
        return [st["q_out"], st["k_pool"], st["v_pool"]]
    dc = st["dc"]
    if op == "latent":
        c = _normed(st["new"][:, :dc], st["k_weight"])
        r = _rotated(st["new"][:, None, dc:].float(), st, pos)[:, 0]
        st["cache"][page, slot] = torch.cat([c, r], -1).to(torch.bfloat16)
        st["q"][..., dc:] = _rotated(st["q_rope"].float(), st, pos).to(torch.bfloat16)
        return [st["q"], st["cache"]]
    q, cache, table, width = st["q"].float(), st["cache"], st["table"].long(), st["cache"].shape[2]
    if op == "decode":                                         # all sequences at once, padded to the longest
        k = cache[table].float().view(table.shape[0], -1, width)
        hidden = torch.arange(k.shape[1], device=k.device) > st["ctx"].long()[:, None, None]
        o, lse = _attention(q, k, dc, st["scale"], hidden)
        return [o.to(torch.bfloat16), lse]
    out, lses, at = [], [], 0
    for b, (c, n) in enumerate(st["lens"]):                    # a sequence at a time
        k = cache[table[b, :(c + n + PAGE - 1) // PAGE]].float().view(-1, width)[:c + n]
        h = q.shape[1]
        last = c + torch.arange(n, device=k.device).repeat_interleave(h)
        o, lse = _attention(q[at:at + n].reshape(n * h, width), k, dc, st["scale"],
                            torch.arange(c + n, device=k.device) > last[:, None])
        out.append(o.view(n, h, dc).to(torch.bfloat16))
        lses.append(lse.view(n, h))
        at += n
    return [torch.cat(out), torch.cat(lses)]


def _turned(x, angle, pairs):
    """Rows [tokens, heads, 2 n] in 64 bits, their channel pairs as complex numbers turned by angle [tokens, n]."""
    z = x.unflatten(-1, (-1, 2)) if pairs == "next" else x.unflatten(-1, (2, -1)).transpose(-1, -2)
    z = torch.view_as_complex(z.contiguous()) * torch.polar(torch.ones_like(angle), angle)[:, None]
    z = torch.view_as_real(z)
    return (z if pairs == "next" else z.transpose(-1, -2)).flatten(-2)


def exact(case, seed):
    """The same in 64 bits, attention one sequence and a few heads at a time."""
    st = prepare(case, seed)
    ctx, new = _lens(case)
    op, r = case["op"], 2 * st["inv_freq"].numel()
    dev = st["ctx"].device
    where = [(b, c + i) for b, (c, n) in enumerate(zip(ctx.tolist(), new.tolist())) for i in range(n)]
    if op in ("rope", "append", "latent"):
        seq, pos = torch.tensor(where, device=dev).T
        slots = st["table"][seq, pos // PAGE].long() * PAGE + pos % PAGE
        angle = pos.double()[:, None] * st["inv_freq"].double()

        def turn(x, weight):
            x = x.double()
            if weight is not None:
                x = x / (x.pow(2).mean(-1, keepdim=True) + EPS).sqrt() * weight.double()
            return torch.cat([_turned(x[..., :r], angle, case["pairs"]), x[..., r:]], -1)
    if op in ("rope", "append"):
        q, k = turn(st["q"], st["q_weight"]), turn(st["k"], st["k_weight"])
        if op == "rope":
            return [q, k]
        pools = []
        for pool, x in ((st["k_pool"], k), (st["v_pool"], st["v"].double())):
            p = pool.double().transpose(1, 2).flatten(0, 1)     # [slots, kv-heads, d]
            p[slots] = x
            pools.append(p.unflatten(0, (-1, PAGE)).transpose(1, 2).contiguous())
        return [q] + pools
    dc, h = case["dc"], case["heads"]
    if op == "latent":
        c = st["new"][:, :dc].double()
        c = c / (c.pow(2).mean(-1, keepdim=True) + EPS).sqrt() * st["k_weight"].double()
        cache = st["cache"].double().flatten(0, 1)
        cache[slots] = torch.cat([c, turn(st["new"][:, None, dc:], None)[:, 0]], -1)
        return [torch.cat([st["q"][..., :dc].double(), turn(st["q_rope"], None)], -1), cache.view(st["cache"].shape)]
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device=dev)
    lse = torch.zeros(st["lse"].shape, dtype=torch.float64, device=dev)
    start = np.concatenate([[0], np.cumsum(new)]).astype(int)
    for b, (c, n) in enumerate(zip(ctx.tolist(), new.tolist())):
        L, at = c + n, slice(int(start[b]), int(start[b]) + n)
        k = st["cache"][st["table"][b, :(L + PAGE - 1) // PAGE].long()].double().flatten(0, 1)[:L]
        kt, v = k.T.contiguous(), k[:, :dc].contiguous()
        hidden = torch.arange(L, device=dev)[None, :] > c + torch.arange(n, device=dev)[:, None]
        step = h if n == 1 else 1                              # heads taken together
        for g in range(0, h, step):
            q = st["q"][at, g:g + step].double().reshape(n * step, -1)
            s = torch.matmul(q, kt) * float(np.float32(st["scale"]))
            s.masked_fill_(hidden if step == 1 else hidden.expand(step, L), -math.inf)
            z = torch.logsumexp(s, -1)
            o = torch.matmul(s.sub_(z[:, None]).exp_(), v)
            out[at, g:g + step], lse[at, g:g + step] = o.view(n, step, dc), z.view(n, step)
    return [out, lse]
