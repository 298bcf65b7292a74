"""Attention over a paged cache of latent rows where workgroups have much to do: shares of many tiles, tiles of more pages than the ids
that a wave holds at once, many sequences, and values that are not finite among them."""
import numpy as np
import pytest
import torch

import paper_2609_35158_amd as pa
from latent_helpers import LatentCase, check, torch_latent
from rope_helpers import dev, inv_freq

pytestmark = pytest.mark.gpu

SCALE = 192.0 ** -0.5


def _batch(heads, dc, ctx, new, seed):
    width = dc + {512: 64, 256: 32}[dc]
    kv = np.add(ctx, new)
    pages = (kv + 15) // 16
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    cache = torch.empty((int(pages.sum()) + 2, 16, width), dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    perm = np.random.default_rng(seed).permutation(len(cache))
    bt = np.full((len(kv), int(pages.max())), -1)
    at = 0
    for b, n in enumerate(pages):
        bt[b, :n] = perm[at:at + n]
        at += n
    cu = np.concatenate([[0], np.cumsum(new)])
    q = (torch.randn((int(cu[-1]), heads, width), generator=gen, device="cuda") * 1.15).to(torch.bfloat16)
    return q, cache, bt, cu, kv


def _check(q, cache, bt, kv, dc, out, lse):
    """One sequence, within the roundings: weights to bf16 (2^-8 of themselves: `size` times that), the result to bf16, and sums over
    the keys in 32 bits (below 2^-10 of `size`)."""
    rows = cache[dev(bt, np.int64)[:(kv + 15) // 16]].flatten(0, 1)[:kv]
    ref, ref_lse, size = torch_latent(q, rows, dc, SCALE)
    off = (out.double() - ref).abs()
    assert float((off - 2.0 ** -8 * ref.abs() - (2.0 ** -8 + 2.0 ** -10) * size).max()) <= 0
    assert float(off.norm() / ref.norm()) < 2.0 ** -8
    assert float((lse.double() - ref_lse).abs().max()) < 3e-5


@pytest.mark.parametrize("heads,dc,ctx,new", [(64, 512, [5000, 30], [500, 90]), (16, 512, [40, 700, 0], [230, 200, 261]), (20, 256, [3000, 0], [600, 900]),
                                              (128, 256, [100], [257])])
def test_many_tiles(heads, dc, ctx, new):
    q, cache, bt, cu, kv = _batch(heads, dc, ctx, new, seed=heads + dc)
    out, lse = pa.latent_prefill_append(q, cache, dev(bt), dev(ctx), dev(cu), max(new), int(kv.max()), SCALE, return_lse=True)
    for b, n in enumerate(kv):
        sl = slice(int(cu[b]), int(cu[b + 1]))
        _check(q[sl], cache, bt[b], int(n), dc, out[sl], lse[sl])


@pytest.mark.parametrize("heads,dc", [(16, 512), (32, 512), (128, 512), (16, 256), (48, 256)])
def test_shares_of_many_pages(heads, dc):
    """More than 64 pages a wave (16 rows a sequence) or 64 stages a share (more rows)."""
    ctx = np.random.default_rng(heads).integers(14000, 15000, size=90)
    q, cache, bt, cu, kv = _batch(heads, dc, ctx, np.ones(90, int), seed=heads)
    out, lse = pa.latent_decode(q, cache, dev(bt), dev(ctx), int(kv.max()), SCALE, return_lse=True)
    for b in (0, 17, 44, 45, 89):
        _check(q[b:b + 1], cache, bt[b], int(kv[b]), dc, out[b:b + 1], lse[b:b + 1])


@pytest.mark.parametrize("heads,dc", [(20, 256), (16, 512)])
def test_not_finite_among_many_tiles(heads, dc):
    """A new token's NaN reaches the tokens from it on, in every channel (its scores are NaN); its infinite channel of a score of minus
    infinity reaches theirs alone.  Tokens before it, and the other sequence, are what they are without."""
    new = [900, 700]
    q, cache, bt, cu, kv = _batch(heads, dc, [0, 11], new, seed=7)
    q[:, :, 5] = q[:, :, 5].abs() + 0.25                       # so that scores of a channel of minus infinity are minus infinity
    args = (dev(bt), dev([0, 11]), dev(cu), max(new), int(kv.max()), SCALE)
    clean, clean_lse = pa.latent_prefill_append(q, cache, *args, return_lse=True)
    for value in (float("nan"), float("-inf")):
        bad = cache.clone()
        for t in (13, 410, 411, 777):
            bad[int(bt[0, t // 16]), t % 16, 5] = value
        out, lse = pa.latent_prefill_append(q, bad, *args, return_lse=True)
        assert torch.equal(out[:13], clean[:13]) and torch.equal(out[900:], clean[900:])
        assert torch.equal(lse[:13], clean_lse[:13]) and torch.equal(lse[900:], clean_lse[900:])
        hit = out[13:900]
        if value != value:
            assert bool(torch.isnan(hit).all())
        else:
            assert bool(torch.isnan(hit[:, :, 5]).all())
            rest = torch.cat([hit[:, :, :5], hit[:, :, 6:]], -1)
            assert bool(torch.isfinite(rest).all()) and bool(torch.isfinite(lse[13:900]).all())


@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("heads,dc", [(64, 512), (100, 512), (128, 512), (128, 256), (8, 512)])
def test_not_finite_in_later_tokens(heads, dc, value):
    """A tile whose rows are all one token's, in a page with later tokens: what these hold does not reach it."""
    ctx, new = [5, 40, 0], [20, 3, 2]
    q, cache, bt, cu, kv = _batch(heads, dc, ctx, new, seed=heads)
    args = (dev(bt), dev(ctx), dev(cu), max(new), int(kv.max()), SCALE)
    bad, first = cache.clone(), [9, 1, 1]
    for b, i in enumerate(first):
        at = ctx[b] + i
        bad[int(bt[b, at // 16]), at % 16, 7:dc:3] = value
    out, lse = pa.latent_prefill_append(q, bad, *args, return_lse=True)
    for b, i in enumerate(first):
        lo, at, hi = int(cu[b]), int(cu[b]) + i, int(cu[b + 1])
        _check(q[lo:at], bad, bt[b], ctx[b] + i, dc, out[lo:at], lse[lo:at])
        assert not bool(torch.isfinite(out[at:hi, :, 7:dc:3]).any())


@pytest.mark.parametrize("batch", [63, 64, 65, 129])
@pytest.mark.parametrize("heads", [4, 20])
def test_batches_around_a_wave(batch, heads):
    """The cut is found in a wave's lanes up to 64 sequences; sequences without new tokens at both ends."""
    rng = np.random.default_rng(batch)
    new = rng.choice([0, 1, 2, 4], size=batch)
    new[0] = new[-1] = 0
    c = LatentCase(heads, 256, rng.integers(0, 70, size=batch), new, seed=batch)
    check(c, *c.prefill())
    c = LatentCase(heads, 256, rng.integers(0, 70, size=batch), np.ones(batch, int), seed=batch)
    check(c, *c.decode())


@pytest.mark.parametrize("batch", [64, 70])
@pytest.mark.parametrize("heads", [16, 32])
def test_one_length_that_cannot_be(batch, heads):
    """Of many sequences the last one's: nothing is written."""
    c = LatentCase(heads, 512, [40] * batch, [1] * batch, seed=batch)
    q, cache, bt, ctx, _ = c.args()
    out = torch.full((batch, heads, 512), 7.0, dtype=torch.bfloat16, device="cuda")
    ctx[-1] = 4000
    pa.latent_decode(q, cache, bt, ctx, c.max_kv, c.scale, out=out)
    assert bool((out == 7).all())
    ctx[-1] = 40
    check(c, *pa.latent_decode(q, cache, bt, ctx, c.max_kv, c.scale, return_lse=True))


def test_two_graphs_share_a_workspace():
    """Captured calls of different shapes and kernels on one workspace, replayed in turn with eager calls between."""
    cases = [LatentCase(16, 512, [3000, 7], [1, 1], seed=1), LatentCase(64, 512, [900, 0], [1, 30], seed=2)]
    args = [c.args() for c in cases]
    ws = torch.empty(80 << 20, dtype=torch.uint8, device="cuda")
    outs = [(torch.empty((c.total, c.heads, 512), dtype=torch.bfloat16, device="cuda"), torch.empty((c.total, c.heads), device="cuda")) for c in cases]

    def call(i, out, lse, work):
        c, (q, cache, bt, ctx, cu) = cases[i], args[i]
        pa.latent_prefill_append(q, cache, bt, ctx, cu, c.max_q, c.max_kv, c.scale, out=out, lse=lse, workspace=work)

    for i in (0, 1):
        call(i, *outs[i], ws)
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    for i, g in enumerate(graphs):
        with torch.cuda.graph(g):
            call(i, *outs[i], ws)
    for r in range(3):
        for i in (0, 1):
            args[i][0].normal_()
            outs[i][0].zero_()
        graphs[r % 2].replay()
        graphs[1 - r % 2].replay()
        graphs[r % 2].replay()
        for i in (0, 1):
            out, lse = torch.empty_like(outs[i][0]), torch.empty_like(outs[i][1])
            call(i, out, lse, ws)
            torch.cuda.synchronize()
            assert torch.equal(out, outs[i][0]) and torch.equal(lse, outs[i][1]), (r, i)


@pytest.mark.parametrize("heads,dc,tokens", [(16, 512, 40), (128, 512, 3), (5, 256, 9000)])
def test_append_into_the_rows_it_reads(heads, dc, tokens):
    """The queries' part rotated in place, in the tails of q: what it is from a buffer of its own."""
    dr = {512: 64, 256: 32}[dc]
    gen = torch.Generator(device="cuda").manual_seed(heads)
    rows = torch.randn((tokens, dc + dr), generator=gen, device="cuda").to(torch.bfloat16)
    q = torch.randn((tokens, heads, dc + dr), generator=gen, device="cuda").to(torch.bfloat16)
    rope = pa.Rope(dev(inv_freq(dr), np.float32), interleaved=heads == 5)
    pages = (tokens + 15) // 16
    bt, ctx, cu = dev(np.arange(pages)[None]), dev([0]), dev([0, tokens])
    got = []
    for own in (False, True):
        out, cache = q.clone(), pa.latent_cache(pages, dc, dr)
        pa.latent_append(out[..., dc:].clone() if own else out[..., dc:], rows, rope, out, cache, bt, ctx, cu, tokens, tokens)
        got.append((out, cache))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
    assert not torch.equal(got[0][0][1:, :, dc:], q[1:, :, dc:])
