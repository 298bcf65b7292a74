"""GPU decode over a cache of MX blocks against the float64 oracle on the values the cache stands for."""
import numpy as np
import pytest
import torch

import oracle
import paper_2609_35158_amd as pa
from gpu_helpers import bits, say
from mx_helpers import MxCase, check, dev

pytestmark = pytest.mark.gpu

FORMATS = (pa.MXFP4, pa.MXFP8)


def run(c, append=False, **kw):
    cache, bt, ctx, _, q, k_new, v_new = c.device(appended=not append)
    kw = dict(dict(scale=c.scale, return_lse=True), **kw)
    if append:
        out, lse = pa.decode_append_mx(q, k_new, v_new, cache, bt, ctx, c.max_kv, **kw)
    else:
        out, lse = pa.decode_mx(q, cache, bt, ctx, c.max_kv, **kw)
    torch.cuda.synchronize()
    return out, lse, cache


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d", (64, 128))
@pytest.mark.parametrize("G", (1, 2, 4, 8))
@pytest.mark.parametrize("hkv", (1, 3))
def test_heads_and_lengths(fmt, d, G, hkv):
    ctx = [0, 1, 14, 15, 16, 17, 47, 62, 63, 64, 65, 127, 200, 511, 1000]
    say("decode_mx fmt=%d d=%d G=%d hkv=%d" % (fmt, d, G, hkv))
    c = MxCase(fmt, d, hkv, G, ctx, [1] * len(ctx), 7 * d + 10 * G + hkv + fmt)
    out, lse, _ = run(c)
    check(c, out, lse)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d", (64, 128))
@pytest.mark.parametrize("ctx", ([0], [15], [16], [5000], [3, 9000], [700] * 9, [2000, 40, 40, 40, 1500, 7], [33] * 90))
def test_one_long_few_and_many(fmt, d, ctx):
    """One sequence cut into many shares, shares over several sequences, and lengths far apart."""
    say("decode_mx fmt=%d d=%d ctx=%s" % (fmt, d, ctx[:6]))
    c = MxCase(fmt, d, 2, 4, ctx, [1] * len(ctx), 31 + d + len(ctx) + fmt)
    out, lse, _ = run(c)
    check(c, out, lse)


@pytest.mark.parametrize("hkv", (8, 12, 80))
def test_several_kv_heads_in_a_workgroup(hkv):
    say("decode_mx hkv=%d" % hkv)
    c = MxCase(4, 64, hkv, 1, [300, 310, 250, 305, 299, 301, 280, 320], [1] * 8, hkv)
    out, lse, _ = run(c)
    check(c, out, lse)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d", (64, 128))
def test_append_is_the_append_and_the_decode(fmt, d):
    ctx = [0, 15, 16, 31, 100, 1000, 47]
    say("decode_append_mx fmt=%d d=%d" % (fmt, d))
    c = MxCase(fmt, d, 3, 2, ctx, [1] * len(ctx), 5 + d + fmt)
    out, lse, cache = run(c, append=True)
    assert np.array_equal(cache.cpu().numpy(), c.after)
    out2, lse2, _ = run(c)
    assert torch.equal(out, out2) and torch.equal(lse, lse2)
    check(c, out, lse)


def test_more_sequences_than_one_group():
    rng = np.random.default_rng(1)
    ctx = rng.integers(0, 40, size=1100)
    say("decode_append_mx of 1100 sequences")
    c = MxCase(4, 64, 1, 2, ctx, [1] * len(ctx), 77)
    out, lse, cache = run(c, append=True)
    assert np.array_equal(cache.cpu().numpy(), c.after)
    check(c, out, lse)


@pytest.mark.parametrize("fmt", FORMATS)
def test_a_steep_softmax_and_tiny_and_huge_values(fmt):
    """Scores far apart (the running maximum has to move), values of very different size."""
    say("decode_mx extremes fmt=%d" % fmt)
    c = MxCase(fmt, 128, 2, 4, [3000, 130], [1, 1], 9 + fmt, q_gain=20.0)
    out, lse, _ = run(c)
    check(c, out, lse)
    c = MxCase(fmt, 128, 2, 4, [500], [1], 10 + fmt)
    vs = slice(c.after.shape[2] - 64, None)
    rng = np.random.default_rng(3)
    c.after[:, :, vs] = rng.integers(1, 200, size=c.after[:, :, vs].shape)   # V scales of 2^-126 .. 2^72
    out, lse, _ = run(c)
    check(c, out, lse)


@pytest.mark.parametrize("fmt", FORMATS)
def test_nan_blocks_reach_their_own_sequence_only(fmt):
    say("decode_mx NaN fmt=%d" % fmt)
    c = MxCase(fmt, 128, 2, 2, [40, 90, 70], [1, 1, 1], 21)
    k_bad, v_bad = c.k_new.clone(), c.v_new.clone()
    k_bad[0, 0, 5] = float("nan")                                  # sequence 0, kv-head 0: every output
    v_bad[2, 1, 100] = float("inf")                                # sequence 2, kv-head 1: channels 96..127
    c.k_new, c.v_new = k_bad, v_bad
    clean = MxCase(fmt, 128, 2, 2, [40, 90, 70], [1, 1, 1], 21)
    ref, ref_lse, _ = run(clean, append=True)
    out, lse, _ = run(c, append=True)
    nan = torch.isnan(out)
    assert nan[0, :2].all() and torch.isnan(lse[0, :2]).all()
    assert nan[2, 2:, 96:].all() and not torch.isnan(lse[2]).any()
    want = torch.zeros_like(nan)
    want[0, :2] = True
    want[2, 2:, 96:] = True
    assert torch.equal(nan, want)
    assert torch.equal(out[~want], ref[~want]) and torch.equal(lse[0, 2:], ref_lse[0, 2:])


def test_lengths_past_the_bounds_write_nothing_and_bad_pages_stay_inside():
    say("decode_mx bad lengths and pages")
    c = MxCase(4, 64, 2, 2, [40, 90, 70], [1, 1, 1], 23)
    cache, bt, ctx, _, q, _, _ = c.device()
    out = torch.full_like(q, 3.0)
    lse = torch.full(q.shape[:2], 5.0, device="cuda")
    pa.decode_mx(q, cache, bt, ctx, 80, scale=c.scale, out=out, lse=lse)         # 91 keys, 80 allowed
    torch.cuda.synchronize()
    assert (out == 3.0).all() and (lse == 5.0).all()
    bt[0, 1], bt[2, 4] = -100, 1 << 30
    pa.decode_mx(q, cache, bt, ctx, c.max_kv, scale=c.scale, out=out, lse=lse)
    torch.cuda.synchronize()
    check(c, out, lse, rows=[1])


def test_two_graphs_of_one_workspace_and_other_streams():
    say("decode_mx graphs")
    c = MxCase(4, 128, 4, 4, [900, 30, 333], [1, 1, 1], 25)
    e = MxCase(4, 128, 4, 4, [64, 2000, 5], [1, 1, 1], 26)
    devs = [x.device(appended=False) for x in (c, e)]
    descs = [pa.binding.make_desc(t[1], t[2], None, 3, 1, x.max_kv) for t, x in zip(devs, (c, e))]
    ws = torch.full((max(pa.workspace_bytes_mx(16, t[0], s) for t, s in zip(devs, descs)),), 255, dtype=torch.uint8, device="cuda")
    want = [run(x) for x in (c, e)]
    graphs, outs = [], []
    side = torch.cuda.Stream()
    for t, x in zip(devs, (c, e)):
        g = torch.cuda.CUDAGraph()
        out, lse = torch.zeros_like(t[4]), torch.zeros(t[4].shape[:2], device="cuda")
        with torch.cuda.graph(g, stream=side):
            pa.decode_append_mx(t[4], t[5], t[6], t[0], t[1], t[2], x.max_kv, scale=x.scale, out=out, lse=lse, workspace=ws)
        graphs.append(g)
        outs.append((out, lse))
    for _ in range(3):
        for g, (out, lse), (ref, ref_lse, cache), t in zip(graphs, outs, want, devs):
            out.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, ref) and torch.equal(lse, ref_lse) and torch.equal(t[0], cache)
        ws.fill_(77)
    cache, bt, ctx, _, q, _, _ = c.device()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        out, lse = pa.decode_mx(q, cache, bt, ctx, c.max_kv, scale=c.scale, return_lse=True, workspace=ws)
    side.synchronize()
    assert torch.equal(out, want[0][0]) and torch.equal(lse, want[0][1])


# Batches whose workgroups hold several kv-heads (8, 4, 2 of them; a last block that overlaps the one before), shares of
# whole and of cut sequences
BIG = [(4, 128, 8, 4, 64, 2048, 8192), (8, 128, 4, 8, 40, 4000, 9000), (4, 128, 2, 2, 256, 1000, 6000),
       (4, 64, 71, 1, 40, 700, 1000), (8, 64, 12, 2, 120, 800, 3000), (4, 128, 16, 1, 100, 900, 4000)]


@pytest.mark.parametrize("n", range(len(BIG)))
def test_large_batches(n):
    from mx_helpers import BigCase
    fmt, d, hkv, G, batch, lo, hi = BIG[n]
    say("decode_mx large fmt=%d d=%d hkv=%d G=%d batch=%d" % (fmt, d, hkv, G, batch))
    rng = np.random.default_rng(n)
    ctx = rng.integers(lo, hi, size=batch)
    c = BigCase(fmt, d, hkv, G, ctx, np.ones(batch, np.int64), n)
    lse = torch.full((batch, c.hq), float("nan"), device="cuda")
    out, lse = pa.decode_mx(c.q, c.cache, c.bt, c.ctx, c.max_kv, scale=c.scale, lse=lse)
    again, _ = pa.decode_mx(c.q, c.cache, c.bt, c.ctx, c.max_kv, scale=c.scale, return_lse=True)
    torch.cuda.synchronize()
    assert torch.isfinite(lse).all() and torch.equal(out, again)       # every row written; no result depends on timing
    c.check(out, lse, [0, 1, batch // 2, batch - 2, batch - 1] + [int(np.argmax(ctx)), int(np.argmin(ctx))])
