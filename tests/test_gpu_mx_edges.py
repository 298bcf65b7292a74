"""GPU calls on caches of MX blocks at their edges: blocks past 4 GiB, calls on two streams at once, pages that sequences
share, lengths past the bounds reported, long contexts of a turn whose keys are split."""
import numpy as np
import pytest
import torch

import oracle
import paper_2609_35158_amd as pa
from gpu_helpers import bits, say
from mx_helpers import BigCase, MxCase, dev

pytestmark = pytest.mark.gpu

FORMATS = (pa.MXFP4, pa.MXFP8)


@pytest.mark.parametrize("fmt", FORMATS)
def test_blocks_past_4_gib(fmt):
    """The same tokens in the last pages of a cache of over 4 GiB, of which the last start past it, and in a small one."""
    say("mx cache past 4 GiB fmt=%d" % fmt)
    hkv, G, d = 8, 4, 128
    block = pa.mx_block_bytes(d, fmt)
    n = np.array([1000, 17, 300])
    pages = (n + 15) // 16
    total = int(pages.sum())
    large = ((1 << 32) // (hkv * block)) + total + 9
    caches = [torch.empty((p, hkv, block), dtype=torch.uint8, device="cuda") for p in (large, total)]
    assert caches[0].numel() > 1 << 32
    bt = np.zeros((3, int(pages.max())), np.int32)
    at = 0
    for b in range(3):
        bt[b, :pages[b]] = np.arange(at, at + pages[b])
        at += pages[b]
    cu = dev(np.concatenate([[0], np.cumsum(n)]).astype(np.int32))
    zero, ctx = dev(np.zeros(3, np.int32)), dev((n - 1).astype(np.int32))
    gen = torch.Generator(device="cuda")
    gen.manual_seed(fmt)
    k, v = (torch.randn((int(n.sum()), hkv, d), generator=gen, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    q = torch.randn((int(n.sum()), hkv * G, d), generator=gen, device="cuda", dtype=torch.bfloat16)
    results = []
    for cache, shift in zip(caches, (large - total, 0)):
        table = dev(bt + np.int32(shift))
        cache[shift:shift + total].zero_()                       # slots behind the sequences' last tokens alike
        pa.kv_append_mx(k, v, cache, table, zero, cu, 1000, 1000)
        rows = pa.kv_pack_mx(cache, table, zero, cu, int(n.sum()), 1000, 1000)
        turn = pa.prefill_append_mx(q, cache, table, zero, cu, 1000, 1000, return_lse=True)
        step = pa.decode_mx(q[:3], cache, table, ctx, 1000, return_lse=True)
        new = pa.decode_append_mx(q[3:6], k[:3], v[:3], cache, table, ctx, 1000, return_lse=True)
        torch.cuda.synchronize()
        results.append((rows, *turn, *step, *new, cache[shift:shift + total]))
    for x, y in zip(*results):
        assert torch.equal(x, y)


def test_two_streams_at_once():
    """Steps of two batches, each on its own stream with its own workspace, beside each other."""
    say("mx calls on two streams")
    cases = [MxCase(4, 128, 8, 4, [900, 30, 333, 64], [1] * 4, 35), MxCase(8, 64, 3, 2, [2000, 5], [1] * 2, 36)]
    state, want = [], []
    for c in cases:
        cache, bt, ctx, _, q, k, v = c.device(appended=False)
        ws = torch.full((pa.workspace_bytes_mx(c.hq, cache, pa.binding.make_desc(bt, ctx, None, len(ctx), 1, c.max_kv)),), 255,
                        dtype=torch.uint8, device="cuda")
        ref = pa.decode_append_mx(q, k, v, cache.clone(), bt, ctx, c.max_kv, scale=c.scale, return_lse=True)
        state.append((cache, bt, ctx, q, k, v, ws, torch.cuda.Stream()))
        want.append(ref)
    torch.cuda.synchronize()
    results = [[], []]
    for _ in range(20):
        for i, (c, (cache, bt, ctx, q, k, v, ws, stream)) in enumerate(zip(cases, state)):
            with torch.cuda.stream(stream):
                results[i].append(pa.decode_append_mx(q, k, v, cache, bt, ctx, c.max_kv, scale=c.scale, return_lse=True,
                                                      workspace=ws))
    torch.cuda.synchronize()
    for i, c in enumerate(cases):
        assert all(torch.equal(o, want[i][0]) and torch.equal(s, want[i][1]) for o, s in results[i])
        assert np.array_equal(state[i][0].cpu().numpy(), c.after)


@pytest.mark.parametrize("fmt", FORMATS)
def test_sequences_that_share_pages(fmt):
    """A prefix in the same pages for every sequence, and the same sequence twice, give what their own copies give."""
    say("mx shared pages fmt=%d" % fmt)
    c = MxCase(fmt, 128, 2, 4, [600, 600, 600], [1] * 3, 45 + fmt)
    cache, bt, ctx, _, q, _, _ = c.device()
    shared = bt.clone()
    shared[1:, :38] = shared[0, :38].clone()                     # sequence 0's 38 pages, in sequence 1 and 2 too
    own = cache.clone()
    for b in (1, 2):
        own[bt[b, :38].long()] = cache[bt[0, :38].long()]
    q[2] = q[1]
    ctx[1:] = dev(np.array([590, 590], np.int32))
    got = pa.decode_mx(q, cache, shared, ctx, c.max_kv, scale=c.scale, return_lse=True)
    want = pa.decode_mx(q, own, bt, ctx, c.max_kv, scale=c.scale, return_lse=True)
    cu = dev(np.array([0, 1, 2, 3], np.int32))
    turn = pa.prefill_append_mx(q, cache, shared, ctx, cu, 1, c.max_kv, scale=c.scale, return_lse=True)
    turn2 = pa.prefill_append_mx(q, own, bt, ctx, cu, 1, c.max_kv, scale=c.scale, return_lse=True)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip((*got, *turn), (*want, *turn2)))
    assert torch.equal(turn[0][1], turn[0][2])


@pytest.mark.parametrize("batch", (5, 1030))
def test_lengths_past_the_bounds_are_reported(monkeypatch, batch):
    """With PEARL_DEBUG=1 a call whose lengths on the device pass its bounds is an error, in whichever group of sequences."""
    say("mx lengths reported batch=%d" % batch)
    c = MxCase(4, 64, 1, 2, [20] * batch, [1] * batch, batch)
    cache, bt, ctx, cu, q, _, _ = c.device()
    monkeypatch.setenv("PEARL_DEBUG", "1")
    pa.decode_mx(q, cache, bt, ctx, c.max_kv)
    pa.prefill_append_mx(q, cache, bt, ctx, cu, 1, c.max_kv)
    for b in (0, batch - 1):
        bad = ctx.clone()
        bad[b] = c.max_kv                                        # one key too many
        for call in (lambda out: pa.decode_mx(q, cache, bt, bad, c.max_kv, out=out),
                     lambda out: pa.prefill_append_mx(q, cache, bt, bad, cu, 1, c.max_kv, out=out)):
            out = torch.full_like(q, 3.0)
            with pytest.raises(pa.PearlError, match="violate the host bounds"):
                call(out)
            group = slice(0, 1024) if b == 0 else slice(batch // 1024 * 1024, batch)
            assert bool((out[group] == 3.0).all())


# few new tokens on long contexts (keys split over workgroups), a batch of many tiles, both formats and head dims
TURNS = [(4, 128, 8, 4, [9000, 15000], [40, 130]), (8, 128, 2, 8, [7000], [33]), (4, 64, 4, 2, [3000, 12000, 1000], [300, 7, 600]),
         (8, 64, 8, 2, [1000] * 5, [700, 900, 1, 333, 1024])]


@pytest.mark.parametrize("n", range(len(TURNS)))
def test_turns_on_long_contexts(n):
    fmt, d, hkv, G, ctx, new = TURNS[n]
    say("prefill_mx large fmt=%d d=%d hkv=%d G=%d ctx=%s new=%s" % (fmt, d, hkv, G, ctx, new))
    c = BigCase(fmt, d, hkv, G, ctx, new, 60 + n)
    lse = torch.full((int(c.new.sum()), c.hq), float("nan"), device="cuda")
    out, lse = pa.prefill_append_mx(c.q, c.cache, c.bt, c.ctx, c.cu, c.max_q, c.max_kv, scale=c.scale, lse=lse)
    torch.cuda.synchronize()
    c.check(out, lse, range(len(ctx)))


@pytest.mark.parametrize("fmt,d,hkv,lo,hi", ((4, 128, 8, 1, 400), (8, 64, 16, 30, 200), (4, 64, 8, 100, 103)))
def test_many_short_sequences(fmt, d, hkv, lo, hi):
    """Shares of many sequences, cut anywhere in them and between them."""
    say("decode_mx many short fmt=%d d=%d hkv=%d" % (fmt, d, hkv))
    ctx = np.random.default_rng(hi).integers(lo, hi, size=900)
    c = BigCase(fmt, d, hkv, 2, ctx, np.ones(900, np.int64), hi)
    lse = torch.full((900, c.hq), float("nan"), device="cuda")
    out, lse = pa.decode_mx(c.q, c.cache, c.bt, c.ctx, c.max_kv, scale=c.scale, lse=lse)
    again = pa.decode_mx(c.q, c.cache, c.bt, c.ctx, c.max_kv, scale=c.scale)
    torch.cuda.synchronize()
    assert torch.isfinite(lse).all() and torch.equal(out, again)
    c.check(out, lse, list(range(0, 900, 9)) + [897, 898, 899])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d", (64, 128))
@pytest.mark.parametrize("new", ([0, 1, 0, 0, 1, 1, 0], [0, 40, 0, 0, 1, 3, 0], [0, 0, 0, 0, 1, 0, 0]))
def test_sequences_without_new_tokens_and_rows_behind_the_last(fmt, d, new):
    """Appended: the sequences' tokens and nothing else.  Read back: rows behind the last sequence stay as they were."""
    say("append/pack fmt=%d d=%d new=%s and 5 rows behind" % (fmt, d, new))
    c = MxCase(fmt, d, 3, 1, [5, 15, 16, 0, 31, 100, 7], new, 70 + d + fmt)
    behind = torch.full((5, 3, d), 2.0, dtype=torch.bfloat16)
    cache, bt, ctx, cu, _, _, _ = c.device(appended=False)
    pa.kv_append_mx(torch.cat([c.k_new, behind]).cuda(), torch.cat([c.v_new, behind]).cuda(), cache, bt, ctx, cu, c.max_q, c.max_kv)
    rows = torch.full((2, c.total + 5, 3, d), 3.0, dtype=torch.bfloat16, device="cuda")
    pa.kv_pack_mx(cache, bt, ctx, cu, c.total + 5, c.max_q, c.max_kv, out=rows)
    torch.cuda.synchronize()
    assert np.array_equal(cache.cpu().numpy(), c.after)
    want = oracle.mx_pack(c.after, d, fmt, c.bt, c.ctx, c.cu)
    assert np.array_equal(bits(rows[:, :c.total]), want) and bool((rows[:, c.total:] == 3.0).all())
