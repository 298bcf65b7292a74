"""GPU prefill-append over a cache of MX blocks against the float64 oracle on the values the cache stands for, and a
turn as it is served: append, prefill, decode steps, hand-over."""
import numpy as np
import pytest
import torch

import oracle
import paper_2609_35158_amd as pa
from gpu_helpers import bits, say
from mx_helpers import MxCase, check, dev

pytestmark = pytest.mark.gpu

FORMATS = (pa.MXFP4, pa.MXFP8)


def run(c, **kw):
    cache, bt, ctx, cu, q, _, _ = c.device()
    kw = dict(dict(scale=c.scale, return_lse=True), **kw)
    out, lse = pa.prefill_append_mx(q, cache, bt, ctx, cu, c.max_q, c.max_kv, **kw)
    torch.cuda.synchronize()
    return out, lse


# contexts and new tokens: single rows, page and stage (64 keys) edges, tile edges (256 rows / G), sequences without
# new tokens, keys split over workgroups
CASES = [([0], [1]), ([0], [17]), ([63, 64, 65, 0], [1, 2, 0, 64]), ([5, 0, 130], [255, 256, 31]),
         ([1500, 3], [300, 70]), ([0, 0], [520, 190])]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d", (64, 128))
@pytest.mark.parametrize("n", range(len(CASES)))
def test_lengths(fmt, d, n):
    ctx, new = CASES[n]
    G, hkv = (1, 2, 4, 8)[n % 4], (2, 1, 3)[n % 3]
    say("prefill_mx fmt=%d d=%d G=%d hkv=%d ctx=%s new=%s" % (fmt, d, G, hkv, ctx, new))
    c = MxCase(fmt, d, hkv, G, ctx, new, 40 + n + d + fmt)
    out, lse = run(c)
    check(c, out, lse)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d", (64, 128))
@pytest.mark.parametrize("G", (1, 2, 4, 8))
def test_groups(fmt, d, G):
    say("prefill_mx fmt=%d d=%d G=%d" % (fmt, d, G))
    c = MxCase(fmt, d, 2, G, [37, 210, 0], [90, 3, 41], 90 + G + d + fmt)
    out, lse = run(c)
    check(c, out, lse)


@pytest.mark.parametrize("fmt", FORMATS)
def test_nan_blocks_and_rows_behind_the_last_sequence(fmt):
    say("prefill_mx NaN fmt=%d" % fmt)
    c = MxCase(fmt, 128, 2, 2, [40, 20], [30, 25], 61)
    cache, bt, ctx, cu, q, k_new, v_new = c.device(appended=False)
    k_new[10, 1, 3] = float("inf")                                 # position 50 of sequence 0, kv-head 1
    pa.kv_append_mx(k_new, v_new, cache, bt, ctx, cu, c.max_q, c.max_kv)
    out = torch.full((60, 4, 128), 3.0, dtype=torch.bfloat16, device="cuda")     # 5 rows more than the batch has
    lse = torch.full((60, 4), 5.0, device="cuda")
    q60 = torch.cat([q, q[:5]])
    pa.prefill_append_mx(q60, cache, bt, ctx, cu, c.max_q, c.max_kv, scale=c.scale, out=out, lse=lse)
    torch.cuda.synchronize()
    assert (out[55:] == 3.0).all() and (lse[55:] == 5.0).all()
    nan = torch.isnan(out)
    want = torch.zeros_like(nan)
    want[10:30, 2:] = True
    assert torch.equal(nan, want)


def test_a_captured_turn_is_replayed():
    say("a turn in a graph")
    c = MxCase(4, 128, 2, 4, [300, 10], [100, 37], 71)
    cache, bt, ctx, cu, q, k_new, v_new = c.device(appended=False)
    want, want_lse = run(c)
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], device="cuda")
    desc = pa.binding.make_desc(bt, ctx, cu, c.total, c.max_q, c.max_kv)
    ws = torch.full((pa.workspace_bytes_mx(c.hq, cache, desc),), 255, dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pa.kv_append_mx(k_new, v_new, cache, bt, ctx, cu, c.max_q, c.max_kv)
        pa.prefill_append_mx(q, cache, bt, ctx, cu, c.max_q, c.max_kv, scale=c.scale, out=out, lse=lse, workspace=ws)
    for _ in range(3):
        out.zero_()
        cache.copy_(dev(c.cache))
        ws.fill_(93)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
        assert np.array_equal(cache.cpu().numpy(), c.after)
    check(c, want, want_lse)


@pytest.mark.parametrize("fmt", FORMATS)
def test_a_turn_and_decode_steps_as_they_are_served(fmt):
    """Prompts appended and prefilled, three decode steps, the contexts handed to another cache, one more step."""
    say("a served turn fmt=%d" % fmt)
    rng = np.random.default_rng(fmt)
    hkv, G, d, n = 2, 4, 64, np.array([37, 90, 5])
    pages = (n + 8 + 15) // 16
    bt = np.zeros((3, int(pages.max())), np.int32)
    perm = rng.permutation(int(pages.sum()))
    for b in range(3):
        bt[b, :pages[b]] = perm[pages[:b].sum():pages[:b + 1].sum()]
    cache = pa.mx_cache(int(pages.sum()), hkv, d, fmt)
    model = cache.cpu().numpy()
    scale = float(np.float32(d ** -0.5))

    def bf(*s):
        return torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to(torch.bfloat16)

    def attended(q, out, ctx, cu):
        k, v = oracle.mx_pools(model, d, fmt)
        ref, _ = oracle.attention(bits(q), k, v, bt, ctx, cu, scale)
        st = oracle.compare(bits(out), ref)
        assert st["max_abs"] <= 1e-2 * max(1.0, np.abs(ref).max()) and st["mean_abs"] <= 1e-3 * max(1.0, np.abs(ref).max()), st

    ctx, cu = np.zeros(3, np.int32), np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    k, v, q = bf(int(n.sum()), hkv, d), bf(int(n.sum()), hkv, d), bf(int(n.sum()), hkv * G, d)
    btd, ctxd, cud = dev(bt), dev(ctx), dev(cu)
    pa.kv_append_mx(k.cuda(), v.cuda(), cache, btd, ctxd, cud, 90, 90)
    out = pa.prefill_append_mx(q.cuda(), cache, btd, ctxd, cud, 90, 90, scale=scale)
    model = oracle.mx_append(model, fmt, bits(k), bits(v), bt, ctx, cu)
    attended(q, out, ctx, cu)
    ctx = n.astype(np.int32)
    for step in range(4):
        if step == 3:                                              # the decode worker's own cache and pages
            lens = np.concatenate([[0], np.cumsum(ctx)]).astype(np.int32)
            zero = dev(np.zeros(3, np.int32))
            rows = pa.kv_pack_mx(cache, btd, zero, dev(lens), int(lens[-1]), int(ctx.max()), int(ctx.max()))
            bt = ((bt + 1) % len(perm)).astype(np.int32)
            btd = dev(bt)
            cache = pa.mx_cache(int(pages.sum()), hkv, d, fmt)
            pa.kv_append_mx(rows[0], rows[1], cache, btd, zero, dev(lens), int(ctx.max()), int(ctx.max()))
            torch.cuda.synchronize()
            model = cache.cpu().numpy()
        k, v, q = bf(3, hkv, d), bf(3, hkv, d), bf(3, hkv * G, d)
        out = pa.decode_append_mx(q.cuda(), k.cuda(), v.cuda(), cache, btd, dev(ctx), 98, scale=scale)
        model = oracle.mx_append(model, fmt, bits(k), bits(v), bt, ctx, None)
        torch.cuda.synchronize()
        assert np.array_equal(cache.cpu().numpy(), model)
        attended(q, out, ctx, None)
        ctx = ctx + 1
