"""Rotary position embedding on the GPU (rope_rows, kv_append_rope) against the oracle in float64: pairings, partial
rotations, norms, far positions, strides, batches with empty sequences and rows behind the last one, bad pages, graphs."""
import numpy as np
import pytest
import torch

import oracle
import paper_2609_35158_amd as pa
from gpu_helpers import bits
from rope_helpers import RopeCase, bf16, check_rows, dev, inv_freq

pytestmark = pytest.mark.gpu


def run_rows(c, **kw):
    bt, ctx, cu = c.args()
    return pa.rope_rows(c.q, c.k, c.rope(), ctx, cu, c.max_q, **kw)


@pytest.mark.parametrize("hq,hkv,d,rotary", [(32, 8, 128, 128), (8, 1, 128, 64), (3, 3, 64, 64), (16, 8, 64, 32),
                                             (1, 1, 64, 16), (5, 5, 128, 16), (14, 7, 128, 112), (8, 4, 64, 48)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_rows_and_append(hq, hkv, d, rotary, interleaved, norm):
    c = RopeCase(hq, hkv, d, rotary, [0, 13, 700, 5, 31], [17, 1, 40, 0, 2], seed=rotary + hq, interleaved=interleaved, norm=norm,
                 factor=1.25 if norm else 1.0, spare=3)
    q, k = run_rows(c, q_out=torch.full_like(c.q.contiguous(), 7.0), k_out=torch.full_like(c.k.contiguous(), 7.0))
    c.check(0, q)
    c.check(1, k)
    assert bool((q[-3:] == 7).all()) and bool((k[-3:] == 7).all())       # rows of no sequence
    if not norm and rotary < d:                                          # channels that stay are copied
        assert torch.equal(q[:-3, :, rotary:], c.q[:-3, :, rotary:]) and torch.equal(k[:-3, :, rotary:], c.k[:-3, :, rotary:])
    # the append: the same rows, in their slots; nothing else changes
    bt, ctx, cu = c.args()
    before = [bits(p) for p in c.pools]
    q2 = pa.kv_append_rope(c.q, c.k, c.v, c.rope(), *c.pools, bt, ctx, cu, c.max_q, c.max_kv, q_out=torch.full_like(q, 7.0))
    assert torch.equal(q2, q)
    n = c.rows - 3
    ref = oracle.kv_append(before[0], before[1], bits(k)[:n], bits(c.v)[:n], c.bt, c.ctx, c.cu)
    assert np.array_equal(bits(c.pools[0]), ref[0]) and np.array_equal(bits(c.pools[1]), ref[1])


@pytest.mark.parametrize("interleaved", [False, True])
def test_far_positions(interleaved):
    """Positions up to 2^25 and beyond: the angle keeps its fraction of a turn."""
    ctx = [(1 << 25) - 20, (1 << 24) + 1, 123456789, (1 << 31) - 40]
    new = [20, 3, 2, 30]
    c = RopeCase(4, 2, 128, 128, [0] * 4, new, seed=3, interleaved=interleaved)
    pos = oracle.positions(np.array(ctx), c.cu, c.rows)
    q, k = pa.rope_rows(c.q, c.k, c.rope(), dev(ctx), dev(c.cu), 30)
    for got, src in ((q, c.q), (k, c.k)):
        check_rows(bits(got), bits(src), pos, c.freq, interleaved)


def test_one_token_a_sequence_and_many():
    for batch in (1, 2, 63, 64, 65, 700, 4097):
        rng = np.random.default_rng(batch)
        ctx = rng.integers(0, 5000, size=batch)
        c = RopeCase(8, 2, 128, 128, ctx, np.ones(batch, int), seed=batch, norm=batch % 2 == 0)
        bt, ctx_d, cu = c.args()
        q, k = pa.rope_rows(c.q, c.k, c.rope(), ctx_d, None, 1)
        c.check(0, q)
        c.check(1, k)
        q1, k1 = pa.rope_rows(c.q, c.k, c.rope(), ctx_d, cu, 1)          # the same tokens by cu_q_lens
        assert torch.equal(q, q1) and torch.equal(k, k1), batch


def test_sequences_are_found():
    """Token counts of many sizes, zeros among them, in batches around the ballots' widths."""
    rng = np.random.default_rng(8)
    for batch in (1, 64, 65, 129, 1000, 4200):
        new = rng.choice([0, 0, 1, 2, 5, 33], size=batch)
        new[rng.integers(batch)] = 3
        c = RopeCase(2, 1, 64, 64, rng.integers(0, 300, size=batch), new, seed=batch, spare=2)
        q, k = run_rows(c)
        c.check(0, q)
        c.check(1, k)


def test_in_place_and_contiguous():
    c = RopeCase(8, 2, 128, 64, [40, 0], [9, 30], seed=5, norm=True)
    want = run_rows(c)
    q, k = c.q.contiguous(), c.k.contiguous()
    got = pa.rope_rows(q, k, c.rope(), dev(c.ctx), dev(c.cu), c.max_q, q_out=q, k_out=k)
    assert got[0].data_ptr() == q.data_ptr() and torch.equal(q, want[0]) and torch.equal(k, want[1])


@pytest.mark.parametrize("tokens", [3000, 20000])
def test_many_tokens(tokens):
    """Enough tokens that a wave takes several groups of rows, and all of them."""
    c = RopeCase(32, 8, 64, 64, [100, 0, 7], [tokens // 2, tokens // 2 - 11, 11], seed=tokens, norm=True)
    q, k = run_rows(c)
    sample = np.zeros(c.rows, bool)
    sample[np.random.default_rng(1).integers(0, c.rows, 300)] = True
    sample[[0, -1, tokens // 2 - 1, tokens // 2]] = True
    c.check(0, q, sample)
    c.check(1, k, sample)
    bt, ctx, cu = c.args()
    before = [bits(p) for p in c.pools]
    q2 = pa.kv_append_rope(c.q, c.k, c.v, c.rope(), *c.pools, bt, ctx, cu, c.max_q, c.max_kv)
    ref = oracle.kv_append(before[0], before[1], bits(k), bits(c.v), c.bt, c.ctx, c.cu)
    assert torch.equal(q2, q) and np.array_equal(bits(c.pools[0]), ref[0]) and np.array_equal(bits(c.pools[1]), ref[1])


def test_pages_that_are_not_there():
    """Page ids outside the pool and logical pages beyond the table: the rows are skipped, their queries are not."""
    c = RopeCase(4, 2, 64, 64, [0, 0], [40, 20], seed=12, bt_pad=0)
    bt = c.bt.copy()
    bt[0, 1], bt[1, 0] = c.num_pages, -1
    before = [bits(p) for p in c.pools]
    q, k = run_rows(c)
    table = dev(bt)[:, :2].contiguous()                                   # sequence 0's third page is beyond the table
    q2 = pa.kv_append_rope(c.q, c.k, c.v, c.rope(), *c.pools, table, dev(c.ctx), dev(c.cu), 20, 32)
    assert torch.equal(q2, q)
    for pool, was, rows in zip(c.pools, before, (bits(k), bits(c.v))):
        want = was.copy()
        want[bt[0, 0], :, :, :] = rows[0:16].transpose(1, 0, 2)
        want[bt[1, 1], :, 0:4, :] = rows[56:60].transpose(1, 0, 2)
        assert np.array_equal(bits(pool), want)


def test_lengths_that_cannot_be():
    c = RopeCase(4, 2, 64, 64, [3, 0, 9], [4, 5, 6], seed=13)
    ctx = c.ctx.copy()
    ctx[1] = -1
    before = [p.clone() for p in c.pools]
    q = pa.kv_append_rope(c.q, c.k, c.v, c.rope(), *c.pools, dev(c.bt), dev(ctx), dev(c.cu), c.max_q, c.max_kv,
                          q_out=torch.full_like(c.q.contiguous(), 7.0))
    assert bool((q[4:9] == 7).all())
    c.check(0, q, np.array([True] * 4 + [False] * 5 + [True] * 6))
    page = int(c.bt[1, 0])
    assert torch.equal(c.pools[0][page], before[0][page]) and torch.equal(c.pools[1][page], before[1][page])


def test_values_that_are_not_finite():
    """An infinity stays in its pair; one in a normalised head makes its own channels NaN and the others 0 (x / inf)."""
    c = RopeCase(2, 2, 128, 64, [5], [3], seed=14)
    x = c.fused.clone()
    x[1, 0, 100], x[1, 1, 3] = float("inf"), float("nan")                 # unrotated, and rotated with channel 35
    q, _ = pa.rope_rows(x[:, :2], c.k, c.rope(), dev(c.ctx), dev(c.cu), 3)
    odd = ~torch.isfinite(q)
    assert odd.sum() == 3 and bool(odd[1, 0, 100]) and bool(odd[1, 1, 3]) and bool(odd[1, 1, 35])
    assert float(q[1, 0, 100]) == float("inf")


@pytest.mark.parametrize("interleaved", [False, True])
def test_values_that_are_not_finite_in_a_normalised_head(interleaved):
    """An infinity makes the mean square infinite: the head's other channels are 0, its own NaN, and the one it is paired with if it is rotated; a NaN
    makes the whole head NaN.  Other heads and tokens are what they are without."""
    c = RopeCase(4, 2, 128, 64, [5], [3], seed=15, interleaved=interleaved, norm=True)
    want = run_rows(c)
    x = c.fused.clone()
    x[1, 0, 100], x[1, 1, 3], x[1, 2, 9], x[2, 4, 40] = float("inf"), float("-inf"), float("nan"), float("inf")
    q, k = pa.rope_rows(x[:, :4], x[:, 4:6], c.rope(), dev(c.ctx), dev(c.cu), 3)
    other = (lambda n: n ^ 1) if interleaved else (lambda n: n + 32 if n < 32 else n - 32)
    for got, ref, odd in ((q, want[0], {(1, 0): [100], (1, 1): [3, other(3)], (1, 2): list(range(128))}), (k, want[1], {(2, 0): [40, other(40)]})):
        for t in range(3):
            for h in range(got.shape[1]):
                if (t, h) not in odd:
                    assert torch.equal(got[t, h], ref[t, h])
                    continue
                nan = torch.zeros(128, dtype=torch.bool, device="cuda")
                nan[odd[t, h]] = True
                assert torch.equal(torch.isnan(got[t, h]), nan) and bool((got[t, h][~nan] == 0).all()), (t, h)


def test_step_by_step_equals_prompt():
    """A prompt in one call, in turns and token by token gives the same pools, bit for bit, and decode_append after
    rope_rows the same as kv_append_rope and decode."""
    c = RopeCase(8, 2, 128, 128, [0, 0], [37, 50], seed=21, norm=True)
    bt, ctx, cu = c.args()
    rope = c.rope()
    whole = [p.clone() for p in c.pools]
    q = pa.kv_append_rope(c.q, c.k, c.v, rope, *whole, bt, ctx, cu, c.max_q, c.max_kv)
    single = [p.clone() for p in c.pools]
    for t in range(50):
        rows = dev([min(t, 36), 37 + t], np.int64)
        n = 2 if t < 37 else 1
        rows = rows[2 - n:]
        at = dev([t] * n)
        args = [x[rows] for x in (c.q, c.k, c.v)]
        table = bt[2 - n:].contiguous()
        if t % 2:
            q1 = pa.kv_append_rope(*args, rope, *single, table, at, None, 1, t + 1)
            o1 = pa.decode(q1, *single, table, at, t + 1)
        else:
            q1, k1 = pa.rope_rows(args[0], args[1], rope, at, None, 1)
            o1 = pa.decode_append(q1, k1, args[2].contiguous(), *single, table, at, t + 1)
        assert torch.equal(q1, q[rows])
        assert bool(torch.isfinite(o1).all())
    assert torch.equal(whole[0], single[0]) and torch.equal(whole[1], single[1])
    out = pa.prefill_append(q, *whole, bt, ctx, cu, c.max_q, c.max_kv)
    ref, _ = oracle.attention(bits(q), bits(whole[0]), bits(whole[1]), c.bt, c.ctx, c.cu, 1.0 / np.sqrt(128))
    st = oracle.compare(bits(out), ref)
    assert st["max_abs"] <= 1e-2 and st["mean_abs"] <= 1e-3
    o_ref = oracle.bf16_bits_to_f64(bits(out))[-1]
    assert np.abs(oracle.bf16_bits_to_f64(bits(o1))[-1] - o_ref).max() <= 2e-2


def test_graph_and_streams():
    c = RopeCase(8, 2, 128, 128, [100, 3, 0], [1, 1, 1], seed=31, norm=True)
    bt, ctx, _ = c.args()
    rope = c.rope()
    q, k, v = c.q.contiguous(), c.k.contiguous(), c.v.contiguous()
    out_g, pools_g = torch.empty_like(q), [p.clone() for p in c.pools]

    def step(out, pools):
        pa.kv_append_rope(q, k, v, rope, *pools, bt, ctx, None, 1, c.max_kv, q_out=out)

    step(out_g, pools_g)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(out_g, pools_g)
    side = torch.cuda.Stream()
    for r in range(3):
        q.normal_(), k.normal_(), v.normal_()
        ctx.add_(1 if r else 0)
        g.replay()
        torch.cuda.synchronize()
        out_e, pools_e = torch.empty_like(q), [p.clone() for p in pools_g]
        with torch.cuda.stream(side):
            step(out_e, pools_e)
        torch.cuda.synchronize()
        assert torch.equal(out_g, out_e) and all(torch.equal(a, b) for a, b in zip(pools_g, pools_e)), r


def test_refusals_of_the_binding():
    c = RopeCase(4, 2, 64, 64, [0], [8], seed=41)
    bt, ctx, cu = c.args()
    rope = c.rope()
    ok = dict(q=c.q, k_new=c.k, rope=rope, ctx_lens=ctx, cu_q_lens=cu, max_q_len=8)

    def refuses(error, text, fn=pa.rope_rows, base=ok, **change):
        with pytest.raises(error, match=text):
            fn(**{**base, **change})

    refuses(TypeError, "bfloat16", q=c.q.float())
    refuses(ValueError, "GPU", q=c.q.cpu())
    refuses(ValueError, "must be contiguous", q=c.q.transpose(0, 1).contiguous().transpose(0, 1))
    refuses(ValueError, "k_new must be", k_new=c.k[:4])
    refuses(ValueError, "q_out must have shape", q_out=torch.empty((8, 4, 128), dtype=torch.bfloat16, device="cuda"))
    refuses(ValueError, "q_out must be contiguous", q_out=c.q)
    refuses(TypeError, "ctx_lens", ctx_lens=ctx.long())
    refuses(ValueError, "batch\\+1", cu_q_lens=cu[:1])
    refuses(pa.PearlError, "rotary_dim", rope=pa.Rope(dev(inv_freq(128), np.float32)))
    refuses(pa.PearlError, "max_q_len", max_q_len=9)
    with pytest.raises(ValueError, match="channels"):
        pa.rope_rows(c.q, c.k, pa.Rope(dev(inv_freq(64), np.float32), q_weight=torch.ones(128, dtype=torch.bfloat16, device="cuda")), ctx, cu, 8)
    app = dict(q=c.q, k_new=c.k, v_new=c.v, rope=rope, k_pool=c.pools[0], v_pool=c.pools[1], block_table=bt, ctx_lens=ctx,
               cu_q_lens=cu, max_q_len=8, max_kv_len=8)
    refuses(ValueError, "v_new must be", pa.kv_append_rope, app, v_new=c.v[:, :1])
    refuses(ValueError, "one shape", pa.kv_append_rope, app, v_pool=c.pools[1][:-1])
    refuses(pa.PearlError, "bt_stride", pa.kv_append_rope, app, max_kv_len=1 << 20)
