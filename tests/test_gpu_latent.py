"""Attention over a paged cache of latent rows on the GPU against the oracle in float64: heads from one to 128, lengths from one
token on, cuts along the keys, causal tiles, values that are not finite, strange lengths, graphs and streams."""
import numpy as np
import pytest
import torch

import oracle
import paper_2609_35158_amd as pa
from gpu_helpers import bits
from latent_helpers import LatentCase, check, from_bits, torch_latent
from rope_helpers import bf16, check_rows, dev, inv_freq, rope_bound

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dc", [512, 256])
@pytest.mark.parametrize("heads", [1, 5, 16, 17, 32, 40, 64, 100, 128])
def test_decode(heads, dc):
    c = LatentCase(heads, dc, [0, 1, 15, 16, 63, 64, 700, 2731], [1] * 8, seed=heads + dc)
    check(c, *c.decode())


@pytest.mark.parametrize("dc", [512, 256])
@pytest.mark.parametrize("ctx", [0, 30, 63, 127, 1000])
def test_decode_one_sequence(ctx, dc):
    for heads in (16, 20):
        c = LatentCase(heads, dc, [ctx], [1], seed=ctx + heads, spread=True)
        check(c, *c.decode())


@pytest.mark.parametrize("dc", [512, 256])
@pytest.mark.parametrize("heads", [1, 3, 16, 20, 64, 128])
def test_prefill(heads, dc):
    c = LatentCase(heads, dc, [0, 37, 0, 300, 64], [70, 5, 0, 33, 1], seed=3 * heads + dc, spare=2)
    q, cache, bt, ctx, cu = c.args()
    out = torch.full((c.total, heads, dc), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((c.total, heads), 7.0, device="cuda")
    pa.latent_prefill_append(q, cache, bt, ctx, cu, c.max_q, c.max_kv, c.scale, out=out, lse=lse)
    check(c, out, lse)
    assert bool((out[-2:] == 7).all()) and bool((lse[-2:] == 7).all())


@pytest.mark.parametrize("new", [[1, 1], [2, 2], [4, 3], [1, 200]])
def test_prefill_few_tokens(new):
    for heads in (4, 16):
        c = LatentCase(heads, 512, [900, 17], new, seed=sum(new) + heads, spread=True)
        check(c, *c.prefill())


def test_prefill_of_single_tokens_is_decode():
    c = LatentCase(16, 512, [5, 1200, 64, 63], [1] * 4, seed=9)
    a, b = c.prefill(), c.decode()
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("batch", [255, 256, 257, 700, 1025])
def test_many_sequences(batch):
    rng = np.random.default_rng(batch)
    c = LatentCase(4, 256, rng.integers(0, 90, size=batch), np.ones(batch, int), seed=batch)
    check(c, *c.decode())
    new = rng.choice([0, 0, 1, 3], size=batch)
    new[batch // 2] = 9
    c = LatentCase(4, 256, rng.integers(0, 90, size=batch), new, seed=batch + 1)
    check(c, *c.prefill())


@pytest.mark.parametrize("heads,dc,ctx,new", [(16, 512, [60000], [1]), (128, 512, [9000, 100], [1, 1]), (16, 512, [9000, 20], [40, 7]),
                                              (64, 256, [12000], [3]), (16, 512, [0, 0], [900, 333])])
def test_long(heads, dc, ctx, new):
    """Contexts that are cut among all workgroups, against 64 bits on the GPU."""
    rng = np.random.default_rng(sum(ctx))
    width = dc + {512: 64, 256: 32}[dc]
    kv = np.add(ctx, new)
    pages = (kv + 15) // 16
    cache = torch.empty((int(pages.sum()) + 2, 16, width), dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    cache.normal_(generator=gen)
    perm = rng.permutation(len(cache))
    bt = np.full((len(kv), int(pages.max())), -1)
    at = 0
    for b, n in enumerate(pages):
        bt[b, :n] = perm[at:at + n]
        at += n
    cu = np.concatenate([[0], np.cumsum(new)])
    q = (torch.randn((int(cu[-1]), heads, width), generator=gen, device="cuda") * 1.15).to(torch.bfloat16)
    scale = 192.0 ** -0.5
    out, lse = pa.latent_prefill_append(q, cache, dev(bt), dev(ctx), dev(cu), max(new), int(kv.max()), scale, return_lse=True)
    for b, n in enumerate(kv):
        rows = cache[dev(bt[b, :pages[b]], np.int64)].flatten(0, 1)[:n]
        sl = slice(int(cu[b]), int(cu[b + 1]))
        ref, ref_lse, size = torch_latent(q[sl], rows, dc, scale)
        off = (out[sl].double() - ref).abs()
        # Weights w_j are rounded to bf16, each off by 2^-8 of itself at most: sum w_j |c_j| 2^-8, `size` times that (a row of few keys has
        # no more to average over); the result's own rounding is 2^-8 of it; sums in 32 bits, as LatentCase.oracle counts them.
        excess = float((off - 2.0 ** -8 * ref.abs() - (2.0 ** -8 + 2.0 ** -10) * size).max())
        assert excess <= 0, (b, excess)
        assert float(off.norm() / ref.norm()) < 2.0 ** -8
        assert float((lse[sl].double() - ref_lse).abs().max()) < 3e-5


@pytest.mark.parametrize("heads", [16, 64])
def test_scores_far_apart(heads):
    """Scores of hundreds, the largest ones late: the maximum moves by more than the weights' range, and rows agree on it."""
    c = LatentCase(heads, 512, [640, 200], [3, 70], seed=77, gain=8.0, spread=True)
    out, lse = c.prefill()
    ref, ref_lse, tol, tol_lse = c.oracle()
    got = oracle.bf16_bits_to_f64(bits(out))
    assert (np.abs(got - ref) <= tol).all() and (np.abs(lse.cpu().numpy() - ref_lse) <= tol_lse).all()


def _odd(c, b, key, channel, value):
    page, slot = int(c.bt[b, key // 16]), key % 16
    c.cache[page, slot, channel] = bits(bf16([value]))[0]


@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("heads", [16, 5])
def test_values_that_are_not_finite(heads, value):
    """A row with such a channel reaches only the tokens that attend to it: those before it are what they are without it."""
    c = LatentCase(heads, 512, [30, 100], [60, 20], seed=heads)
    for b, i in ((0, 33), (1, 11)):
        _odd(c, b, int(c.ctx[b]) + i, 40, value)
    out, lse = c.prefill()
    # The tokens before: what the oracle says, within its bounds (their rounding may differ from a run without the value, as rows of
    # a tile take up a new maximum together).
    ref, ref_lse, tol, tol_lse = c.oracle()
    got, got_lse = oracle.bf16_bits_to_f64(bits(out)), lse.cpu().numpy()
    for b, i in ((0, 33), (1, 11)):
        lo, at, hi = int(c.cu[b]), int(c.cu[b]) + i, int(c.cu[b + 1])
        assert (np.abs(got - ref) <= tol)[lo:at].all() and (np.abs(got_lse - ref_lse) <= tol_lse)[lo:at].all()
        assert not bool(torch.isfinite(out[at:hi, :, 40]).any())


def test_scores_of_minus_infinity():
    """Keys whose scores are minus infinity have weight 0."""
    c = LatentCase(16, 512, [200], [1], seed=4)
    q = bits(c.q).copy()
    q[..., 512] = bits(bf16([2.0]))[0]
    c.q = from_bits(q)
    for key in list(range(0, 70)) + [150]:
        _odd(c, 0, key, 512, float("-inf"))                    # of the rotated part: no value is touched
    out, lse = c.decode()
    ref, ref_lse, _ = oracle.latent_attention(bits(c.q), c.cache, c.bt, c.ctx, c.cu, 512, c.scale)
    assert np.isfinite(ref).all()
    off = np.abs(oracle.bf16_bits_to_f64(bits(out)) - ref)
    assert (off <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -8 * 5).all() and np.abs(lse.cpu().numpy() - ref_lse).max() < 1e-4


def test_lengths_that_cannot_be():
    """A length beyond the host bounds: nothing is written."""
    c = LatentCase(16, 512, [20, 30], [3, 4], seed=6)
    q, cache, bt, ctx, cu = c.args()
    for bad_ctx, bad_cu in (([20, 5000], c.cu), ([-1, 30], c.cu), ([20, 30], [0, 5, 7]), ([20, 30], [0, 3, 9]), ([20, 30], [0, 3, 2])):
        out = torch.full((7, 16, 512), 7.0, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((7, 16), 7.0, device="cuda")
        pa.latent_prefill_append(q, cache, bt, dev(bad_ctx), dev(bad_cu), 4, c.max_kv, c.scale, out=out, lse=lse)
        torch.cuda.synchronize()
        assert bool((out == 7).all()) and bool((lse == 7).all()), (bad_ctx, bad_cu)


def test_debug_mode_reports(monkeypatch):
    c = LatentCase(16, 512, [20, 30], [3, 4], seed=6)
    monkeypatch.setenv("PEARL_DEBUG", "1")
    check(c, *c.prefill())
    c.ctx = c.ctx + np.array([0, 4000])
    with pytest.raises(pa.PearlError, match="host bounds"):
        c.prefill()


def test_pages_that_are_not_there():
    """Page ids outside the cache are clamped: no fault, and other sequences are not touched."""
    c = LatentCase(16, 512, [100, 90], [2, 2], seed=8)
    good = c.prefill()
    c.bt[0, 2], c.bt[0, 3] = -5, 10 ** 6
    out, _ = c.prefill()
    assert torch.equal(out[2:], good[0][2:])


def test_cache_past_4_gib():
    """Byte offsets beyond 32 bits."""
    pages = (5 << 30) // (16 * 576 * 2)
    cache = torch.zeros((pages, 16, 576), dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    rows = torch.randn((200, 576), generator=gen, device="cuda").to(torch.bfloat16)
    bt = np.arange(pages - 13, pages)[::-1].copy()[None]
    freq = dev(inv_freq(64), np.float32)
    rope = pa.Rope(freq, interleaved=True)
    q = torch.randn((200, 16, 576), generator=gen, device="cuda").to(torch.bfloat16)
    q_rope = q[..., 512:].contiguous()
    zero, cu = dev([0]), dev([0, 200])
    pa.latent_append(q_rope, rows, rope, q, cache, dev(bt), zero, cu, 200, 200)
    out, lse = pa.latent_prefill_append(q, cache, dev(bt), zero, cu, 200, 200, 0.07, return_lse=True)
    flat = cache[dev(bt[0], np.int64)].flatten(0, 1)
    assert torch.equal(flat[:200, :512], rows[:, :512]) and not bool(flat[200:].any())
    ref, ref_lse, _ = torch_latent(q, flat[:200], 512, 0.07)
    assert float((out.double() - ref).norm() / ref.norm()) < 2.0 ** -8
    assert float((lse.double() - ref_lse).abs().max()) < 3e-5


@pytest.mark.parametrize("heads,dc,interleaved,norm", [(16, 512, True, True), (128, 512, True, True), (1, 512, False, False),
                                                       (7, 256, True, False), (20, 256, False, True), (15, 512, False, True)])
def test_append(heads, dc, interleaved, norm):
    dr = {512: 64, 256: 32}[dc]
    rng = np.random.default_rng(heads)
    ctx, new = np.array([0, 13, 700, 5]), np.array([17, 1, 0, 40])
    cu = np.concatenate([[0], np.cumsum(new)])
    rows = int(cu[-1]) + 2
    pages = (ctx + new + 15) // 16
    perm = rng.permutation(int(pages.sum()) + 2)
    bt = np.full((4, int(pages.max()) + 1), -1)
    at = 0
    for b, n in enumerate(pages):
        bt[b, :n] = perm[at:at + n]
        at += n
    before = bits(bf16(rng.standard_normal((len(perm), 16, dc + dr))))
    cache = from_bits(before).cuda()
    wide = bf16(rng.standard_normal((rows, dc + dr + 24))).cuda()
    new_rows = wide[:, 16:16 + dc + dr]                        # parts of wider rows and of wider heads
    heads_wide = bf16(rng.standard_normal((rows, heads, dr + 128))).cuda()
    q_rope = heads_wide[..., 128:]
    q0 = bf16(rng.standard_normal((rows, heads, dc + dr))).cuda()
    q = q0.clone()
    w = bf16(1 + 0.25 * rng.standard_normal(dc)) if norm else None
    freq = inv_freq(dr)
    rope = pa.Rope(dev(freq, np.float32), interleaved=interleaved, factor=1.0, k_weight=None if w is None else w.cuda())
    pa.latent_append(q_rope, new_rows, rope, q, cache, dev(bt), dev(ctx), dev(cu), 40, 700)
    pos = oracle.positions(ctx, cu, rows)
    own = pos >= 0
    assert torch.equal(q[..., :dc], q0[..., :dc]) and torch.equal(q[-2:], q0[-2:])
    check_rows(bits(q[..., dc:])[own], bits(q_rope)[own], pos[own], freq, interleaved)
    # the cache's rows, and nothing else
    seq = np.searchsorted(cu, np.arange(rows), side="right") - 1
    got, want = bits(cache), before.copy()
    wrote = np.stack([got[bt[seq[i], pos[i] // 16], pos[i] % 16] for i in np.flatnonzero(own)])
    for n, i in enumerate(np.flatnonzero(own)):
        want[bt[seq[i], pos[i] // 16], pos[i] % 16] = wrote[n]
    assert np.array_equal(got, want)
    src = bits(new_rows)[own]
    ref = oracle.latent_rows(src, pos[own], dc, freq, interleaved, 1.0, None if w is None else bits(w))
    tol = rope_bound(src[:, None, dc:], ref[:, None, dc:], dr, interleaved)[:, 0]
    val = oracle.bf16_bits_to_f64(wrote)
    assert (np.abs(val[:, dc:] - ref[:, dc:]) <= tol).all()
    if norm:                                                   # the sum of squares and the root in 32 bits, a rounding
        assert (np.abs(val[:, :dc] - ref[:, :dc]) <= (2.0 ** -8 + 2.0 ** -19) * np.abs(ref[:, :dc])).all()
    else:
        assert np.array_equal(wrote[:, :dc], src[:, :dc])
    # rows of pages that are not there are skipped, their queries are not
    bt2 = bt.copy()
    bt2[0, 1], bt2[3, 0] = len(perm), -3
    cache2, q2 = from_bits(before).cuda(), q0.clone()
    pa.latent_append(q_rope, new_rows, rope, q2, cache2, dev(bt2), dev(ctx), dev(cu), 40, 700)
    assert torch.equal(q2, q)
    keep = before.copy()
    for n, i in enumerate(np.flatnonzero(own)):
        page = bt2[seq[i], pos[i] // 16]
        if 0 <= page < len(perm):
            keep[page, pos[i] % 16] = wrote[n]
    assert np.array_equal(bits(cache2), keep)


@pytest.mark.parametrize("dc", [512, 256])
def test_append_of_values_that_are_not_finite(dc):
    """In a normalised latent part an infinity makes the other channels 0 and its own NaN, a NaN all of them; the rotated part and other tokens are
    what they are without."""
    dr = {512: 64, 256: 32}[dc]
    rng = np.random.default_rng(dc)
    rows = bf16(rng.standard_normal((4, dc + dr))).cuda()
    q_rope, rope = bf16(rng.standard_normal((4, 3, dr))).cuda(), pa.Rope(dev(inv_freq(dr), np.float32), k_weight=bf16(1 + 0.25 * rng.standard_normal(dc)).cuda())
    got = []
    for odd in (False, True):
        x = rows.clone()
        if odd:
            x[1, 77], x[2, 200] = float("-inf"), float("nan")
        cache, q = pa.latent_cache(1, dc, dr), torch.zeros((4, 3, dc + dr), dtype=torch.bfloat16, device="cuda")
        pa.latent_append(q_rope, x, rope, q, cache, dev([[0]]), dev([7]), dev([0, 4]), 4, 11)
        got.append((cache[0], q))
    want = got[0][0].clone()
    want[8, :dc], want[9, :dc] = 0, float("nan")
    want[8, 77] = float("nan")
    same = torch.eq(got[1][0], want) | (torch.isnan(got[1][0]) & torch.isnan(want))
    assert bool(same.all()) and torch.equal(got[0][1], got[1][1])


def test_turns_and_steps_equal_one_prompt():
    """A prompt in one call, or in turns and single tokens (append, then attention), gives the same cache and the same outputs."""
    rng = np.random.default_rng(2)
    n, heads, dc, dr = 90, 16, 512, 64
    rows = bf16(rng.standard_normal((n, dc + dr))).cuda()
    q_rope = bf16(rng.standard_normal((n, heads, dr))).cuda()
    q_c = bf16(1.2 * rng.standard_normal((n, heads, dc + dr))).cuda()
    rope = pa.Rope(dev(inv_freq(dr), np.float32), interleaved=True, k_weight=torch.ones(dc, dtype=torch.bfloat16, device="cuda"))
    bt = dev(rng.permutation(8)[None, :6])
    scale = 192.0 ** -0.5

    def run(cuts):
        cache, outs, qs = pa.latent_cache(8, dc, dr), [], []
        for lo, hi in zip(cuts[:-1], cuts[1:]):
            q = q_c[lo:hi].clone()
            at, cu = dev([lo]), dev([0, hi - lo])
            pa.latent_append(q_rope[lo:hi], rows[lo:hi], rope, q, cache, bt, at, cu, hi - lo, hi)
            if hi - lo == 1:
                outs.append(pa.latent_decode(q, cache, bt, at, hi, scale))
            else:
                outs.append(pa.latent_prefill_append(q, cache, bt, at, cu, hi - lo, hi, scale))
            qs.append(q)
        return cache, torch.cat(outs), torch.cat(qs)

    one, turns = run([0, n]), run([0, 1, 2, 40, 41, 64, 65, 89, n])
    assert torch.equal(one[0], turns[0]) and torch.equal(one[2], turns[2])
    d = (one[1].float() - turns[1].float()).abs()
    assert bool((d <= 2.0 ** -7 * one[1].float().abs() + 2.0 ** -7).all())
    ref, _, _ = torch_latent(one[2], one[0][bt[0].long()].flatten(0, 1)[:n], dc, scale)
    assert float((turns[1].double() - ref).norm() / ref.norm()) < 2.0 ** -8


def test_graph_streams_and_shared_workspace():
    """A captured step replayed, with eager calls of other sizes in between on the same workspace and on another stream."""
    c = LatentCase(16, 512, [1500, 3, 0], [1, 1, 1], seed=31)
    d = LatentCase(16, 512, [400, 90], [30, 2], seed=32)
    q, cache, bt, ctx, _ = c.args()
    dq, dcache, dbt, dctx, dcu = d.args()
    from paper_2609_35158_amd import binding as bd
    need = max(pa.workspace_bytes_latent(16, cache, bd.make_desc(bt, ctx, None, 3, 1, 1520)),
               pa.workspace_bytes_latent(16, dcache, bd.make_desc(dbt, dctx, dcu, d.total, d.max_q, d.max_kv)))
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    out_g, lse_g = torch.empty((3, 16, 512), dtype=torch.bfloat16, device="cuda"), torch.empty((3, 16), device="cuda")

    def step(out, lse, work):
        pa.latent_decode(q, cache, bt, ctx, 1520, c.scale, out=out, lse=lse, workspace=work)

    step(out_g, lse_g, ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(out_g, lse_g, ws)
    side = torch.cuda.Stream()
    for r in range(3):
        q.normal_()
        out_g.zero_()
        g.replay()
        check(d, *pa.latent_prefill_append(dq, dcache, dbt, dctx, dcu, d.max_q, d.max_kv, d.scale, return_lse=True, workspace=ws))
        out_e, lse_e = torch.empty_like(out_g), torch.empty_like(lse_g)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            step(out_e, lse_e, torch.empty_like(ws))
        torch.cuda.synchronize()
        assert torch.equal(out_g, out_e) and torch.equal(lse_g, lse_e), r


def test_two_calls_at_once():
    cases = [LatentCase(16, 512, [3000, 50], [1, 1], seed=51), LatentCase(128, 512, [700], [1], seed=52)]
    args = [c.args() for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(4):
        for i, (c, a, s) in enumerate(zip(cases, args, streams)):
            with torch.cuda.stream(s):
                got[i].append(pa.latent_decode(a[0], a[1], a[2], a[3], c.max_kv, c.scale, return_lse=True))
    torch.cuda.synchronize()
    for c, outs in zip(cases, got):
        check(c, *outs[0])
        assert all(torch.equal(outs[0][0], o[0]) and torch.equal(outs[0][1], o[1]) for o in outs)


def test_refusals_of_the_binding():
    c = LatentCase(16, 512, [20], [4], seed=1)
    q, cache, bt, ctx, cu = c.args()
    ok = dict(q=q, cache=cache, block_table=bt, ctx_lens=ctx, cu_q_lens=cu, max_q_len=4, max_kv_len=24, scale=0.1)

    def refuses(error, text, fn=pa.latent_prefill_append, base=ok, **change):
        with pytest.raises(error, match=text):
            fn(**{**base, **change})

    refuses(TypeError, "bfloat16", q=q.float())
    refuses(ValueError, "channels", q=q[..., :288].contiguous())
    refuses(ValueError, "cache must be", cache=cache[..., :64].contiguous())
    refuses(ValueError, "contiguous", q=q.transpose(0, 1))
    refuses(ValueError, "out must have shape", out=torch.empty_like(q))
    refuses(ValueError, "lse must be", lse=torch.empty((4, 8), device="cuda"))
    refuses(ValueError, "GPU", cache=cache.cpu())
    refuses(pa.PearlError, "scale", scale=0.0)
    refuses(pa.PearlError, "workspace_bytes", workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    refuses(pa.PearlError, "max_q_len", max_q_len=5)
    refuses(pa.PearlError, "num_q_heads", q=torch.empty((4, 129, 576), dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(pa.PearlError, match="total_q"):
        pa.latent_decode(q, cache, bt, ctx, 24, 0.1)
    with pytest.raises(ValueError):
        pa.latent_cache(4, 512, 32)
    rope = pa.Rope(dev(inv_freq(64), np.float32), interleaved=True)
    app = dict(q_rope=q[..., 512:], rows_new=torch.zeros((4, 576), dtype=torch.bfloat16, device="cuda"), rope=rope, q=q.clone(), cache=cache,
               block_table=bt, ctx_lens=ctx, cu_q_lens=cu, max_q_len=4, max_kv_len=24)
    refuses(ValueError, "evenly spaced", pa.latent_append, app, q_rope=torch.empty((4, 20, 64), dtype=torch.bfloat16, device="cuda")[:, :16])
    refuses(ValueError, "rows_new", pa.latent_append, app, rows_new=torch.zeros((4, 512), dtype=torch.bfloat16, device="cuda"))
    refuses(pa.PearlError, "rotary_dim", pa.latent_append, app, rope=pa.Rope(dev(inv_freq(32), np.float32)))
    refuses(ValueError, "k_weight", pa.latent_append, app, rope=pa.Rope(dev(inv_freq(64), np.float32), k_weight=torch.ones(64, dtype=torch.bfloat16, device="cuda")))
