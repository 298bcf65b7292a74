"""GPU attention over a cache of MX blocks whose attended elements of V are infinite or NaN: in the outputs of their own
channel, of the rows that attend them, and nowhere else.

Such elements come from E4M3's NaN codes, from scales above the ones that keep every element finite, from appended numbers of
1.75 * 2^127 and more, which are read back as infinity, and from appended infinities and NaN, which make all 32
channels of their block NaN."""
import numpy as np
import pytest
import torch

import oracle
import paper_2609_35158_amd as pa
from gpu_helpers import bits, say
from mx_helpers import MxCase, dev
from oracle.mx_cache import _places

pytestmark = pytest.mark.gpu

FORMATS = (pa.MXFP4, pa.MXFP8)
LARGEST = float(torch.finfo(torch.bfloat16).max)


def _codes(c, b, h, pos, channel):
    """(page, byte, shift, mask) of the code of V's element."""
    byte = int(_places(pos % 16, c.d, c.fmt)[1][channel // 2 if c.fmt == 4 else channel])
    shift = 4 * (channel % 2) if c.fmt == 4 else 0
    return int(c.bt[b, pos // 16]), byte, shift, 15 if c.fmt == 4 else 255


def put(c, cache, b, h, pos, channel, code, scale=None):
    """Writes one element's code, and its block's scale with zeros in the other 31 elements."""
    if scale is not None:
        for i in range(channel // 32 * 32, channel // 32 * 32 + 32):
            put(c, cache, b, h, pos, i, 0)
        cache[int(c.bt[b, pos // 16]), h, int(_places(pos % 16, c.d, c.fmt)[3][channel // 32])] = scale
    page, byte, shift, mask = _codes(c, b, h, pos, channel)
    cache[page, h, byte] = (int(cache[page, h, byte]) & ~(mask << shift)) | code << shift


def without(c, cache):
    """The cache with zeros in place of V's infinite and NaN elements, wherever they are."""
    out = cache.copy()
    _, v = oracle.mx_pools(cache, c.d, c.fmt)
    odd = (v & 0x7f80) == 0x7f80                                   # [pages, heads, 16, d]
    for slot in range(16):
        _, vc, _, vs = _places(slot, c.d, c.fmt)
        for ch in range(c.d):
            byte, shift = (vc[ch // 2], 4 * (ch % 2)) if c.fmt == 4 else (vc[ch], 0)
            mask = (15 if c.fmt == 4 else 255) << shift
            out[:, :, byte] = np.where(odd[:, :, slot, ch], out[:, :, byte] & (255 ^ mask), out[:, :, byte])
        for blk in range(c.d // 32):                               # (0 times NaN)
            out[:, :, vs[blk]] = np.where(out[:, :, vs[blk]] == 255, 1, out[:, :, vs[blk]])
    return out


def expected(c, cache):
    """What the outputs are that infinities and NaN reach, 0 elsewhere: of a row's attended elements of its channel."""
    _, v = oracle.mx_pools(cache, c.d, c.fmt)
    v = oracle.bf16_bits_to_f64(v)
    v = np.where(np.isfinite(v), 0.0, v)
    out = np.zeros((c.total, c.hq, c.d))
    for b in range(len(c.ctx)):
        pos = np.arange(c.kv[b])
        rows = v[c.bt[b, pos // 16], :, pos % 16]                  # [kv, heads, d]
        with np.errstate(invalid="ignore"):
            upto = np.cumsum(rows, axis=0)
        for t in range(int(c.new[b])):
            out[c.cu[b] + t] = np.repeat(upto[c.ctx[b] + t], c.G, 0)
    return out


def check(c, cache, out, lse):
    odd = expected(c, cache)
    got = oracle.bf16_bits_to_f64(bits(out))
    where = ~np.isfinite(odd) | ~np.isfinite(got)
    assert np.array_equal(got[where], odd[where], equal_nan=True), [
        (tuple(i), got[tuple(i)], odd[tuple(i)]) for i in np.argwhere(where)
        if not np.array_equal(got[tuple(i)], odd[tuple(i)], equal_nan=True)][:6]
    kept, c.after = c.after, without(c, cache)
    ref, ref_lse, tol, tol_lse = c.oracle()
    c.after = kept
    bad = ~where & ~(np.abs(got - ref) <= tol)
    assert not bad.any(), (np.argwhere(bad)[:4], np.abs(got - ref)[~where].max())
    assert (np.abs(lse.cpu().numpy().astype(np.float64) - ref_lse) <= tol_lse).all()


def decode(c, cache, **kw):
    _, bt, ctx, _, q, _, _ = c.device()
    out, lse = pa.decode_mx(q, dev(cache), bt, ctx, c.max_kv, scale=c.scale, return_lse=True, **kw)
    torch.cuda.synchronize()
    return out, lse


# the code of a large element and the scales under which it is infinite: the least one, and the largest
LARGE = {4: (6, 253, 254), 8: (0x7e, 247, 254)}


def plant(c, rng, per_sequence):
    """A cache with so many infinite and NaN elements of V at random places that every sequence attends to."""
    cache = c.after.copy()
    code, *scales = LARGE[c.fmt]
    for b in range(len(c.ctx)):
        for _ in range(per_sequence):
            pos = int(rng.integers(c.kv[b]))
            h, ch, sign = int(rng.integers(c.hkv)), int(rng.integers(c.d)), int(rng.integers(2))
            if c.fmt == 8 and rng.random() < 0.4:
                put(c, cache, b, h, pos, ch, 0x7f | sign << 7)
            else:
                put(c, cache, b, h, pos, ch, code | sign << (c.fmt - 1), int(scales[rng.integers(2)]))
    return cache


DECODE = ([0], [40], [300, 5, 1000], [63], [5000], [200] * 70, [17, 900, 33, 31])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d", (64, 128))
@pytest.mark.parametrize("n", range(len(DECODE)))
def test_decode(fmt, d, n):
    say("decode_mx with infinite and NaN values fmt=%d d=%d ctx=%s" % (fmt, d, DECODE[n][:5]))
    G, hkv = (1, 2, 4, 8)[n % 4], (2, 1, 3)[n % 3]
    rng = np.random.default_rng(100 + n + d + fmt)
    c = MxCase(fmt, d, hkv, G, DECODE[n], [1] * len(DECODE[n]), 200 + n + d + fmt)
    cache = plant(c, rng, 3)
    check(c, cache, *decode(c, cache))
    # every kind in neighbouring channels of the new token, the largest of its own sequence by a wide margin
    cache = c.after.copy()
    code, s, _ = LARGE[fmt]
    for b in range(len(c.ctx)):
        put(c, cache, b, 0, int(c.ctx[b]), 6, code, s)
        put(c, cache, b, 0, int(c.ctx[b]), 9, code | 1 << (fmt - 1))
        put(c, cache, b, 0, int(c.ctx[b]), 12, code)
        put(c, cache, b, 0, int(c.ctx[b]), 13, code | 1 << (fmt - 1))
        if c.ctx[b]:
            put(c, cache, b, 0, int(c.ctx[b]) - 1, 12, code | 1 << (fmt - 1), s)    # both signs: NaN
    check(c, cache, *decode(c, cache))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("channel", (6, 7, 95))
def test_appended_numbers_that_are_read_back_as_infinity(fmt, channel):
    """The largest bf16, finite, in an even and in an odd channel: its own channel is infinite, as prefill's."""
    say("decode_append_mx of the largest bf16 fmt=%d channel=%d" % (fmt, channel))
    c = MxCase(fmt, 128, 2, 4, [300, 5, 1000, 0], [1] * 4, 300 + fmt)
    c.v_new[:, 1, channel] = torch.tensor([LARGEST, -LARGEST, LARGEST, -LARGEST], dtype=torch.bfloat16)
    cache, bt, ctx, cu, q, _, _ = c.device(appended=False)
    out, lse = pa.decode_append_mx(q, c.k_new.cuda(), c.v_new.cuda(), cache, bt, ctx, c.max_kv, scale=c.scale, return_lse=True)
    torch.cuda.synchronize()
    after = oracle.mx_append(c.cache, fmt, bits(c.k_new), bits(c.v_new), c.bt, c.ctx, c.cu)
    assert np.array_equal(cache.cpu().numpy(), after)
    assert np.isinf(expected(c, after)[:, 4:, channel]).all()
    check(c, after, out, lse)
    turn, _ = pa.prefill_append_mx(q, cache, bt, ctx, cu, 1, c.max_kv, scale=c.scale, return_lse=True)
    torch.cuda.synchronize()
    same = np.isfinite(oracle.bf16_bits_to_f64(bits(turn)))
    got = oracle.bf16_bits_to_f64(bits(out))
    assert np.array_equal(np.isfinite(got), same)
    assert np.array_equal(got[~same], oracle.bf16_bits_to_f64(bits(turn))[~same])


def test_decode_of_several_kv_heads_a_workgroup():
    """Workgroups of 8 kv-heads, whose waves finish by themselves, and of 4, joined in LDS."""
    for fmt, d, hkv in ((4, 128, 8), (8, 64, 8), (4, 64, 4)):
        say("decode_mx with infinite and NaN values fmt=%d d=%d hkv=%d" % (fmt, d, hkv))
        rng = np.random.default_rng(hkv + d)
        ctx = rng.integers(200, 420, size=40)
        c = MxCase(fmt, d, hkv, 1, ctx, [1] * len(ctx), 400 + d + hkv)
        cache = plant(c, rng, 2)
        check(c, cache, *decode(c, cache))


def prefill(c, cache, **kw):
    _, bt, ctx, cu, q, _, _ = c.device()
    out, lse = pa.prefill_append_mx(q, dev(cache), bt, ctx, cu, c.max_q, c.max_kv, scale=c.scale, return_lse=True, **kw)
    torch.cuda.synchronize()
    return out, lse


# single rows, page, stage (64 keys) and tile edges, several tiles, long contexts whose keys are split over workgroups
TURNS = [([0], [17]), ([63, 64, 65, 0], [1, 2, 0, 64]), ([5, 0, 130], [255, 256, 31]), ([1500, 3], [300, 70]), ([0], [520]),
         ([9000], [40]), ([6000, 20], [3, 90])]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d", (64, 128))
@pytest.mark.parametrize("n", range(len(TURNS)))
def test_prefill(fmt, d, n):
    """In the rows from an element's position on, whether its key is masked for rows of the same tile or not."""
    ctx, new = TURNS[n]
    say("prefill_mx with infinite and NaN values fmt=%d d=%d ctx=%s new=%s" % (fmt, d, ctx, new))
    G, hkv = (1, 2, 4, 8)[n % 4], (2, 1, 3)[n % 3]
    rng = np.random.default_rng(500 + n + d + fmt)
    c = MxCase(fmt, d, hkv, G, ctx, new, 600 + n + d + fmt)
    cache = plant(c, rng, 2)
    for b in range(len(ctx)):                                      # and among the new tokens
        code, s, _ = LARGE[fmt]
        for _ in range(3 if new[b] else 0):
            pos, ch = int(ctx[b] + rng.integers(new[b])), int(rng.integers(d))
            put(c, cache, b, int(rng.integers(hkv)), pos, ch, code | int(rng.integers(2)) << (fmt - 1), s)
    check(c, cache, *prefill(c, cache))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("value", (float("nan"), float("inf"), -LARGEST))
def test_a_turns_values_do_not_reach_the_tokens_before_them(fmt, value):
    say("prefill_mx with a new value of %s fmt=%d" % (value, fmt))
    c = MxCase(fmt, 128, 2, 4, [40, 1000, 0], [100, 30, 7], 700 + fmt)
    v_new, at = c.v_new.clone(), {0: 53, 1: 4, 2: 6}               # the token of each sequence
    for b, t in at.items():
        v_new[int(c.cu[b]) + t, 1, 77] = value
    cache, bt, ctx, cu, q, k, _ = c.device(appended=False)
    pa.kv_append_mx(k, v_new.cuda(), cache, bt, ctx, cu, c.max_q, c.max_kv)
    out, lse = pa.prefill_append_mx(q, cache, bt, ctx, cu, c.max_q, c.max_kv, scale=c.scale, return_lse=True)
    torch.cuda.synchronize()
    check(c, cache.cpu().numpy(), out, lse)
    reached = torch.zeros_like(out, dtype=torch.bool)
    for b, t in at.items():
        reached[int(c.cu[b]) + t:int(c.cu[b + 1]), 4:, slice(64, 96) if not np.isfinite(value) else 77] = True
    assert torch.equal(~torch.isfinite(out), reached)


def test_prefill_items_one_after_another():
    """More items than workgroups, some with such elements: none are left over for the next item."""
    say("prefill_mx with infinite and NaN values in some of many items")
    rng = np.random.default_rng(9)
    ctx, new = [0] * 160, [3 + (5 * i) % 20 for i in range(160)]
    c = MxCase(4, 64, 4, 1, ctx, new, 800)
    cache = c.after.copy()
    code, s, _ = LARGE[4]
    for b in range(0, 160, 7):
        put(c, cache, b, int(rng.integers(4)), int(rng.integers(new[b])), int(rng.integers(64)), code, s)
    check(c, cache, *prefill(c, cache))


def put_k(c, cache, b, positions, channel):
    """K of these positions: an element of 2^128 or more, which is read back as infinity, and 31 zeros in its block."""
    code, _, scale = LARGE[c.fmt]
    for pos in positions:
        page = int(c.bt[b, pos // 16])
        codes, _, scales, _ = _places(pos % 16, c.d, c.fmt)
        at = codes.reshape(c.d // 32, -1)[channel // 32]
        cache[page][:, at] = 0
        cache[page][:, scales[channel // 32]] = scale
        byte = int(codes[channel // 2 if c.fmt == 4 else channel])
        cache[page][:, byte] = code << (4 * (channel % 2) if c.fmt == 4 else 0)


def check_k(c, cache, out, lse):
    """Against the oracle, where scores of minus infinity are weights of 0; bounds as MxCase.oracle's, with the largest
    attended |v| for the weighted sums of them, whose weights these keys change."""
    k, v = oracle.mx_pools(cache, c.d, c.fmt)
    with np.errstate(invalid="ignore"):
        ref, ref_lse = oracle.attention(bits(c.q), k, v, c.bt, c.ctx, c.cu, c.scale)
    got = oracle.bf16_bits_to_f64(bits(out))
    assert np.array_equal(np.isnan(got), np.isnan(ref))
    kn = vm = 0.0
    for b in range(len(c.ctx)):
        pos = np.arange(c.kv[b])
        for x, is_v in ((k, False), (v, True)):
            rows = oracle.bf16_bits_to_f64(x[c.bt[b, pos // 16], :, pos % 16])
            rows = np.where(np.isfinite(rows), rows, 0.0)
            if is_v:
                vm = max(vm, float(np.abs(rows).max()))
            else:
                kn = max(kn, float(np.linalg.norm(rows, axis=-1).max()))
    score = c.scale * np.linalg.norm(oracle.bf16_bits_to_f64(bits(c.q)), axis=-1) * kn
    off = c.d * 2.0 ** -24 * score + 2.0 ** -21 * score
    sums = (c.max_kv / 4 + 64) * 2.0 ** -24
    weight = 2.0 ** -16 if c.max_q == 1 else 2.0 ** -8
    tol = 2.0 ** -8 * np.abs(ref) + (2 * off + 2 * sums + weight)[..., None] * vm
    seen = ~np.isnan(ref)
    assert (np.abs(got - ref) <= tol)[seen].all(), float(np.abs(got - ref)[seen].max())
    seen = ~np.isnan(ref_lse)
    tol_lse = off + sums + 2.0 ** -21 * np.abs(ref_lse) + 1e-6
    assert (np.abs(lse.cpu().numpy().astype(np.float64) - ref_lse) <= tol_lse)[seen].all()


def against(c, channel):
    """Heads 0, 2, .. whose scores with such keys are minus infinity, and the others, where they are infinity: NaN."""
    sign = torch.tensor([-1.0, 1.0] * c.hq)[:c.hq]
    c.q[:, :, channel] = (c.q[:, :, channel].float().abs() + 0.25).to(torch.bfloat16) * sign.to(torch.bfloat16)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d,hkv", ((64, 2), (128, 2), (128, 8)))
def test_keys_whose_scores_are_minus_infinity(fmt, d, hkv):
    """They have weight 0, also where a unit, a share or a split of the keys holds no others."""
    say("mx attention with infinite keys fmt=%d d=%d hkv=%d" % (fmt, d, hkv))
    ctx = [64, 16, 200, 1000, 33, 5000]
    c = MxCase(fmt, d, hkv, 2, ctx, [1] * len(ctx), 900 + d + fmt + hkv)
    against(c, 3)
    cache = c.after.copy()
    for b, n in enumerate(ctx):                                    # the new token, alone in its page or not
        put_k(c, cache, b, [n], 3)
    put_k(c, cache, 2, range(64), 3)                               # the first units
    put_k(c, cache, 3, range(900), 3)
    put_k(c, cache, 5, range(200, 4700), 3)                        # whole shares
    check_k(c, cache, *decode(c, cache))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d", (64, 128))
def test_a_turns_keys_whose_scores_are_minus_infinity(fmt, d):
    say("prefill_mx with infinite keys fmt=%d d=%d" % (fmt, d))
    c = MxCase(fmt, d, 2, 2, [100, 0, 6000, 300], [30, 90, 3, 64], 950 + d + fmt)
    against(c, 3)
    cache = c.after.copy()
    put_k(c, cache, 0, [107], 3)                                   # a new token
    put_k(c, cache, 1, range(10, 80), 3)
    put_k(c, cache, 2, range(5900), 3)                             # splits without other keys
    put_k(c, cache, 3, range(64), 3)                               # the first stage
    check_k(c, cache, *prefill(c, cache))


def only_owned(c, cache):
    """The cache with zeros in every slot that no sequence's token owns."""
    out = np.zeros_like(cache)
    for b in range(len(c.ctx)):
        for pos in range(int(c.kv[b])):
            at = np.concatenate(_places(pos % 16, c.d, c.fmt))
            out[c.bt[b, pos // 16]][:, at] = cache[c.bt[b, pos // 16]][:, at]
    return out


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d", (64, 128))
def test_bytes_that_no_token_owns_change_no_result(fmt, d):
    """Bit for bit, of NaN scales and codes beside the last tokens too: such bytes do not even send an item into the form
    that infinite and NaN elements take, which rounds in another order (and is slow)."""
    say("mx attention beside bytes that no token owns fmt=%d d=%d" % (fmt, d))
    rng = np.random.default_rng(30)
    c = MxCase(fmt, d, 3, 4, [100, 0, 3000, 45], [70, 90, 33, 1], 1000 + d + fmt)
    clean = only_owned(c, c.after)
    for trial in range(3):
        cache = np.where(only_owned(c, np.full_like(clean, 255)) > 0, clean,
                         255 if trial == 0 else rng.integers(0, 256, size=clean.shape, dtype=np.uint8)).astype(np.uint8)
        for x, y in zip(prefill(c, cache), prefill(c, clean)):
            assert torch.equal(x, y)
    e = MxCase(fmt, d, 3, 4, [100, 15, 3000, 45], [1] * 4, 1001 + d + fmt)
    clean = only_owned(e, e.after)
    cache = np.where(only_owned(e, np.full_like(clean, 255)) > 0, clean, 255).astype(np.uint8)
    for x, y in zip(decode(e, cache), decode(e, clean)):
        assert torch.equal(x, y)
