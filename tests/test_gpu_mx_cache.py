"""GPU append into and read-back out of a cache of MX blocks, byte for byte against the oracle."""
import numpy as np
import pytest
import torch

import oracle
import paper_2609_35158_amd as pa
from gpu_helpers import bits, say

pytestmark = pytest.mark.gpu

FORMATS = (pa.MXFP4, pa.MXFP8)


def rows_bf16(rng, *shape):
    """Rows whose blocks of 32 channels span many magnitudes, with ties, zeros, NaN and infinities among them."""
    x = rng.standard_normal(shape) * np.exp2(rng.integers(-135, 126, size=shape[:-1] + (1,)))
    ties = rng.integers(-28, 29, size=shape) / 4.0
    x = np.where(rng.random(shape[:-1] + (1,)) < 0.3, ties, x)
    x = np.where(rng.random(shape[:-1] + (1,)) < 0.4, rng.standard_normal(shape), x)
    x[rng.random(shape) < 2e-4] = np.nan
    x[rng.random(shape) < 1e-4] = -np.inf
    x[rng.random(shape) < 0.01] = -0.0
    return torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16)


def tables(rng, kv, num_pages, extra_cols=1):
    pages = (kv + 15) // 16
    perm = rng.permutation(num_pages).astype(np.int32)
    bt = np.full((len(kv), int(pages.max()) + extra_cols), -1, np.int32)     # entries past the end: no page
    at = 0
    for b, n in enumerate(pages):
        bt[b, :n] = perm[at:at + n]
        at += n
    return bt


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def case(fmt, d, hkv, ctx, new, seed):
    rng = np.random.default_rng(seed)
    ctx, new = np.asarray(ctx), np.asarray(new)
    kv = np.maximum(ctx + new, 1)
    num_pages = int(((kv + 15) // 16).sum()) + 3
    bt = tables(rng, kv, num_pages)
    cache = rng.integers(0, 256, size=(num_pages, hkv, oracle.mx_block_bytes(d, fmt)), dtype=np.uint8)
    total = int(new.sum())
    k, v = rows_bf16(rng, total, hkv, d), rows_bf16(rng, total, hkv, d)
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    return cache, k, v, bt, ctx.astype(np.int32), cu


def assert_rows(got, want):
    """Equal bits, any NaN equal to any NaN."""
    nan = (want & 0x7fff) > 0x7f80
    assert np.array_equal((got & 0x7fff) > 0x7f80, nan)
    assert np.array_equal(got[~nan], want[~nan])


CTX_NEW = [([0], [1]), ([37], [1]), ([0, 15, 16, 31], [17, 1, 16, 2]), ([100, 3, 0, 64], [0, 45, 33, 7]),
           ([5, 200, 77], [300, 1, 40])]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d", (64, 128))
@pytest.mark.parametrize("hkv", (1, 3))
@pytest.mark.parametrize("n", range(len(CTX_NEW)))
def test_append_and_pack(fmt, d, hkv, n):
    ctx, new = CTX_NEW[n]
    say("append/pack fmt=%d d=%d hkv=%d ctx=%s new=%s" % (fmt, d, hkv, ctx, new))
    cache, k, v, bt, ctx, cu = case(fmt, d, hkv, ctx, new, 100 * n + d + fmt + hkv)
    want = oracle.mx_append(cache, fmt, bits(k), bits(v), bt, ctx, cu)
    c, btd, ctxd, cud = dev(cache), dev(bt), dev(ctx), dev(cu)
    max_q, max_kv = int(np.diff(cu).max()), int((ctx + np.diff(cu)).max())
    pa.kv_append_mx(k.cuda(), v.cuda(), c, btd, ctxd, cud, max_q, max_kv)
    torch.cuda.synchronize()
    got = c.cpu().numpy()
    assert np.array_equal(got, want), np.argwhere(got != want)[:5]
    rows = pa.kv_pack_mx(c, btd, ctxd, cud, int(cu[-1]), max_q, max_kv)
    torch.cuda.synchronize()
    assert_rows(bits(rows), oracle.mx_pack(want, d, fmt, bt, ctx, cu))
    # read back and appended elsewhere: the same values
    c2 = torch.randint(0, 256, c.shape, dtype=torch.uint8, device="cuda")
    pa.kv_append_mx(rows[0], rows[1], c2, btd, ctxd, cud, max_q, max_kv)
    again = pa.kv_pack_mx(c2, btd, ctxd, cud, int(cu[-1]), max_q, max_kv)
    torch.cuda.synchronize()
    assert_rows(bits(again), bits(rows))


@pytest.mark.parametrize("batch", (2, 7, 63, 64, 65, 200, 4100))
@pytest.mark.parametrize("fmt,d,hkv", ((4, 64, 3), (8, 128, 1)))
def test_one_long_sequence_among_short_ones(fmt, d, hkv, batch):
    """Token counts of which few are near the longest, where the kernels look an item's sequence up: the long one
    first, last or between, and sequences without a new token on both sides of it."""
    rng = np.random.default_rng(batch)
    for at in sorted({0, batch // 2, batch - 1}):
        say("ragged fmt=%d batch=%d long at %d" % (fmt, batch, at))
        new = rng.integers(0, 3, size=batch)
        new[at] = 40 * batch if batch <= 65 else 1500
        cache, k, v, bt, ctx, cu = case(fmt, d, hkv, rng.integers(0, 40, size=batch), new, batch + at)
        want = oracle.mx_append(cache, fmt, bits(k), bits(v), bt, ctx, cu)
        c, btd, ctxd, cud = dev(cache), dev(bt), dev(ctx), dev(cu)
        max_q, max_kv = int(new.max()), int((ctx + new).max())
        pa.kv_append_mx(k.cuda(), v.cuda(), c, btd, ctxd, cud, max_q, max_kv)
        rows = pa.kv_pack_mx(c, btd, ctxd, cud, int(cu[-1]), max_q, max_kv)
        torch.cuda.synchronize()
        got = c.cpu().numpy()
        assert np.array_equal(got, want), np.argwhere(got != want)[:5]
        assert_rows(bits(rows), oracle.mx_pack(want, d, fmt, bt, ctx, cu))


@pytest.mark.parametrize("fmt", FORMATS)
def test_every_bf16_and_every_code(fmt):
    """All bf16 numbers through the quantiser, alone in their block and beside a larger one, and all codes under all
    scales back."""
    say("every bf16 fmt=%d" % fmt)
    x = np.arange(65536, dtype=np.uint16)
    x = np.repeat(x[:, None], 64, 1)
    x[:, 1:32] = 0
    x[:, 33:] = 0x3fc0                                             # 1.5
    k = torch.from_numpy(x.view(np.int16)).view(torch.bfloat16).view(65536, 1, 64)
    v = torch.roll(k, 7, 0).contiguous()
    cache = np.zeros((4096, 1, oracle.mx_block_bytes(64, fmt)), np.uint8)
    bt, ctx, cu = np.arange(4096, dtype=np.int32)[None], np.zeros(1, np.int32), np.array([0, 65536], np.int32)
    c = dev(cache)
    pa.kv_append_mx(k.cuda(), v.cuda(), c, dev(bt), dev(ctx), dev(cu), 65536, 65536)
    torch.cuda.synchronize()
    kc, ks = oracle.mx_quantise(bits(k)[:, 0], fmt)
    vc, vs = oracle.mx_quantise(bits(v)[:, 0], fmt)
    want = oracle.mx_append(cache[:64], fmt, bits(k)[:1024], bits(v)[:1024], bt[:, :64], ctx, np.array([0, 1024]))
    assert np.array_equal(c[:64].cpu().numpy(), want)
    rows = pa.kv_pack_mx(c, dev(bt), dev(ctx), dev(cu), 65536, 65536, 65536)
    torch.cuda.synchronize()
    got = bits(rows)[:, :, 0]
    for r, (code, s) in zip(got, ((kc, ks), (vc, vs))):
        assert_rows(r, oracle.f64_to_bf16_bits(oracle.mx_values(code, s, fmt)))
    # random bytes: every code under every scale
    c = torch.randint(0, 256, c.shape, dtype=torch.uint8, device="cuda")
    rows = pa.kv_pack_mx(c, dev(bt), dev(ctx), dev(cu), 65536, 65536, 65536)
    torch.cuda.synchronize()
    kp, vp = oracle.mx_pools(c.cpu().numpy(), 64, fmt)
    assert_rows(bits(rows)[0, :, 0], kp.reshape(65536, 64))
    assert_rows(bits(rows)[1, :, 0], vp.reshape(65536, 64))


@pytest.mark.parametrize("fmt", FORMATS)
def test_rows_beyond_the_caches(fmt):
    """An append of over 48 MiB of rows (read past the caches) gives the bytes of its parts' appends."""
    say("large append fmt=%d" % fmt)
    rng, n, hkv, d = np.random.default_rng(5), 13000, 8, 128
    k, v = (torch.randn((n, hkv, d), device="cuda", dtype=torch.bfloat16) for _ in range(2))
    pages = n // 16 + 3
    bt = dev(rng.permutation(pages).astype(np.int32)[None])
    ctx = dev(np.array([5], np.int32))
    whole, parts = (torch.zeros((pages, hkv, oracle.mx_block_bytes(d, fmt)), dtype=torch.uint8, device="cuda") for _ in range(2))
    pa.kv_append_mx(k, v, whole, bt, ctx, dev(np.array([0, n], np.int32)), n, n + 5)
    for a, b in ((0, 6001), (6001, n)):
        pa.kv_append_mx(k[a:b].contiguous(), v[a:b].contiguous(), parts, bt, ctx + a, dev(np.array([0, b - a], np.int32)), b - a, n + 5)
    torch.cuda.synchronize()
    assert torch.equal(whole, parts)


@pytest.mark.parametrize("fmt", FORMATS)
def test_pages_out_of_range_and_null_cu(fmt):
    say("bad pages fmt=%d" % fmt)
    cache, k, v, bt, ctx, cu = case(fmt, 128, 2, [40, 3, 70], [1, 1, 1], 7)
    bt[0, 2], bt[2, 4] = -5, 1 << 30                               # the pages these tokens go to
    c = dev(cache)
    pa.kv_append_mx(k.cuda(), v.cuda(), c, dev(bt), dev(ctx), None, 1, 80)
    rows = pa.kv_pack_mx(c, dev(bt), dev(ctx), None, 3, 1, 80)
    torch.cuda.synchronize()
    want = oracle.mx_append(cache, fmt, bits(k)[1:2], bits(v)[1:2], bt[1:2], ctx[1:2], None)
    assert np.array_equal(c.cpu().numpy(), want)
    got = bits(rows)
    assert not got[:, 0].any() and not got[:, 2].any()
    assert_rows(got[:, 1], oracle.mx_pack(want, 128, fmt, bt[1:2], ctx[1:2], None)[:, 0])


def test_captured_and_on_another_stream():
    say("graph and side stream")
    cache, k, v, bt, ctx, cu = case(4, 128, 4, [10, 33], [50, 9], 11)
    kd, vd, btd, ctxd, cud = k.cuda(), v.cuda(), dev(bt), dev(ctx), dev(cu)
    want = oracle.mx_append(cache, 4, bits(k), bits(v), bt, ctx, cu)
    side = torch.cuda.Stream()
    c = dev(cache)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        pa.kv_append_mx(kd, vd, c, btd, ctxd, cud, 50, 60)
    side.synchronize()
    assert np.array_equal(c.cpu().numpy(), want)
    c = dev(cache)
    buf = torch.zeros((2, 59, 4, 128), dtype=torch.bfloat16, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pa.kv_append_mx(kd, vd, c, btd, ctxd, cud, 50, 60)
        pa.kv_pack_mx(c, btd, ctxd, cud, 59, 50, 60, out=buf)
    for i in range(3):
        c.copy_(dev(cache))
        buf.zero_()
        if i == 2:
            kd.copy_(vd)                                           # other inputs of the same addresses
            want = oracle.mx_append(cache, 4, bits(v), bits(v), bt, ctx, cu)
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(c.cpu().numpy(), want)
        assert_rows(bits(buf), oracle.mx_pack(want, 128, 4, bt, ctx, cu))


def test_refusals_on_the_gpu():
    cache = pa.mx_cache(4, 2, 64, pa.MXFP4)
    k = torch.zeros((3, 2, 64), dtype=torch.bfloat16, device="cuda")
    bt, ctx = torch.zeros((3, 1), dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="k_new and v_new"):
        pa.kv_append_mx(k[:, :1].contiguous(), k[:, :1].contiguous(), cache, bt, ctx, None, 1, 1)
    with pytest.raises(ValueError, match="contiguous"):
        pa.kv_append_mx(k.transpose(0, 1), k, cache, bt, ctx, None, 1, 1)
    with pytest.raises(ValueError, match="cache must be"):
        pa.kv_pack_mx(cache[:, :, :1000].contiguous(), bt, ctx, None, 3, 1, 1)
    with pytest.raises(ValueError, match="out must have shape"):
        pa.kv_pack_mx(cache, bt, ctx, None, 3, 1, 1, out=k)
    with pytest.raises(pa.PearlError, match="bt_stride"):
        pa.kv_pack_mx(cache, bt, ctx, None, 3, 1, 17)
