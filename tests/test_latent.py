"""Attention over latent rows without a GPU: the oracle against worked values, and the library's refusals of arguments (each
before any HIP call)."""
import ctypes

import numpy as np
import pytest

import oracle
import paper_2609_35158_amd as pa
from paper_2609_35158_amd import binding as bd

FAKE = 0x10000
INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3


def _bf16(x):
    return oracle.f64_to_bf16_bits(np.asarray(x, np.float64))


def test_oracle_worked_values():
    # Two keys whose scores differ by ln 3 weigh 1/4 and 3/4; the value is the latent part alone.
    cache = np.zeros((2, 16, 6))
    cache[1, 0], cache[1, 1] = [1, 0, 0, 8, 0, 0], [0, 1, 0, 0, 2, 0]
    q = np.zeros((1, 1, 6))
    q[0, 0, 0], q[0, 0, 4] = 1.0, 0.5                          # scores 1 and 1: equal weights
    bt = np.array([[1]])
    out, lse, size = oracle.latent_attention(_bf16(q), _bf16(cache), bt, np.array([1]), None, 4, 1.0)
    assert np.allclose(out[0, 0], [0.5, 0.5, 0, 4.0]) and np.allclose(size, out) and np.isclose(lse[0, 0], 1 + np.log(2))
    out, lse, _ = oracle.latent_attention(_bf16(q), _bf16(cache), bt, np.array([0]), None, 4, 1.0)
    assert np.allclose(out[0, 0], [1, 0, 0, 8]) and np.isclose(lse[0, 0], 1)      # the second key is not seen


def test_oracle_is_gqa_attention_of_one_head():
    """With the row as key and, padded with zeros, as value, it is the paged GQA oracle with one kv-head."""
    rng = np.random.default_rng(0)
    cache = _bf16(rng.standard_normal((4, 16, 24)))
    q = _bf16(rng.standard_normal((5, 3, 24)))
    bt, ctx, cu = np.array([[2, 0], [3, 1]]), np.array([20, 3]), np.array([0, 3, 5])
    out, lse, _ = oracle.latent_attention(q, cache, bt, ctx, cu, 16, 0.25)
    pool = cache[:, None]
    ref, ref_lse = oracle.attention(q, pool, pool, bt, ctx, cu, 0.25)
    assert np.allclose(out, ref[..., :16]) and np.allclose(lse, ref_lse)


def shape(h=16, dc=512, dr=64, ps=16, n=100):
    return bd.LatentShape(h, dc, dr, ps, n)


def desc(batch=4, stride=64, cu=None, total=None, max_q=1, max_kv=1000, bt=FAKE, ctx=FAKE):
    return bd.SeqDesc(bt, stride, ctx, cu, batch, batch if total is None else total, max_q, max_kv)


def ref(x):
    return None if x is None else ctypes.byref(x)


def attend(fn, s=shape(), d=desc(), q=FAKE, cache=FAKE, scale=0.1, out=FAKE, lse=None, ws=FAKE, wsb=1 << 30):
    return getattr(pa.load(), fn)(ref(s), ref(d), q, cache, scale, out, lse, ws, wsb, None), pa.last_error()


def append(s=shape(), d=desc(), r=bd.RopeDesc(FAKE, 64, 1, 1.0, 1e-6, None, FAKE), q_rope=FAKE, qs=64, rows=FAKE, rs=576, q=FAKE,
           cache=FAKE):
    return pa.load().pearl_latent_append(ref(s), ref(d), ref(r), q_rope, qs, rows, rs, q, cache, None), pa.last_error()


BAD_SHAPES = [(shape(h=0), INVALID), (shape(h=129), UNSUPPORTED), (shape(dc=256), UNSUPPORTED), (shape(dr=32), UNSUPPORTED),
              (shape(dc=128, dr=64), UNSUPPORTED), (shape(ps=32), UNSUPPORTED), (shape(n=0), INVALID), (None, INVALID)]
BAD_SEQS = [(None, INVALID), (desc(batch=0), INVALID), (desc(bt=None), INVALID), (desc(ctx=None), INVALID), (desc(stride=2), INVALID),
            (desc(total=5), INVALID), (desc(max_kv=1 << 26, stride=1 << 23), UNSUPPORTED)]


@pytest.mark.parametrize("fn", ["pearl_attn_latent_decode", "pearl_attn_latent_prefill_append"])
def test_attention_refusals(fn):
    for s, st in BAD_SHAPES:
        assert attend(fn, s=s)[0] == st
    for d, st in BAD_SEQS:
        assert attend(fn, d=d)[0] == st
    for name in ("q", "cache", "out"):
        assert attend(fn, **{name: None})[0] == INVALID
        assert attend(fn, **{name: FAKE + 8})[0] == INVALID
    assert attend(fn, lse=FAKE + 2)[0] == INVALID
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert attend(fn, scale=scale)[0] == INVALID
    assert attend(fn, ws=None)[0] == WORKSPACE and attend(fn, ws=FAKE + 128)[0] == WORKSPACE and attend(fn, wsb=4096)[0] == WORKSPACE
    big = desc(batch=1 << 14, cu=FAKE, total=1 << 25, max_q=1 << 11, max_kv=1 << 12, stride=1 << 9)
    assert attend("pearl_attn_latent_prefill_append", s=shape(h=128), d=big)[0] == UNSUPPORTED


def test_decode_takes_no_cu():
    st, msg = attend("pearl_attn_latent_decode", d=desc(cu=FAKE))
    assert st == INVALID and "cu_q_lens" in msg


def test_append_refusals():
    for s, st in BAD_SHAPES:
        assert append(s=s)[0] == st
    for d, st in BAD_SEQS:
        assert append(d=d)[0] == st
    good = bd.RopeDesc(FAKE, 64, 1, 1.0, 1e-6, None, None)
    for r, st in ((None, INVALID), (bd.RopeDesc(FAKE, 32, 1, 1.0, 1e-6, None, None), INVALID),
                  (bd.RopeDesc(FAKE, 128, 1, 1.0, 1e-6, None, None), UNSUPPORTED), (bd.RopeDesc(None, 64, 1, 1.0, 1e-6, None, None), INVALID),
                  (bd.RopeDesc(FAKE, 64, 1, 1.0, 1e-6, FAKE, None), INVALID), (bd.RopeDesc(FAKE, 64, 1, 1.0, -1.0, None, None), INVALID)):
        assert append(r=r)[0] == st
    for kw in (dict(qs=56), dict(qs=68), dict(qs=0), dict(rs=568), dict(rs=580), dict(rs=-576)):
        st, msg = append(r=good, **kw)
        assert st == INVALID and "stride" in msg
    for name in ("q_rope", "rows", "q", "cache"):
        assert append(**{name: None})[0] == INVALID and append(**{name: FAKE + 4})[0] == INVALID
    assert append(d=desc(cu=FAKE, total=0, max_q=0))[0] == 0


def test_workspace_bytes():
    f = pa.load().pearl_latent_workspace_bytes

    def size(s, d):
        return f(ref(s), ref(d))

    small, wide, prompt = size(shape(), desc()), size(shape(h=64), desc()), size(shape(), desc(cu=FAKE, total=100, max_q=50))
    assert 0 < small < wide == prompt < 68 << 20 and small % 256 == 0
    assert size(shape(), desc(batch=600, total=600, max_kv=1020)) == small       # by the bounds, not by the batch
    assert size(shape(h=0), desc()) == 0 and "num_q_heads" in pa.last_error()
    assert size(shape(), desc(stride=2)) == 0 and "bt_stride" in pa.last_error()
