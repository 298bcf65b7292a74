"""Rotary position embedding without a GPU: the oracle against worked values and its own properties, and the library's
refusals of arguments (each before any HIP call)."""
import ctypes

import numpy as np
import pytest

import oracle
import paper_2609_35158_amd as pa
from paper_2609_35158_amd import binding as bd

FAKE = 0x10000
INVALID, UNSUPPORTED = 1, 2


def test_oracle_worked_values():
    # two channels by a quarter turn a position: (1, 0) -> (0, 1) -> (-1, 0)
    x = np.zeros((3, 1, 4))
    x[:, 0] = [1.0, 2.0, 0.0, 5.0]
    quarter = np.array([np.pi / 2, 0.0], np.float32)
    half = oracle.rotate(x, np.array([0, 1, 2]), quarter, False)
    assert np.allclose(half[:, 0], [[1, 2, 0, 5], [0, 2, 1, 5], [-1, 2, 0, 5]], atol=1e-6)
    nxt = oracle.rotate(x, np.array([0, 1, 2]), quarter, True)
    assert np.allclose(nxt[:, 0], [[1, 2, 0, 5], [-2, 1, 0, 5], [-1, -2, 0, 5]], atol=1e-6)


@pytest.mark.parametrize("interleaved", [False, True])
def test_oracle_scores_depend_on_distance(interleaved):
    rng = np.random.default_rng(1)
    f = (10000.0 ** (-np.arange(0, 32, 2) / 32)).astype(np.float32)
    q, k = rng.standard_normal((2, 1, 1, 64))

    def score(p, r):
        a, b = (oracle.rotate(x, np.array([at]), f, interleaved) for x, at in ((q, p), (k, r)))
        return float((a * b).sum())

    assert abs(score(1000, 990) - score(17, 7)) < 1e-9
    assert abs(score(1000, 990) - score(1000, 991)) > 1e-6


def test_oracle_norm_and_positions():
    x = np.array([[3.0, 4.0]])
    assert np.allclose(oracle.norm_rows(x, np.array([1.0, 2.0]), 0.0), [[3 / np.sqrt(12.5), 8 / np.sqrt(12.5)]])
    assert list(oracle.positions(np.array([5, -1, 7]), np.array([0, 2, 3, 5]), 6)) == [5, 6, -1, 7, 8, -1]
    assert list(oracle.positions(np.array([5, 0]), None, 2)) == [5, 0]


def shape(hq=32, hkv=8, d=128, ps=16, n=100):
    return bd.KvShape(hq, hkv, d, ps, n)


def desc(batch=4, stride=64, cu=None, total=None, max_q=1, max_kv=1000, bt=FAKE, ctx=FAKE):
    return bd.SeqDesc(bt, stride, ctx, cu, batch, batch if total is None else total, max_q, max_kv)


def rope(freq=FAKE, rotary=128, next_=0, factor=1.0, eps=1e-6, qw=None, kw=None):
    return bd.RopeDesc(freq, rotary, next_, factor, eps, qw, kw)


def ref(x):
    return None if x is None else ctypes.byref(x)


def rows(s=None, d=None, r=None, q=FAKE, qs=4096, k=FAKE + 4096, ks=1024, qo=FAKE + 8192, ko=FAKE + 12288, **kw):
    s, d, r = s or shape(), d or desc(), r or rope()
    return pa.load().pearl_rope_rows(ref(s), ref(d), ref(r), q, qs, k, ks, qo, ko, None), pa.last_error()


def append(s=None, d=None, r=None, q=FAKE, qs=4096, k=FAKE, ks=1024, v=FAKE, vs=1024, qo=FAKE + 8192, kp=FAKE, vp=FAKE):
    s, d, r = s or shape(), d or desc(), r or rope()
    return pa.load().pearl_kv_append_rope(ref(s), ref(d), ref(r), q, qs, k, ks, v, vs, qo, kp, vp, None), pa.last_error()


@pytest.mark.parametrize("call", [rows, append])
def test_refusals(call):
    assert call(s=shape(hkv=6))[0] == INVALID
    assert call(s=shape(d=96))[0] == UNSUPPORTED
    assert call(s=shape(hq=32, hkv=2))[0] == UNSUPPORTED
    assert call(d=desc(batch=0))[0] == INVALID
    assert call(d=desc(ctx=None))[0] == INVALID
    assert call(d=desc(total=9))[0] == INVALID
    assert call(d=desc(cu=FAKE, total=3, max_q=4))[0] == INVALID
    for rotary in (0, -16, 8, 24, 136, 144):
        st, msg = call(r=rope(rotary=rotary))
        assert st == UNSUPPORTED and "rotary_dim" in msg, rotary
    st, msg = call(s=shape(d=64), r=rope(rotary=128))
    assert st == UNSUPPORTED and "rotary_dim" in msg
    for bad in (rope(freq=None), rope(freq=FAKE + 2), rope(next_=2), rope(factor=float("inf")), rope(factor=float("nan")),
                rope(eps=-1e-6), rope(eps=float("nan")), rope(qw=FAKE + 8), rope(kw=FAKE + 2)):
        assert call(r=bad)[0] == INVALID
    for name, width in (("qs", 4096), ("ks", 1024)):
        for stride in (0, -width, width - 8, width + 4, 1 << 62):
            st, msg = call(**{name: stride})
            assert st == INVALID and "stride" in msg, (name, stride)
    for name in ("q", "k", "qo"):
        assert call(**{name: None})[0] == INVALID
        assert call(**{name: FAKE + 8})[0] == INVALID
    st, msg = call(q=FAKE, qo=FAKE, qs=4104)                            # in place, but not contiguous
    assert st == INVALID and "in place" in msg


def test_refusals_of_one_call():
    st, msg = rows(k=FAKE, ko=FAKE, ks=1032)
    assert st == INVALID and "in place" in msg
    assert rows(ko=None)[0] == INVALID
    assert append(d=desc(bt=None))[0] == INVALID
    assert append(d=desc(stride=2))[0] == INVALID
    assert append(vs=1020)[0] == INVALID
    for name in ("v", "kp", "vp"):
        assert append(**{name: None})[0] == INVALID
        assert append(**{name: FAKE + 4})[0] == INVALID
    for f, n in ((pa.load().pearl_rope_rows, 9), (pa.load().pearl_kv_append_rope, 12)):
        assert f(*[None] * 3, *([FAKE, 4096] if n else []), FAKE, 1024, *([FAKE, 1024] if n == 12 else []), FAKE, FAKE,
                 *([FAKE] if n == 12 else []), None) == INVALID          # no shape


def test_no_rows_is_no_work():
    d = desc(cu=FAKE, total=0, max_q=0, max_kv=0)
    assert rows(d=d)[0] == 0 and append(d=d)[0] == 0
