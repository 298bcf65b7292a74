"""The cache of MX blocks on the CPU: the oracle's quantiser against the format's definition, and the entry points'
refusals (every call below fails validation before any HIP call)."""
import ctypes

import numpy as np
import pytest
import torch

import oracle
import paper_2609_35158_amd as pa
from paper_2609_35158_amd import binding as bd
from test_abi import FAKE, INVALID, UNSUPPORTED, WORKSPACE, desc, shape

FORMATS = (pa.MXFP4, pa.MXFP8)


def bf16(x):
    return torch.as_tensor(x, dtype=torch.float64).to(torch.bfloat16).view(torch.int16).numpy().view(np.uint16)


def test_element_values():
    assert oracle.mx_element_values(4)[:8].tolist() == [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    assert oracle.mx_element_values(4)[8:].tolist() == [-v for v in [0, 0.5, 1, 1.5, 2, 3, 4, 6]]
    e4m3 = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(oracle.mx_element_values(8), e4m3, equal_nan=True)


@pytest.mark.parametrize("fmt", FORMATS)
def test_quantise_by_the_definition(fmt):
    """Least scale, nearest element, ties to the even code, over blocks of many magnitudes."""
    rng = np.random.default_rng(fmt)
    x = rng.standard_normal((400, 32)) * np.exp2(rng.integers(-130, 124, size=(400, 1)))
    x[:40] = rng.integers(-16, 17, size=(40, 32)) / 4.0                    # many ties
    xb = bf16(x)
    x = oracle.bf16_bits_to_f64(xb)
    codes, scales = oracle.mx_quantise(xb, fmt)
    e_max, most = (2, 6.0) if fmt == 4 else (8, 448.0)
    values = oracle.mx_element_values(fmt)
    back = oracle.mx_values(codes, scales, fmt)
    for r in range(len(x)):
        s, top = int(scales[r, 0]), np.abs(x[r]).max()
        assert top <= 1.75 * 2.0 ** (e_max + s - 127)
        assert s == 1 or top > 1.75 * 2.0 ** (e_max + s - 128)
        unit = 2.0 ** (s - 127)
        for i in range(32):
            y, c = x[r, i] / unit, int(codes[r, i])
            off = np.abs(values - np.clip(y, -most, most))
            assert abs(values[c] - np.clip(y, -most, most)) == np.nanmin(off)
            ties = np.flatnonzero(off == np.nanmin(off))
            if len(set(values[ties])) > 1:
                assert c % 2 == 0
            assert back[r, i] == values[c] * unit
            assert np.signbit(values[c]) == np.signbit(y)


@pytest.mark.parametrize("fmt", FORMATS)
def test_values_survive_a_second_quantisation(fmt):
    rng = np.random.default_rng(10 + fmt)
    x = rng.standard_normal((3000, 64)) * np.exp2(rng.integers(-100, 100, size=(3000, 1)))
    x[0] = 0.0
    values = oracle.mx_values(*oracle.mx_quantise(bf16(x), fmt), fmt)
    rows = oracle.f64_to_bf16_bits(values)
    assert np.array_equal(oracle.bf16_bits_to_f64(rows), values)           # exact in bf16
    assert np.array_equal(oracle.mx_values(*oracle.mx_quantise(rows, fmt), fmt), values)


@pytest.mark.parametrize("fmt", FORMATS)
def test_blocks_with_nan_infinity_zero_and_the_least_numbers(fmt):
    x = np.zeros((5, 64))
    x[0, 3], x[1, 40], x[2, 63] = np.nan, np.inf, -np.inf
    x[3, 0], x[3, 1] = 2.0 ** -133, -0.0
    codes, scales = oracle.mx_quantise(bf16(x), fmt)
    assert scales.tolist() == [[255, 1], [1, 255], [1, 255], [1, 1], [1, 1]]
    back = oracle.mx_values(codes, scales, fmt)
    assert np.isnan(back[0, :32]).all() and (back[0, 32:] == 0).all() and np.isnan(back[1, 32:]).all()
    assert codes[3, 1] == 1 << (fmt - 1) and not codes[4].any()
    assert back[3, 0] == (0.0 if fmt == 4 else 2.0 ** -133)                # half the least step of E2M1 ties to 0


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d", (64, 128))
def test_layout_places_every_byte_once(fmt, d):
    from oracle.mx_cache import _places
    seen = np.concatenate([np.concatenate(_places(s, d, fmt)) for s in range(16)])
    assert sorted(seen) == list(range(oracle.mx_block_bytes(d, fmt)))
    assert pa.mx_block_bytes(d, fmt) == oracle.mx_block_bytes(d, fmt)


def test_append_and_pack_round_trip_on_the_oracle():
    rng = np.random.default_rng(3)
    for fmt in FORMATS:
        for d in (64, 128):
            ctx, cu = np.array([5, 30]), np.array([0, 20, 23])
            bt = np.array([[4, 1, 0], [2, 5, 3]])
            cache = rng.integers(0, 256, size=(6, 2, oracle.mx_block_bytes(d, fmt)), dtype=np.uint8)
            k, v = (bf16(rng.standard_normal((23, 2, d))) for _ in range(2))
            after = oracle.mx_append(cache, fmt, k, v, bt, ctx, cu)
            rows = oracle.mx_pack(after, d, fmt, bt, ctx, cu)
            for x, r in ((k, rows[0]), (v, rows[1])):
                assert np.array_equal(oracle.bf16_bits_to_f64(r), oracle.mx_values(*oracle.mx_quantise(x, fmt), fmt))
            touched = (after != cache).sum()
            assert 0 < touched <= 23 * 2 * 2 * (d * fmt // 8 + d // 32)


# --------------------------------------------------------------------------------- refusals

def _copy_args(fn, a, b, c):
    return (a, b, c) if fn == "pearl_kv_append_mx" else (a, c)


@pytest.mark.parametrize("fn", ["pearl_kv_append_mx", "pearl_kv_pack_mx"])
def test_copy_refusals(fn):
    f = getattr(pa.load(), fn)

    def call(s, d, fmt=4, a=FAKE, b=FAKE, c=FAKE):
        return f(None if s is None else ctypes.byref(s), None if d is None else ctypes.byref(d), fmt,
                 *_copy_args(fn, a, b, c), None), pa.last_error()

    assert call(None, desc())[0] == INVALID
    assert call(shape(), None)[0] == INVALID
    for fmt in (0, 5, 16, -4):
        st, msg = call(shape(), desc(), fmt=fmt)
        assert st == UNSUPPORTED and "format" in msg
    assert call(shape(d=96), desc())[0] == UNSUPPORTED
    assert call(shape(ps=32), desc())[0] == UNSUPPORTED
    assert call(shape(hq=24), desc())[0] == UNSUPPORTED
    assert call(shape(n=0), desc())[0] == INVALID
    assert call(shape(), desc(batch=0))[0] == INVALID
    assert call(shape(), desc(stride=10, max_kv=1000))[0] == INVALID
    assert call(shape(), desc(total=5))[0] == INVALID
    assert call(shape(), desc(cu=FAKE, total=0, max_q=0)) == (0, "")         # nothing to move
    for at in ("a", "c"):
        assert call(shape(), desc(), **{at: None})[0] == INVALID
        st, msg = call(shape(), desc(), **{at: FAKE + 8})
        assert st == INVALID and "aligned" in msg


def test_block_bytes_refuses_other_shapes():
    for d, fmt in ((96, 4), (0, 8), (128, 6), (64, 0)):
        assert pa.load().pearl_mx_block_bytes(d, fmt) == 0 and pa.last_error()
        with pytest.raises(pa.PearlError):
            pa.mx_block_bytes(d, fmt)


def test_binding_checks_tensors_before_the_library():
    cache = pa.mx_cache(4, 2, 64, pa.MXFP4, device="cpu")
    assert tuple(cache.shape) == (4, 2, 1088) and cache.dtype == torch.uint8
    k = torch.zeros((3, 2, 64), dtype=torch.bfloat16)
    bt, ctx = torch.zeros((3, 1), dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):
        pa.kv_append_mx(k, k, cache, bt, ctx, None, 1, 1)
    with pytest.raises(TypeError, match="k_new"):
        pa.kv_append_mx(k.float(), k, cache, bt, ctx, None, 1, 1)
    with pytest.raises(ValueError, match="GPU"):
        pa.kv_pack_mx(cache, bt, ctx, None, 3, 1, 1)
    with pytest.raises(TypeError, match="cache"):
        pa.kv_pack_mx(cache.float(), bt, ctx, None, 3, 1, 1)


ATTENTION = ("pearl_attn_decode_mx", "pearl_attn_decode_append_mx", "pearl_attn_prefill_append_mx")


@pytest.mark.parametrize("fn", ATTENTION)
def test_attention_refusals(fn):
    f = getattr(pa.load(), fn)
    prefill, append = fn == ATTENTION[2], fn == ATTENTION[1]

    def call(s, d, fmt=4, q=FAKE, k=FAKE, v=FAKE, cache=FAKE, scale=0.1, out=FAKE, lse=None, ws=FAKE, wsb=1 << 30):
        st = f(None if s is None else ctypes.byref(s), None if d is None else ctypes.byref(d), fmt, q,
               *((k, v) if append else ()), cache, scale, out, lse, ws, wsb, None)
        return st, pa.last_error()

    ok = dict(cu=FAKE, total=9, max_q=5) if prefill else {}
    assert call(None, desc(**ok))[0] == INVALID
    assert call(shape(), None)[0] == INVALID
    for fmt in (0, 3, 9):
        st, msg = call(shape(), desc(**ok), fmt=fmt)
        assert st == UNSUPPORTED and "format" in msg
    for s in (shape(d=80), shape(ps=8), shape(hq=24), shape(hq=128, hkv=8)):
        assert call(s, desc(**ok))[0] == UNSUPPORTED
    assert call(shape(hkv=5), desc(**ok))[0] == INVALID
    for bad in (dict(batch=0), dict(stride=0), dict(stride=10, max_kv=1000)):
        assert call(shape(), desc(**dict(ok, **bad)))[0] == INVALID
    for name in ("q", "cache", "out") + (("k", "v") if append else ()):
        assert call(shape(), desc(**ok), **{name: None})[0] == INVALID
        st, msg = call(shape(), desc(**ok), **{name: FAKE + 8})
        assert st == INVALID and "aligned" in msg, name
    assert call(shape(), desc(**ok), lse=FAKE + 2)[0] == INVALID
    assert call(shape(), desc(**ok), ws=None)[0] == WORKSPACE
    assert call(shape(), desc(**ok), ws=FAKE + 16)[0] == WORKSPACE
    st, msg = call(shape(), desc(**ok), wsb=100)
    assert st == WORKSPACE and "100" in msg
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert call(shape(), desc(**ok), scale=scale)[0] == INVALID
    if not prefill:
        st, msg = call(shape(), desc(cu=FAKE))
        assert st == INVALID and "cu_q_lens" in msg
        assert call(shape(), desc(total=5))[0] == INVALID
    assert call(shape(), desc(batch=1, stride=(1 << 21) + 1, max_kv=(1 << 25) + 1, **({} if not prefill else dict(cu=FAKE, total=1))))[0] == UNSUPPORTED


def test_no_query_heads_are_not_taken_for_as_many_as_kv_heads():
    cache = (5, 2, pa.mx_block_bytes(64, pa.MXFP4))
    assert bd._mx_geometry(None, cache)[0].num_q_heads == 2
    none, _, ref = bd._mx_geometry(0, cache)
    assert none.num_q_heads == 0
    q = desc()
    assert pa.load().pearl_attn_workspace_bytes(ref, ctypes.byref(q)) == 0
    assert "num_q_heads (0)" in bd.last_error()
