"""Attention over a paged cache of latent rows: values that are not finite at up to 16 rows a sequence and where all scores of a cut tile's
piece are minus infinity, and batches with rows behind the last sequence."""
import numpy as np
import pytest
import torch

import oracle
import paper_2609_35158_amd as pa
from gpu_helpers import bits
from latent_helpers import LatentCase, check
from rope_helpers import bf16

pytestmark = pytest.mark.gpu


def put(c, b, key, channels, value):
    c.cache[int(c.bt[b, key // 16]), key % 16, channels] = bits(bf16([value]))[0]


def positive(c, channels):
    """Queries that make an infinity of these channels one of the same sign in their scores."""
    q = oracle.bf16_bits_to_f64(bits(c.q))
    q[..., channels] = np.abs(q[..., channels]) + 0.25
    c.q = bf16(q)


def check_odd(c, out, lse):
    """Elements are finite where the oracle's are, and within its bounds there."""
    ref, ref_lse, tol, tol_lse = c.oracle()
    n = c.owned
    got, got_lse = oracle.bf16_bits_to_f64(bits(out))[:n], lse.cpu().numpy().astype(np.float64)[:n]
    for g, r, t in ((got, ref[:n], tol[:n]), (got_lse, ref_lse[:n], tol_lse[:n])):
        finite = np.isfinite(r)
        assert np.array_equal(np.isfinite(g), finite), np.argwhere(np.isfinite(g) != finite)[:4]
        assert (np.abs(g - r)[finite] <= t[finite]).all()
    return ref[:n]


NEW = {4: [4, 3, 1, 4], 1: [16, 9, 2], 16: [1, 1], 5: [3, 2, 0, 3]}


@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("dc", [512, 256])
@pytest.mark.parametrize("heads", [4, 1, 5])
def test_not_finite_at_16_rows(heads, dc, value):
    """Several channels of several new tokens; tokens before them in the same page, and other sequences, see nothing of it, also where the
    tile is cut (a context of 2000)."""
    new = NEW[heads]
    ctx = [30, 2000, 15, 64][:len(new)]
    c = LatentCase(heads, dc, ctx, new, seed=heads + dc)
    channels = [0, 7, 8, 15, 100, 129, dc - 1]
    positive(c, channels)
    for b, n in enumerate(new):
        for i in range(1, n):
            put(c, b, ctx[b] + i, channels[i % 3::3], value)
    ref = check_odd(c, *c.prefill())
    rows = int(np.isnan(ref).any((1, 2)).sum())
    assert rows == sum(max(n - 1, 0) for n in new)             # as the case is meant


@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("heads,dc", [(16, 512), (40, 512), (128, 512), (20, 256), (7, 256)])
def test_not_finite_at_64_rows(heads, dc, value):
    ctx, new = [30, 1500, 5, 64], [20, 7, 0, 40]
    c = LatentCase(heads, dc, ctx, new, seed=heads + dc)
    channels = [1, 8, 17, 64, 130, dc - 1]
    positive(c, channels)
    for b, n in enumerate(new):
        for i in range(3, n, 5):
            put(c, b, ctx[b] + i, channels[i % 3::3], value)
    ref = check_odd(c, *c.prefill())
    assert int(np.isnan(ref).any((1, 2)).sum()) == sum(max(n - 3, 0) for n in new)


@pytest.mark.parametrize("ctx", [20, 5000])
@pytest.mark.parametrize("heads,dc", [(16, 512), (64, 512), (4, 256), (30, 256)])
def test_all_scores_minus_infinity(heads, dc, ctx):
    """NaN, as 0 / 0 is, and the logarithm of 0; in that sequence alone."""
    c = LatentCase(heads, dc, [ctx, 100], [1, 1], seed=heads)
    positive(c, [dc + 3])
    for key in range(ctx + 1):
        put(c, 0, key, dc + 3, float("-inf"))
    out, lse = c.decode()
    assert bool(torch.isnan(out[0]).all()) and bool((lse[0] == float("-inf")).all())
    ref, ref_lse, tol, tol_lse = c.oracle()
    got = oracle.bf16_bits_to_f64(bits(out))
    assert (np.abs(got - ref) <= tol)[1].all() and (np.abs(lse.cpu().numpy() - ref_lse) <= tol_lse)[1].all()


@pytest.mark.parametrize("dc", [512, 256])
def test_notes_of_a_tile_end_with_it(dc):
    """Many short sequences, several tiles a workgroup, every third with values that are not finite."""
    rng = np.random.default_rng(dc)
    new = rng.integers(1, 5, size=700)
    ctx = rng.integers(0, 60, size=700)
    c = LatentCase(4, dc, ctx, new, seed=dc)
    positive(c, list(range(dc)))
    for b in range(0, 700, 3):
        if new[b] > 1:
            put(c, b, int(ctx[b] + new[b]) - 1, [b % dc, (7 * b + 8) % dc], (float("-inf"), float("nan"))[b % 2])
    check_odd(c, *c.prefill())


@pytest.mark.parametrize("heads,dc", [(16, 512), (16, 256), (64, 512), (64, 256)])
def test_pieces_of_scores_of_minus_infinity(heads, dc):
    """A cut tile's piece whose scores are all minus infinity has weight 0, and its channels that are not finite are NaN in the output
    (0 times infinity), as in a tile that is not cut."""
    c = LatentCase(heads, dc, [4000, 200], [1, 1], seed=heads)
    positive(c, [5, 40, dc])
    for key in range(1500):
        put(c, 0, key, dc, float("-inf"))                      # of the rotated part
    put(c, 0, 100, 5, float("-inf"))
    put(c, 0, 1100, 40, float("-inf"))
    ref = check_odd(c, *c.decode())
    assert np.isnan(ref[0][:, [5, 40]]).all() and np.isnan(ref).sum() == 2 * heads


@pytest.mark.parametrize("heads,dc,ctx,new,spare", [(16, 512, [3000, 40], [1, 1], 62), (4, 512, [900, 17, 5], [4, 1, 3], 200),
                                                    (1, 256, [5000], [16], 1000), (16, 512, [700, 1200], [4, 3], 500),
                                                    (128, 512, [2000, 30, 77], [1, 1, 1], 61)])
def test_rows_behind_the_last_sequence(heads, dc, ctx, new, spare):
    """They take no part: the call's outputs are those without them, bit for bit."""
    c = LatentCase(heads, dc, ctx, new, seed=heads, spare=spare)
    out, lse = c.prefill()
    check(c, out, lse)
    q, cache, bt, ctx_d, cu = c.args()
    alone = pa.latent_prefill_append(q[:c.owned].contiguous(), cache, bt, ctx_d, cu, c.max_q, c.max_kv, c.scale, return_lse=True)
    assert torch.equal(out[:c.owned], alone[0]) and torch.equal(lse[:c.owned], alone[1])
