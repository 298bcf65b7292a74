"""How decode over MX blocks cuts a batch: workgroups of 8, 4 and 2 kv-heads and of one, seen by the partials that they
leave in a workspace filled with a pattern, and the precision of the results."""
import numpy as np
import pytest
import torch

import paper_2609_35158_amd as pa
from gpu_helpers import say
from mx_helpers import BigCase, dev, torch_attention

pytestmark = pytest.mark.gpu

FILL = 0x7f7f7f7f


def _grid(fmt, d):
    """Workgroups of the decode grid: one per compute unit, two at head_dim 64 in 4 bits."""
    return torch.cuda.get_device_properties(0).multi_processor_count * (2 if d * fmt == 256 else 1)


def _slot_runs(ctx, H, bound):
    """Runs that the workspace's partial slots allow: two slots each, or one more than one per sequence."""
    B, longest = len(ctx), -(-bound // 16)
    pps = min(512, -(-max(16, -(-B * H * longest // 4096)) // 16) * 16)
    slots = B * -(-longest // pps)
    return max(1, slots // 2, slots - B)


def _partials(ctx, runs, shares, cost):
    """Partials per kv-head of a page list cut into runs of equal shares, where `cost` entries stand before each sequence's
    pages: one per run that holds pages of a sequence, for every sequence in more than one run."""
    pages = np.asarray(ctx) // 16 + 1
    end = np.cumsum(pages + cost)                                  # entries; a sequence's last `pages` ones are its pages
    share, more = divmod(int(end[-1]), runs * shares)
    begin = np.array([shares * x * share + min(shares * x, more) for x in range(runs)])
    first = np.searchsorted(begin, end - pages, side="right")
    last = np.searchsorted(begin, end - 1, side="right")
    return int((last - first + 1)[last > first].sum())


# format, head_dim, kv-heads, G, sequences, shortest and longest context, bound (0: the longest); kv-heads per workgroup
CASES = [
    (4, 128, 8, 4, 64, 2000, 8000, 0, 8),
    (8, 128, 8, 4, 64, 2000, 8000, 0, 8),
    (8, 128, 8, 2, 512, 64, 1024, 0, 8),
    (4, 128, 8, 1, 512, 64, 1024, 32768, 8),
    (8, 64, 8, 2, 48, 500, 6000, 0, 8),
    (4, 64, 8, 1, 130, 2000, 6200, 65536, 8),
    (8, 128, 4, 8, 130, 2000, 6000, 0, 4),
    (4, 128, 12, 2, 150, 400, 1200, 0, 4),
    (8, 64, 4, 2, 300, 600, 3000, 65536, 4),
    (4, 128, 2, 2, 256, 1000, 6000, 0, 2),
    (8, 128, 10, 1, 300, 400, 1200, 0, 2),
    # a last block of 8 kv-heads that overlaps the one before, by 1 and by 7
    (4, 128, 71, 1, 28, 400, 1200, 0, 8),
    (8, 64, 129, 1, 30, 500, 900, 32768, 8),
    # too few partial slots, or too many pieces of the longest sequence
    (4, 64, 8, 1, 130, 2000, 6200, 0, 1),
    (4, 128, 8, 2, 16, 2000, 30000, 0, 1),
    (8, 128, 8, 4, 20, 2000, 9000, 0, 1),
]


@pytest.mark.parametrize("n", range(len(CASES)))
def test_kv_heads_per_workgroup(n):
    fmt, d, hkv, G, batch, lo, hi, bound, heads = CASES[n]
    say("decode_mx shares fmt=%d d=%d hkv=%d G=%d, %d sequences of %d-%d" % (fmt, d, hkv, G, batch, lo, hi))
    rng = np.random.default_rng(200 + n)
    ctx = rng.integers(lo, hi, size=batch, endpoint=True)
    ctx[0], ctx[-1] = hi, lo
    c = BigCase(fmt, d, hkv, G, ctx, np.ones(batch, np.int64), 200 + n)
    bound = bound or c.max_kv
    bt = torch.nn.functional.pad(c.bt, (0, max(0, -(-bound // 16) - c.bt.shape[1])), value=-1)
    desc = pa.binding.make_desc(bt, c.ctx, None, batch, 1, bound)
    ws = torch.full((pa.workspace_bytes_mx(c.hq, c.cache, desc) // 4,), FILL, dtype=torch.int32, device="cuda")
    lse = torch.full((batch, c.hq), float("nan"), device="cuda")
    out, lse = pa.decode_mx(c.q, c.cache, bt, c.ctx, bound, scale=c.scale, lse=lse, workspace=ws.view(torch.uint8))
    torch.cuda.synchronize()
    assert int(ws[3]) == 0 and torch.isfinite(lse).all() and torch.isfinite(out.float()).all()
    counters = (4 * batch * hkv + 255) // 256 * 64
    written = int((ws[64:ws.numel() - counters] != FILL).sum())
    assert written % (hkv * G * (d + 2)) == 0
    partials = written // (hkv * G * (d + 2))
    runs = min(max(1, _grid(fmt, d) // -(-hkv // heads)), _slot_runs(ctx, hkv, bound))
    say("   partials per kv-head %d" % partials)
    if heads > 1:
        assert partials == _partials(ctx, runs, 8 // heads, 4 if heads == 8 else 0)
    else:
        assert partials <= 2 * runs
        assert partials not in {_partials(ctx, min(max(1, _grid(fmt, d) // -(-hkv // h)), _slot_runs(ctx, hkv, bound)), 8 // h,
                                          4 if h == 8 else 0) for h in (2, 4, 8)}
    # The weights' 16 bits (2^-16 of each) and the sums in 32 bits disappear beside the rounding of the outputs to bf16,
    # whose errors are spread over +-2^-8 of a value: together in squares less than 1.01 of it.
    zero = torch.zeros(1, dtype=torch.int32, device="cuda")
    err = least = 0.0
    for b in sorted({0, 1, batch // 2, batch - 2, batch - 1} | {int(x) for x in rng.integers(0, batch, size=4)}):
        L = int(c.kv[b])
        k, v = pa.kv_pack_mx(c.cache, c.bt[b:b + 1], zero, dev(np.array([0, L], np.int32)), L, L, L)
        ref, ref_lse = torch_attention(c.q[b:b + 1], k, v, c.scale)
        err += float((out[b:b + 1].double() - ref).square().sum())
        least += float((ref.to(torch.bfloat16).double() - ref).square().sum())
        assert float((lse[b:b + 1].double() - ref_lse).abs().max()) < 2e-5, b
    say("   error %.4f of the rounding's" % (err / least) ** 0.5)
    assert err <= 1.01 ** 2 * least
