"""GPU calls on caches of MX blocks as a program makes them: the timing hook, and which form a batch takes."""
import numpy as np
import pytest
import torch

import paper_2609_35158_amd as pa
from gpu_helpers import say
from mx_helpers import dev

pytestmark = pytest.mark.gpu


def test_timing_events_enclose_every_group_of_sequences():
    """1024 sequences, timed alone and with a short one more, which is a group of its own: not less."""
    say("timing events of 1025 sequences")
    hkv, d, n = 2, 64, 1025
    ctx = np.full(n, 1500, np.int32)
    ctx[-1] = 3
    pages = 200                                                    # shared by all
    cache = torch.randint(0, 100, (pages, hkv, pa.mx_block_bytes(d, pa.MXFP4)), dtype=torch.uint8, device="cuda")
    bt = dev(np.random.default_rng(0).integers(0, pages, size=(n, 94)).astype(np.int32))
    q = torch.randn((n, 4, d), device="cuda").to(torch.bfloat16)
    pair = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
    for e in pair:
        e.record()

    def time(batch):
        best = float("inf")
        args = q[:batch].contiguous(), cache, bt[:batch].contiguous(), dev(ctx[:batch])
        for _ in range(10):
            pa.binding.set_kernel_events(*(e.cuda_event for e in pair))
            try:
                pa.decode_mx(*args, 1504)
            finally:
                pa.binding.set_kernel_events(None, None)
            torch.cuda.synchronize()
            best = min(best, pair[0].elapsed_time(pair[1]))
        return best

    alone, both = time(1024), time(1025)
    say("   %.1f and %.1f us" % (1e3 * alone, 1e3 * both))
    assert both > 0.8 * alone
