"""Limits of the calls on a cache of MX blocks, on the CPU: every call below fails validation before any HIP call."""
import ctypes

import pytest

import paper_2609_35158_amd as pa
from test_abi import FAKE, UNSUPPORTED, WORKSPACE, desc, shape


@pytest.mark.parametrize("fn", ["pearl_attn_decode_mx", "pearl_attn_decode_append_mx"])
def test_pages_that_a_group_of_sequences_can_hold(fn):
    """The kernel cuts a list of the group's pages with 4 entries more for each of its up to 1024 sequences, in int32; past
    it the cut would begin shares at negative entries and read block tables in front of the first one."""
    def call(batch, pages):
        new = (FAKE, FAKE) if fn.endswith("append_mx") else ()
        d = desc(batch=batch, stride=pages, max_kv=16 * pages)
        st = getattr(pa.load(), fn)(ctypes.byref(shape()), ctypes.byref(d), 4, FAKE, *new, FAKE, 0.1, FAKE, None, FAKE, 1 << 20, None)
        return st, pa.last_error()

    most = (1 << 31) // 1024 - 1 - 4
    assert call(1024, most)[0] == WORKSPACE                        # as far as its workspace of 1 MiB
    for pages in (most + 1, most + 4):
        st, msg = call(1024, pages)
        assert st == UNSUPPORTED and "int32 pages" in msg
    assert call(1023, most + 4)[0] == WORKSPACE
    assert call(2048, 1 << 19)[0] == WORKSPACE                     # groups of 1024
