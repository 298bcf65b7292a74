"""ctypes binding of libpearl_attn.so (the C ABI in include/pearl_attn.h).

Argument marshalling only: every step of the computation runs in the library's HIP kernels.
Tensors are torch tensors on the current HIP device; the torch current stream is passed as the
launch stream.  If the library is missing or fails to load, every call raises -- there is no
fallback implementation.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import Optional, Tuple

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libpearl_attn.so")

PEARL_OK = 0
PAGE_SIZE = 16                                      # tokens per page
_lib = None


class PearlError(RuntimeError):
    def __init__(self, status: int, func: str, detail: str):
        super().__init__("%s failed: %s: %s" % (func, _status_name(status), detail))
        self.status = status


class KvShape(ctypes.Structure):
    _fields_ = [("num_q_heads", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("num_pages", ctypes.c_int32)]


class SeqDesc(ctypes.Structure):
    _fields_ = [("block_table", ctypes.c_void_p), ("bt_stride", ctypes.c_int32),
                ("ctx_lens", ctypes.c_void_p), ("cu_q_lens", ctypes.c_void_p),
                ("batch", ctypes.c_int32), ("total_q", ctypes.c_int32),
                ("max_q_len", ctypes.c_int32), ("max_kv_len", ctypes.c_int32)]


class RopeDesc(ctypes.Structure):
    _fields_ = [("inv_freq", ctypes.c_void_p), ("rotary_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32),
                ("factor", ctypes.c_float), ("eps", ctypes.c_float), ("q_weight", ctypes.c_void_p),
                ("k_weight", ctypes.c_void_p)]


class LatentShape(ctypes.Structure):
    _fields_ = [("num_q_heads", ctypes.c_int32), ("latent_dim", ctypes.c_int32), ("rope_dim", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("num_pages", ctypes.c_int32)]


EXPORTED = ("pearl_abi_version", "pearl_status_str", "pearl_last_error", "pearl_kv_append",
            "pearl_attn_workspace_bytes", "pearl_attn_prefill_append", "pearl_attn_decode",
            "pearl_attn_mixed", "pearl_kv_pack", "pearl_kv_unpack", "pearl_set_kernel_events",
            "pearl_hbm_copy", "pearl_hbm_read", "pearl_hbm_read_nt", "pearl_hbm_fill", "pearl_attn_decode_static",
            "pearl_attn_decode_static_max_bytes", "pearl_attn_decode_append", "pearl_mx_block_bytes",
            "pearl_kv_append_mx", "pearl_kv_pack_mx", "pearl_attn_decode_mx", "pearl_attn_decode_append_mx",
            "pearl_attn_prefill_append_mx", "pearl_rope_rows", "pearl_kv_append_rope", "pearl_latent_append",
            "pearl_latent_workspace_bytes", "pearl_attn_latent_decode", "pearl_attn_latent_prefill_append")


def load(path: str = LIB_PATH):
    """Load (once) and type the library.  Raises if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError("HIP library %s is not built (run __graft_entry__.build() or "
                           "python -m paper_2609_35158_amd.build)" % path)
    lib = ctypes.CDLL(path)
    P = ctypes.POINTER
    lib.pearl_abi_version.restype = ctypes.c_int
    lib.pearl_abi_version.argtypes = []
    lib.pearl_status_str.restype = ctypes.c_char_p
    lib.pearl_status_str.argtypes = [ctypes.c_int]
    lib.pearl_last_error.restype = ctypes.c_char_p
    lib.pearl_last_error.argtypes = []
    lib.pearl_kv_append.restype = ctypes.c_int
    lib.pearl_kv_append.argtypes = [P(KvShape), P(SeqDesc), ctypes.c_void_p, ctypes.c_void_p,
                                    ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]
    for name in ("pearl_kv_pack", "pearl_kv_unpack"):
        f = getattr(lib, name)
        f.restype = ctypes.c_int
        f.argtypes = [P(KvShape), P(SeqDesc), ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                      ctypes.c_void_p]
    lib.pearl_attn_workspace_bytes.restype = ctypes.c_size_t
    lib.pearl_attn_workspace_bytes.argtypes = [P(KvShape), P(SeqDesc)]
    for name in ("pearl_attn_prefill_append", "pearl_attn_decode", "pearl_attn_mixed"):
        f = getattr(lib, name)
        f.restype = ctypes.c_int
        f.argtypes = [P(KvShape), P(SeqDesc), ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                      ctypes.c_float, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                      ctypes.c_size_t, ctypes.c_void_p]
    lib.pearl_attn_decode_append.restype = ctypes.c_int
    lib.pearl_attn_decode_append.argtypes = [P(KvShape), P(SeqDesc), ctypes.c_void_p, ctypes.c_void_p,
                                             ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_float,
                                             ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t,
                                             ctypes.c_void_p]
    lib.pearl_attn_decode_static.restype = ctypes.c_int
    lib.pearl_attn_decode_static.argtypes = [P(KvShape), P(SeqDesc), ctypes.c_void_p, ctypes.c_void_p,
                                             ctypes.c_void_p, ctypes.c_float, ctypes.c_void_p, ctypes.c_void_p,
                                             ctypes.c_void_p]
    lib.pearl_attn_decode_static_max_bytes.restype = ctypes.c_size_t
    lib.pearl_attn_decode_static_max_bytes.argtypes = []
    lib.pearl_mx_block_bytes.restype = ctypes.c_size_t
    lib.pearl_mx_block_bytes.argtypes = [ctypes.c_int, ctypes.c_int]
    lib.pearl_kv_append_mx.restype = ctypes.c_int
    lib.pearl_kv_append_mx.argtypes = [P(KvShape), P(SeqDesc), ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p,
                                       ctypes.c_void_p, ctypes.c_void_p]
    lib.pearl_kv_pack_mx.restype = ctypes.c_int
    lib.pearl_kv_pack_mx.argtypes = [P(KvShape), P(SeqDesc), ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p,
                                     ctypes.c_void_p]
    for name in ("pearl_attn_decode_mx", "pearl_attn_prefill_append_mx"):
        f = getattr(lib, name)
        f.restype = ctypes.c_int
        f.argtypes = [P(KvShape), P(SeqDesc), ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_float,
                      ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
    lib.pearl_attn_decode_append_mx.restype = ctypes.c_int
    lib.pearl_attn_decode_append_mx.argtypes = [P(KvShape), P(SeqDesc), ctypes.c_int, ctypes.c_void_p,
                                                ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_float,
                                                ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t,
                                                ctypes.c_void_p]
    R, I64, V = P(RopeDesc), ctypes.c_int64, ctypes.c_void_p
    lib.pearl_rope_rows.restype = ctypes.c_int
    lib.pearl_rope_rows.argtypes = [P(KvShape), P(SeqDesc), R, V, I64, V, I64, V, V, V]
    lib.pearl_kv_append_rope.restype = ctypes.c_int
    lib.pearl_kv_append_rope.argtypes = [P(KvShape), P(SeqDesc), R, V, I64, V, I64, V, I64, V, V, V, V]
    lib.pearl_latent_append.restype = ctypes.c_int
    lib.pearl_latent_append.argtypes = [P(LatentShape), P(SeqDesc), R, V, I64, V, I64, V, V, V]
    lib.pearl_latent_workspace_bytes.restype = ctypes.c_size_t
    lib.pearl_latent_workspace_bytes.argtypes = [P(LatentShape), P(SeqDesc)]
    for name in ("pearl_attn_latent_decode", "pearl_attn_latent_prefill_append"):
        f = getattr(lib, name)
        f.restype = ctypes.c_int
        f.argtypes = [P(LatentShape), P(SeqDesc), V, V, ctypes.c_float, V, V, V, ctypes.c_size_t, V]
    lib.pearl_set_kernel_events.restype = None
    lib.pearl_set_kernel_events.argtypes = [ctypes.c_void_p, ctypes.c_void_p]
    # measurement tooling (include/pearl_bench.h)
    lib.pearl_hbm_copy.restype = ctypes.c_int
    lib.pearl_hbm_copy.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
    for name in ("pearl_hbm_read", "pearl_hbm_read_nt"):
        f = getattr(lib, name)
        f.restype = ctypes.c_int
        f.argtypes = [ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_void_p]
    lib.pearl_hbm_fill.restype = ctypes.c_int
    lib.pearl_hbm_fill.argtypes = [ctypes.c_void_p, ctypes.c_size_t, ctypes.c_uint32, ctypes.c_void_p]
    _lib = lib
    return lib


def set_kernel_events(before: Optional[int], after: Optional[int]) -> None:
    """Record raw hipEvent_t handles around the next calls' main kernel (None, None clears)."""
    load().pearl_set_kernel_events(before, after)


def _status_name(st: int) -> str:
    try:
        return load().pearl_status_str(st).decode()
    except Exception:
        return str(st)


def last_error() -> str:
    return load().pearl_last_error().decode()


def abi_version() -> int:
    return int(load().pearl_abi_version())


def _check(st: int, func: str) -> None:
    if st != PEARL_OK:
        raise PearlError(st, func, last_error())


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _need(t: torch.Tensor, name: str, dtype: torch.dtype) -> None:
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a torch.Tensor" % name)
    if t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if not t.is_cuda:
        raise ValueError("%s must be on the GPU" % name)
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)


# The raw handle of torch's current stream: building the Stream object that
# torch.cuda.current_stream() returns takes 2.7 us, a fifth of a small decode step's host time.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


# The current device, without the check of torch.cuda.current_device() for a context, which the tensors have (0.1 us).
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _stream() -> int:
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


def make_shape(num_q_heads: int, k_pool: torch.Tensor) -> KvShape:
    if k_pool.dim() != 4:
        raise ValueError("pools must be [num_pages][num_kv_heads][page_size][head_dim]")
    n, hkv, ps, d = k_pool.shape
    return KvShape(int(num_q_heads), int(hkv), int(d), int(ps), int(n))


def make_desc(block_table: torch.Tensor, ctx_lens: torch.Tensor, cu_q_lens: Optional[torch.Tensor],
              total_q: int, max_q_len: int, max_kv_len: int, need=_need) -> SeqDesc:
    need(block_table, "block_table", torch.int32)
    need(ctx_lens, "ctx_lens", torch.int32)
    table = block_table.shape
    if len(table) != 2:
        raise ValueError("block_table must be [batch][bt_stride]")
    batch = int(ctx_lens.shape[0])
    if table[0] != batch:
        raise ValueError("block_table rows (%d) != batch (%d)" % (table[0], batch))
    if cu_q_lens is not None:
        need(cu_q_lens, "cu_q_lens", torch.int32)
        if cu_q_lens.shape[0] != batch + 1:
            raise ValueError("cu_q_lens must have batch+1 entries")
    return SeqDesc(block_table.data_ptr(), int(table[1]), ctx_lens.data_ptr(),
                   _ptr(cu_q_lens), batch, int(total_q), int(max_q_len), int(max_kv_len))


def workspace_bytes(num_q_heads: int, k_pool: torch.Tensor, desc: SeqDesc) -> int:
    shape = make_shape(num_q_heads, k_pool)
    n = load().pearl_attn_workspace_bytes(ctypes.byref(shape), ctypes.byref(desc))
    if n == 0:
        raise PearlError(1, "pearl_attn_workspace_bytes", last_error())
    return int(n)


def kv_append(k_new: torch.Tensor, v_new: torch.Tensor, k_pool: torch.Tensor, v_pool: torch.Tensor,
              block_table: torch.Tensor, ctx_lens: torch.Tensor, cu_q_lens: Optional[torch.Tensor],
              max_q_len: int, max_kv_len: int) -> None:
    """Scatter new K/V rows [total_q][H_kv][d] into the pools (pearl_kv_append)."""
    for t, n in ((k_new, "k_new"), (v_new, "v_new"), (k_pool, "k_pool"), (v_pool, "v_pool")):
        _need(t, n, torch.bfloat16)
    desc = make_desc(block_table, ctx_lens, cu_q_lens, int(k_new.shape[0]), max_q_len, max_kv_len)
    shape = make_shape(k_pool.shape[1], k_pool)   # H_q is not used by the append
    st = load().pearl_kv_append(ctypes.byref(shape), ctypes.byref(desc), k_new.data_ptr(),
                                v_new.data_ptr(), k_pool.data_ptr(), v_pool.data_ptr(), _stream())
    _check(st, "pearl_kv_append")


def kv_pack(k_pool: torch.Tensor, v_pool: torch.Tensor, block_table: torch.Tensor, ctx_lens: torch.Tensor,
            cu_q_lens: Optional[torch.Tensor], total: int, max_q_len: int, max_kv_len: int,
            out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Gather token ranges [ctx_lens[b], ctx_lens[b] + n_b) of every sequence out of the pools into
    a transfer buffer bf16 [2][total][H_kv][d] (pearl_kv_pack)."""
    for t, n in ((k_pool, "k_pool"), (v_pool, "v_pool")):
        _need(t, n, torch.bfloat16)
    H_kv, d = int(k_pool.shape[1]), int(k_pool.shape[3])
    if out is None:
        out = torch.empty((2, total, H_kv, d), dtype=torch.bfloat16, device=k_pool.device)
    _need(out, "out", torch.bfloat16)
    if tuple(out.shape) != (2, total, H_kv, d):
        raise ValueError("out must have shape (2, %d, %d, %d)" % (total, H_kv, d))
    desc = make_desc(block_table, ctx_lens, cu_q_lens, total, max_q_len, max_kv_len)
    shape = make_shape(H_kv, k_pool)
    st = load().pearl_kv_pack(ctypes.byref(shape), ctypes.byref(desc), k_pool.data_ptr(), v_pool.data_ptr(),
                              out.data_ptr(), _stream())
    _check(st, "pearl_kv_pack")
    return out


def kv_unpack(buf: torch.Tensor, k_pool: torch.Tensor, v_pool: torch.Tensor, block_table: torch.Tensor,
              ctx_lens: torch.Tensor, cu_q_lens: Optional[torch.Tensor], max_q_len: int,
              max_kv_len: int) -> None:
    """Scatter a transfer buffer bf16 [2][total][H_kv][d] into the pools at positions
    ctx_lens[b] + t through this pool's block table (pearl_kv_unpack)."""
    for t, n in ((buf, "buf"), (k_pool, "k_pool"), (v_pool, "v_pool")):
        _need(t, n, torch.bfloat16)
    if buf.dim() != 4 or buf.shape[0] != 2:
        raise ValueError("buf must have shape (2, total, H_kv, d)")
    desc = make_desc(block_table, ctx_lens, cu_q_lens, int(buf.shape[1]), max_q_len, max_kv_len)
    shape = make_shape(k_pool.shape[1], k_pool)
    st = load().pearl_kv_unpack(ctypes.byref(shape), ctypes.byref(desc), buf.data_ptr(), k_pool.data_ptr(),
                                v_pool.data_ptr(), _stream())
    _check(st, "pearl_kv_unpack")


def _attention(fname: str, q: torch.Tensor, k_pool: torch.Tensor, v_pool: torch.Tensor,
               block_table: torch.Tensor, ctx_lens: torch.Tensor, cu_q_lens: Optional[torch.Tensor],
               max_q_len: int, max_kv_len: int, scale: Optional[float], return_lse: bool,
               out: Optional[torch.Tensor], lse: Optional[torch.Tensor],
               workspace: Optional[torch.Tensor]):
    _need(q, "q", torch.bfloat16)
    _need(k_pool, "k_pool", torch.bfloat16)
    _need(v_pool, "v_pool", torch.bfloat16)
    if q.dim() != 3:
        raise ValueError("q must be [total_q][num_q_heads][head_dim]")
    total_q, H_q, d = q.shape
    desc = make_desc(block_table, ctx_lens, cu_q_lens, total_q, max_q_len, max_kv_len)
    shape = make_shape(H_q, k_pool)
    if out is None:
        out = torch.empty_like(q)
    _need(out, "out", torch.bfloat16)
    if return_lse and lse is None:
        lse = torch.empty((total_q, H_q), dtype=torch.float32, device=q.device)
    if lse is not None:
        _need(lse, "lse", torch.float32)
    if workspace is None:
        nbytes = load().pearl_attn_workspace_bytes(ctypes.byref(shape), ctypes.byref(desc))
        if nbytes == 0:
            raise PearlError(1, "pearl_attn_workspace_bytes", last_error())
        workspace = torch.empty(nbytes, dtype=torch.uint8, device=q.device)
    else:
        _need(workspace, "workspace", torch.uint8)   # the library checks its size
    if scale is None:
        scale = 1.0 / float(d) ** 0.5
    st = getattr(load(), fname)(ctypes.byref(shape), ctypes.byref(desc), q.data_ptr(),
                                k_pool.data_ptr(), v_pool.data_ptr(), float(scale), out.data_ptr(),
                                _ptr(lse), workspace.data_ptr(), workspace.numel(), _stream())
    _check(st, fname)
    return (out, lse) if (return_lse or lse is not None) else out


def prefill_append(q, k_pool, v_pool, block_table, ctx_lens, cu_q_lens, max_q_len, max_kv_len,
                   scale=None, return_lse=False, out=None, lse=None, workspace=None):
    """Causal prefill-append attention of each sequence's new tokens (pearl_attn_prefill_append)."""
    return _attention("pearl_attn_prefill_append", q, k_pool, v_pool, block_table, ctx_lens, cu_q_lens,
                      max_q_len, max_kv_len, scale, return_lse, out, lse, workspace)


def decode(q, k_pool, v_pool, block_table, ctx_lens, max_kv_len, scale=None, return_lse=False,
           out=None, lse=None, workspace=None):
    """Single-token decode for every sequence (pearl_attn_decode); q is [batch][H_q][d]."""
    return _attention("pearl_attn_decode", q, k_pool, v_pool, block_table, ctx_lens, None,
                      1, max_kv_len, scale, return_lse, out, lse, workspace)


def decode_append(q, k_new, v_new, k_pool, v_pool, block_table, ctx_lens, max_kv_len, scale=None,
                  return_lse=False, out=None, lse=None, workspace=None):
    """One decode step with its append (pearl_attn_decode_append): k_new / v_new [batch][H_kv][d]
    are written at position ctx_lens[b] of every sequence, which then attends over ctx_lens[b] + 1
    keys; q is [batch][H_q][d]."""
    for t, n in ((q, "q"), (k_new, "k_new"), (v_new, "v_new"), (k_pool, "k_pool"), (v_pool, "v_pool")):
        _need(t, n, torch.bfloat16)
    if q.dim() != 3:
        raise ValueError("q must be [batch][num_q_heads][head_dim]")
    batch, H_q, d = q.shape
    if tuple(k_new.shape) != (batch, k_pool.shape[1], d) or tuple(v_new.shape) != tuple(k_new.shape):
        raise ValueError("k_new and v_new must be [batch][num_kv_heads][head_dim]")
    desc = make_desc(block_table, ctx_lens, None, batch, 1, max_kv_len)
    shape = make_shape(H_q, k_pool)
    if out is None:
        out = torch.empty_like(q)
    _need(out, "out", torch.bfloat16)
    if return_lse and lse is None:
        lse = torch.empty((batch, H_q), dtype=torch.float32, device=q.device)
    if lse is not None:
        _need(lse, "lse", torch.float32)
    if workspace is None:
        nbytes = load().pearl_attn_workspace_bytes(ctypes.byref(shape), ctypes.byref(desc))
        if nbytes == 0:
            raise PearlError(1, "pearl_attn_workspace_bytes", last_error())
        workspace = torch.empty(nbytes, dtype=torch.uint8, device=q.device)
    else:
        _need(workspace, "workspace", torch.uint8)
    if scale is None:
        scale = 1.0 / float(d) ** 0.5
    st = load().pearl_attn_decode_append(ctypes.byref(shape), ctypes.byref(desc), q.data_ptr(), k_new.data_ptr(),
                                         v_new.data_ptr(), k_pool.data_ptr(), v_pool.data_ptr(), float(scale),
                                         out.data_ptr(), _ptr(lse), workspace.data_ptr(), workspace.numel(),
                                         _stream())
    _check(st, "pearl_attn_decode_append")
    return (out, lse) if (return_lse or lse is not None) else out


def decode_static(q, k_pool, v_pool, block_table, ctx_lens, max_kv_len, scale=None, return_lse=False,
                  out=None, lse=None):
    """Single-token decode with the library's static per-GPU workspace (pearl_attn_decode_static):
    no device memory is allocated by the call (out and lse are allocated here only when not
    given)."""
    for t, n in ((q, "q"), (k_pool, "k_pool"), (v_pool, "v_pool")):
        _need(t, n, torch.bfloat16)
    if q.dim() != 3:
        raise ValueError("q must be [batch][num_q_heads][head_dim]")
    batch, H_q, d = q.shape
    desc = make_desc(block_table, ctx_lens, None, batch, 1, max_kv_len)
    shape = make_shape(H_q, k_pool)
    if out is None:
        out = torch.empty_like(q)
    _need(out, "out", torch.bfloat16)
    if return_lse and lse is None:
        lse = torch.empty((batch, H_q), dtype=torch.float32, device=q.device)
    if lse is not None:
        _need(lse, "lse", torch.float32)
    if scale is None:
        scale = 1.0 / float(d) ** 0.5
    st = load().pearl_attn_decode_static(ctypes.byref(shape), ctypes.byref(desc), q.data_ptr(), k_pool.data_ptr(),
                                         v_pool.data_ptr(), float(scale), out.data_ptr(), _ptr(lse), _stream())
    _check(st, "pearl_attn_decode_static")
    return (out, lse) if (return_lse or lse is not None) else out


def decode_static_max_bytes() -> int:
    return int(load().pearl_attn_decode_static_max_bytes())


def mixed(q, k_pool, v_pool, block_table, ctx_lens, cu_q_lens, max_q_len, max_kv_len, scale=None,
          return_lse=False, out=None, lse=None, workspace=None):
    """Colocated prefill chunks and decodes in one attention launch (pearl_attn_mixed)."""
    return _attention("pearl_attn_mixed", q, k_pool, v_pool, block_table, ctx_lens, cu_q_lens,
                      max_q_len, max_kv_len, scale, return_lse, out, lse, workspace)


# ------------------------------------------------------------------------------------------------
# KV cache in MX blocks (4 or 8 bits an element)
# ------------------------------------------------------------------------------------------------

MXFP4, MXFP8 = 4, 8
_MX_BLOCKS = {}                                     # block bytes -> (head_dim, format)


def mx_block_bytes(head_dim: int, fmt: int) -> int:
    """Bytes of the block of one (page, kv-head) in a cache of MX blocks (pearl_mx_block_bytes)."""
    n = int(load().pearl_mx_block_bytes(int(head_dim), int(fmt)))
    if n == 0:
        raise PearlError(2, "pearl_mx_block_bytes", last_error())
    return n


def mx_cache(num_pages: int, num_kv_heads: int, head_dim: int, fmt: int, device="cuda") -> torch.Tensor:
    """A cache of MX blocks, zeroed: uint8 [num_pages][num_kv_heads][mx_block_bytes(head_dim, fmt)], fmt
    MXFP4 or MXFP8.  head_dim and format follow from the block's size, so the calls below take the
    cache alone."""
    return torch.zeros((num_pages, num_kv_heads, mx_block_bytes(head_dim, fmt)), dtype=torch.uint8, device=device)


@functools.lru_cache(maxsize=256)
def _mx_geometry(num_q_heads: Optional[int], cache_shape: Tuple[int, int, int]):
    """(KvShape, format, a reference to the shape for the library) of a cache [num_pages][H_kv][block]."""
    if not _MX_BLOCKS:
        _MX_BLOCKS.update({mx_block_bytes(d, f): (d, f) for d in (64, 128) for f in (MXFP4, MXFP8)})
    if len(cache_shape) != 3 or cache_shape[2] not in _MX_BLOCKS:
        raise ValueError("cache must be [num_pages][num_kv_heads][mx_block_bytes(head_dim, fmt)]")
    d, fmt = _MX_BLOCKS[cache_shape[2]]
    shape = KvShape(cache_shape[1] if num_q_heads is None else num_q_heads, cache_shape[1], d, PAGE_SIZE, cache_shape[0])
    shape.row = (cache_shape[1], d)                 # of the rows bf16 [tokens][num_kv_heads][head_dim]
    return shape, fmt, ctypes.byref(shape)


class _MxCall:
    """What the calls on a cache of MX blocks have in common: its geometry (num_q_heads None: as many as kv-heads,
    for calls that have no queries), and that every tensor is on the current device, where the library launches."""

    def __init__(self, cache: torch.Tensor, num_q_heads: Optional[int] = None):
        _need(cache, "cache", torch.uint8)
        shape, self.fmt, self.ref = _mx_geometry(num_q_heads, tuple(cache.shape))
        self.row = shape.row
        self.dev = cache.get_device()
        if self.dev != _current_device():
            raise ValueError("cache is on cuda:%d, the current device is cuda:%d" % (self.dev, _current_device()))

    def need(self, t: torch.Tensor, name: str, dtype: torch.dtype) -> None:
        if not (isinstance(t, torch.Tensor) and t.dtype is dtype and t.get_device() == self.dev and t.is_contiguous()):
            _need(t, name, dtype)
            raise ValueError("%s must be on the cache's device (cuda:%d), got %s" % (name, self.dev, t.device))

    def stream(self) -> int:
        return _stream() if _raw_stream is None else _raw_stream(self.dev)


def kv_append_mx(k_new: torch.Tensor, v_new: torch.Tensor, cache: torch.Tensor, block_table: torch.Tensor,
                 ctx_lens: torch.Tensor, cu_q_lens: Optional[torch.Tensor], max_q_len: int, max_kv_len: int) -> None:
    """Quantise new K/V rows bf16 [total_q][H_kv][d] into their slots of a cache of MX blocks
    (pearl_kv_append_mx)."""
    if getattr(k_new, "dtype", None) != torch.bfloat16:
        _need(k_new, "k_new", torch.bfloat16)
    c = _MxCall(cache)
    c.need(k_new, "k_new", torch.bfloat16)
    c.need(v_new, "v_new", torch.bfloat16)
    rows = k_new.shape
    if rows[1:] != c.row or v_new.shape != rows:
        raise ValueError("k_new and v_new must be [total_q][%d][%d]" % c.row)
    total = rows[0]
    desc = make_desc(block_table, ctx_lens, cu_q_lens, total, max_q_len, max_kv_len, c.need)
    st = load().pearl_kv_append_mx(c.ref, ctypes.byref(desc), c.fmt, k_new.data_ptr(), v_new.data_ptr(),
                                   cache.data_ptr(), c.stream())
    _check(st, "pearl_kv_append_mx")


def kv_pack_mx(cache: torch.Tensor, block_table: torch.Tensor, ctx_lens: torch.Tensor,
               cu_q_lens: Optional[torch.Tensor], total: int, max_q_len: int, max_kv_len: int,
               out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Read token ranges [ctx_lens[b], ctx_lens[b] + n_b) of every sequence back out of a cache of MX
    blocks, as bf16 [2][total][H_kv][d] (pearl_kv_pack_mx)."""
    c = _MxCall(cache)
    want = (2, int(total)) + c.row
    if out is None:
        out = torch.empty(want, dtype=torch.bfloat16, device=cache.device)
    else:
        c.need(out, "out", torch.bfloat16)
        if out.shape != want:
            raise ValueError("out must have shape %s" % (want,))
    desc = make_desc(block_table, ctx_lens, cu_q_lens, total, max_q_len, max_kv_len, c.need)
    st = load().pearl_kv_pack_mx(c.ref, ctypes.byref(desc), c.fmt, cache.data_ptr(), out.data_ptr(), c.stream())
    _check(st, "pearl_kv_pack_mx")
    return out


def workspace_bytes_mx(num_q_heads: int, cache: torch.Tensor, desc: SeqDesc) -> int:
    """Bytes of workspace that the attention calls over this cache need (pearl_attn_workspace_bytes)."""
    _need(cache, "cache", torch.uint8)
    n = load().pearl_attn_workspace_bytes(_mx_geometry(int(num_q_heads), tuple(cache.shape))[2], ctypes.byref(desc))
    if n == 0:
        raise PearlError(1, "pearl_attn_workspace_bytes", last_error())
    return int(n)


def _attention_mx(fname: str, q: torch.Tensor, new, cache: torch.Tensor, block_table: torch.Tensor,
                  ctx_lens: torch.Tensor, cu_q_lens: Optional[torch.Tensor], max_q_len: int, max_kv_len: int,
                  scale: Optional[float], return_lse: bool, out: Optional[torch.Tensor], lse: Optional[torch.Tensor],
                  workspace: Optional[torch.Tensor]):
    _need(q, "q", torch.bfloat16)
    if q.dim() != 3:
        raise ValueError("q must be [total_q][num_q_heads][head_dim]")
    total_q, H_q, d = q.shape
    c = _MxCall(cache, H_q)
    c.need(q, "q", torch.bfloat16)
    if d != c.row[1]:
        raise ValueError("q has head_dim %d, the cache %d" % (d, c.row[1]))
    for t, n in zip(new, ("k_new", "v_new")):
        c.need(t, n, torch.bfloat16)
        if t.shape != (total_q,) + c.row:
            raise ValueError("k_new and v_new must be [batch][num_kv_heads][head_dim]")
    desc = make_desc(block_table, ctx_lens, cu_q_lens, total_q, max_q_len, max_kv_len, c.need)
    if out is None:
        out = torch.empty_like(q)
    else:
        c.need(out, "out", torch.bfloat16)
        if out.shape != q.shape:
            raise ValueError("out must have q's shape")
    if lse is not None:
        c.need(lse, "lse", torch.float32)
        if lse.shape != (total_q, H_q):
            raise ValueError("lse must be [total_q][num_q_heads]")
    elif return_lse:
        lse = torch.empty((total_q, H_q), dtype=torch.float32, device=q.device)
    if workspace is None:
        workspace = torch.empty(workspace_bytes_mx(H_q, cache, desc), dtype=torch.uint8, device=q.device)
    else:
        c.need(workspace, "workspace", torch.uint8)  # the library checks its size
    if scale is None:
        scale = 1.0 / float(d) ** 0.5
    st = getattr(load(), fname)(c.ref, ctypes.byref(desc), c.fmt, q.data_ptr(), *[t.data_ptr() for t in new],
                                cache.data_ptr(), float(scale), out.data_ptr(), _ptr(lse), workspace.data_ptr(),
                                workspace.numel(), c.stream())
    _check(st, fname)
    return (out, lse) if lse is not None else out


def decode_mx(q, cache, block_table, ctx_lens, max_kv_len, scale=None, return_lse=False, out=None, lse=None,
              workspace=None):
    """Single-token decode over a cache of MX blocks (pearl_attn_decode_mx); q is [batch][H_q][d]."""
    return _attention_mx("pearl_attn_decode_mx", q, (), cache, block_table, ctx_lens, None, 1, max_kv_len, scale,
                         return_lse, out, lse, workspace)


def decode_append_mx(q, k_new, v_new, cache, block_table, ctx_lens, max_kv_len, scale=None, return_lse=False, out=None,
                     lse=None, workspace=None):
    """One decode step with its append over a cache of MX blocks (pearl_attn_decode_append_mx): k_new / v_new
    [batch][H_kv][d] are quantised into position ctx_lens[b] of every sequence, which then attends over
    ctx_lens[b] + 1 keys."""
    return _attention_mx("pearl_attn_decode_append_mx", q, (k_new, v_new), cache, block_table, ctx_lens, None, 1,
                         max_kv_len, scale, return_lse, out, lse, workspace)


def prefill_append_mx(q, cache, block_table, ctx_lens, cu_q_lens, max_q_len, max_kv_len, scale=None, return_lse=False,
                      out=None, lse=None, workspace=None):
    """Causal prefill-append attention over a cache of MX blocks that holds the new tokens
    (pearl_attn_prefill_append_mx)."""
    return _attention_mx("pearl_attn_prefill_append_mx", q, (), cache, block_table, ctx_lens, cu_q_lens, max_q_len,
                         max_kv_len, scale, return_lse, out, lse, workspace)


# ------------------------------------------------------------------------------------------------
# Rotary position embedding
# ------------------------------------------------------------------------------------------------

class Rope:
    """The rotation of a layer's queries and keys (pearl_rope): inv_freq fp32 [rotary_dim / 2] radians a position; pairs of
    channels (n, n + rotary_dim / 2), or (2n, 2n + 1) if interleaved; cosines and sines times `factor`; q_weight and k_weight
    bf16 [head_dim], or None, of the RMS norm that comes before (latent_append: k_weight [latent_dim], q_weight None).  Keeps its tensors; build it once a layer."""

    def __init__(self, inv_freq: torch.Tensor, interleaved: bool = False, factor: float = 1.0,
                 q_weight: Optional[torch.Tensor] = None, k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6):
        _need(inv_freq, "inv_freq", torch.float32)
        if inv_freq.dim() != 1:
            raise ValueError("inv_freq must be [rotary_dim / 2]")
        for t, n in ((q_weight, "q_weight"), (k_weight, "k_weight")):
            if t is not None:
                _need(t, n, torch.bfloat16)
                if t.dim() != 1 or t.get_device() != inv_freq.get_device():
                    raise ValueError("%s must be one row on inv_freq's device" % n)
        self.inv_freq, self.q_weight, self.k_weight = inv_freq, q_weight, k_weight
        self.dev = inv_freq.get_device()
        self.q_channels = None if q_weight is None else q_weight.shape[0]
        self.k_channels = None if k_weight is None else k_weight.shape[0]
        self.desc = RopeDesc(inv_freq.data_ptr(), 2 * inv_freq.shape[0], int(bool(interleaved)), float(factor), float(eps),
                             _ptr(q_weight), _ptr(k_weight))
        self.ref = ctypes.byref(self.desc)

    def weights(self, q: Optional[int], k: int) -> None:
        """That the norms' weights are of so many channels (q None: queries have none)."""
        if self.q_channels is not None and self.q_channels != q:
            raise ValueError("q_weight has %d channels, %s" % (self.q_channels, "the call takes none" if q is None else "a head %d" % q))
        if self.k_channels is not None and self.k_channels != k:
            raise ValueError("k_weight has %d channels, not %d" % (self.k_channels, k))


def _on(dev: int):
    """What checks a call's tensors: type, contiguity, and that they are on the current device, where the library launches."""
    if dev != _current_device():
        raise ValueError("tensors are on cuda:%d, the current device is cuda:%d" % (dev, _current_device()))

    def need(t: torch.Tensor, name: str, dtype: torch.dtype) -> None:
        if not (isinstance(t, torch.Tensor) and t.dtype is dtype and t.get_device() == dev and t.is_contiguous()):
            _need(t, name, dtype)
            raise ValueError("%s must be on cuda:%d, got %s" % (name, dev, t.device))
    return need


def _bf16_on(t: torch.Tensor, name: str, dev: int) -> None:
    if not isinstance(t, torch.Tensor) or t.dtype is not torch.bfloat16 or t.get_device() != dev:
        _need(t, name, torch.bfloat16)
        raise ValueError("%s must be on cuda:%d, got %s" % (name, dev, t.device))


def _rows(t: torch.Tensor, name: str, dev: int, tokens: Optional[int] = None, heads: Optional[int] = None,
          channels: Optional[int] = None):
    """Of bf16 rows [tokens][heads][channels], of which a token's are contiguous: the sizes, and the elements from a token to the
    next one."""
    _bf16_on(t, name, dev)
    size = t.shape
    if len(size) != 3 or (tokens is not None and size[0] != tokens) or (heads is not None and size[1] != heads) or \
            (channels is not None and size[2] != channels):
        raise ValueError("%s must be [%s]" % (name, "][".join("any" if w is None else str(w) for w in (tokens, heads, channels))))
    n0, n1, n2 = size
    s0, s1, s2 = t.stride()
    if (n2 > 1 and s2 != 1) or (n1 > 1 and s1 != n2):
        raise ValueError("a token's rows of %s must be contiguous" % name)
    return size, s0 if n0 > 1 else n1 * n2


# A shape argument of a call, which the library only reads: building one takes 1 us, as long as a tenth of a small call.
@functools.lru_cache(maxsize=512)
def _kv_shape_ref(*sizes: int):
    return ctypes.byref(KvShape(*sizes))


@functools.lru_cache(maxsize=512)
def _latent_shape_ref(*sizes: int):
    return ctypes.byref(LatentShape(*sizes))


def _stream_on(dev: int) -> int:
    return _stream() if _raw_stream is None else _raw_stream(dev)


def rope_rows(q: torch.Tensor, k_new: torch.Tensor, rope: Rope, ctx_lens: torch.Tensor, cu_q_lens: Optional[torch.Tensor],
              max_q_len: int, q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None):
    """Queries [total_q][H_q][d] and keys [total_q][H_kv][d] normalised and rotated at positions ctx_lens[b] + i
    (pearl_rope_rows); both may be parts of wider rows.  q_out / k_out: contiguous, allocated if not given, q and k_new
    themselves where those are contiguous.  Returns (q_out, k_out)."""
    dev = rope.dev
    need = _on(dev)
    q_size, q_stride = _rows(q, "q", dev)
    total, H_q, d = q_size
    k_size, k_stride = _rows(k_new, "k_new", dev, total, None, d)
    rope.weights(d, d)
    if q_out is None:
        q_out = torch.empty(q_size, dtype=torch.bfloat16, device=q.device)
    if k_out is None:
        k_out = torch.empty(k_size, dtype=torch.bfloat16, device=q.device)
    need(q_out, "q_out", torch.bfloat16)
    need(k_out, "k_out", torch.bfloat16)
    if q_out.shape != q_size:
        raise ValueError("q_out must have shape %s" % (tuple(q_size),))
    if k_out.shape != k_size:
        raise ValueError("k_out must have shape %s" % (tuple(k_size),))
    desc = _lens_desc(ctx_lens, cu_q_lens, total, max_q_len, need)
    st = load().pearl_rope_rows(_kv_shape_ref(H_q, k_size[1], d, PAGE_SIZE, 1), ctypes.byref(desc), rope.ref, q.data_ptr(), q_stride,
                                k_new.data_ptr(), k_stride, q_out.data_ptr(), k_out.data_ptr(), _stream_on(dev))
    _check(st, "pearl_rope_rows")
    return q_out, k_out


def _lens_desc(ctx_lens: torch.Tensor, cu_q_lens: Optional[torch.Tensor], total_q: int, max_q_len: int, need) -> SeqDesc:
    """A batch of which no page is read or written."""
    need(ctx_lens, "ctx_lens", torch.int32)
    batch = int(ctx_lens.shape[0])
    if cu_q_lens is not None:
        need(cu_q_lens, "cu_q_lens", torch.int32)
        if cu_q_lens.shape[0] != batch + 1:
            raise ValueError("cu_q_lens must have batch+1 entries")
    return SeqDesc(None, 0, ctx_lens.data_ptr(), _ptr(cu_q_lens), batch, int(total_q), int(max_q_len), 0)


def kv_append_rope(q: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor, rope: Rope, k_pool: torch.Tensor,
                   v_pool: torch.Tensor, block_table: torch.Tensor, ctx_lens: torch.Tensor,
                   cu_q_lens: Optional[torch.Tensor], max_q_len: int, max_kv_len: int,
                   q_out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """rope_rows with k_new (rotated) and v_new going into the pools (pearl_kv_append_rope); returns q_out."""
    dev = rope.dev
    need = _on(dev)
    need(k_pool, "k_pool", torch.bfloat16)
    need(v_pool, "v_pool", torch.bfloat16)
    pool = k_pool.shape
    if len(pool) != 4:
        raise ValueError("pools must be [num_pages][num_kv_heads][page_size][head_dim]")
    if v_pool.shape != pool:
        raise ValueError("k_pool and v_pool must have one shape")
    pages, H_kv, page_size, d = pool
    q_size, q_stride = _rows(q, "q", dev, None, None, d)
    total = q_size[0]
    _, k_stride = _rows(k_new, "k_new", dev, total, H_kv, d)
    _, v_stride = _rows(v_new, "v_new", dev, total, H_kv, d)
    rope.weights(d, d)
    if q_out is None:
        q_out = torch.empty(q_size, dtype=torch.bfloat16, device=q.device)
    need(q_out, "q_out", torch.bfloat16)
    if q_out.shape != q_size:
        raise ValueError("q_out must have shape %s" % (tuple(q_size),))
    desc = make_desc(block_table, ctx_lens, cu_q_lens, total, max_q_len, max_kv_len, need)
    st = load().pearl_kv_append_rope(_kv_shape_ref(q_size[1], H_kv, d, page_size, pages), ctypes.byref(desc), rope.ref, q.data_ptr(),
                                     q_stride, k_new.data_ptr(), k_stride, v_new.data_ptr(), v_stride, q_out.data_ptr(),
                                     k_pool.data_ptr(), v_pool.data_ptr(), _stream_on(dev))
    _check(st, "pearl_kv_append_rope")
    return q_out


# ------------------------------------------------------------------------------------------------
# Attention over a paged cache of latent vectors
# ------------------------------------------------------------------------------------------------

_LATENT_DIMS = {576: (512, 64), 288: (256, 32)}     # row width -> (latent_dim, rope_dim)


def latent_cache(num_pages: int, latent_dim: int, rope_dim: int, device="cuda") -> torch.Tensor:
    """A cache of latent rows, zeroed: bf16 [num_pages][16][latent_dim + rope_dim], (512, 64) or (256, 32).  Both dims follow from
    the row's width, so the calls below take the cache alone."""
    if _LATENT_DIMS.get(latent_dim + rope_dim) != (latent_dim, rope_dim):
        raise ValueError("(latent_dim, rope_dim) must be (512, 64) or (256, 32)")
    return torch.zeros((num_pages, PAGE_SIZE, latent_dim + rope_dim), dtype=torch.bfloat16, device=device)


def _latent_sizes(num_q_heads: int, cache: torch.Tensor) -> Tuple[int, int, int, int, int]:
    size = cache.shape
    if len(size) != 3 or size[1] != PAGE_SIZE or size[2] not in _LATENT_DIMS:
        raise ValueError("cache must be [num_pages][16][latent_dim + rope_dim], (512, 64) or (256, 32)")
    dc, dr = _LATENT_DIMS[size[2]]
    return num_q_heads, dc, dr, PAGE_SIZE, size[0]


def latent_append(q_rope: torch.Tensor, rows_new: torch.Tensor, rope: Rope, q: torch.Tensor, cache: torch.Tensor,
                  block_table: torch.Tensor, ctx_lens: torch.Tensor, cu_q_lens: Optional[torch.Tensor], max_q_len: int,
                  max_kv_len: int) -> None:
    """New latent rows [total_q][latent_dim + rope_dim] into the cache, the latent part normalised (rope.k_weight), the
    rest rotated; q_rope [total_q][H][rope_dim], rotated, into the last channels of the absorbed queries q
    [total_q][H][latent_dim + rope_dim] (pearl_latent_append).  rows_new may be a part of wider rows, q_rope of wider heads, or the
    tails of q themselves."""
    dev = rope.dev
    need = _on(dev)
    need(cache, "cache", torch.bfloat16)
    need(q, "q", torch.bfloat16)
    q_size = q.shape
    if len(q_size) != 3:
        raise ValueError("q must be [total_q][num_q_heads][latent_dim + rope_dim]")
    total, H, width = q_size
    sizes = _latent_sizes(H, cache)
    _, dc, dr, _, _ = sizes
    if width != dc + dr:
        raise ValueError("q has %d channels, the cache %d" % (width, dc + dr))
    _bf16_on(rows_new, "rows_new", dev)
    if rows_new.shape != (total, width):
        raise ValueError("rows_new must be [%d][%d]" % (total, width))
    rows_stride, by_channel = rows_new.stride()
    if by_channel != 1:
        raise ValueError("the rows of rows_new must be contiguous")
    if total <= 1:
        rows_stride = width
    _bf16_on(q_rope, "q_rope", dev)
    if q_rope.shape != (total, H, dr):
        raise ValueError("q_rope must be [%d][%d][%d]" % (total, H, dr))
    by_token, by_head, by_channel = q_rope.stride()
    if by_channel != 1:
        raise ValueError("the heads of q_rope must be contiguous")
    if H == 1:
        by_head = by_token
    elif total > 1 and by_token != H * by_head:
        raise ValueError("q_rope's heads must be evenly spaced, a token's last to the next one's first alike")
    if total * H <= 1:
        by_head = dr
    rope.weights(None, dc)
    desc = make_desc(block_table, ctx_lens, cu_q_lens, total, max_q_len, max_kv_len, need)
    st = load().pearl_latent_append(_latent_shape_ref(*sizes), ctypes.byref(desc), rope.ref, q_rope.data_ptr(), by_head,
                                    rows_new.data_ptr(), rows_stride, q.data_ptr(), cache.data_ptr(), _stream_on(dev))
    _check(st, "pearl_latent_append")


def workspace_bytes_latent(num_q_heads: int, cache: torch.Tensor, desc: SeqDesc) -> int:
    """Bytes of workspace that the attention calls over this cache need (pearl_latent_workspace_bytes)."""
    n = load().pearl_latent_workspace_bytes(_latent_shape_ref(*_latent_sizes(int(num_q_heads), cache)), ctypes.byref(desc))
    if n == 0:
        raise PearlError(1, "pearl_latent_workspace_bytes", last_error())
    return int(n)


def _attention_latent(fname: str, q: torch.Tensor, cache: torch.Tensor, block_table: torch.Tensor, ctx_lens: torch.Tensor,
                      cu_q_lens: Optional[torch.Tensor], max_q_len: int, max_kv_len: int, scale: float, return_lse: bool,
                      out: Optional[torch.Tensor], lse: Optional[torch.Tensor], workspace: Optional[torch.Tensor]):
    _need(cache, "cache", torch.bfloat16)
    dev = cache.get_device()
    need = _on(dev)
    need(q, "q", torch.bfloat16)
    q_size = q.shape
    if len(q_size) != 3:
        raise ValueError("q must be [total_q][num_q_heads][latent_dim + rope_dim]")
    total, H, width = q_size
    sizes = _latent_sizes(H, cache)
    _, dc, dr, _, _ = sizes
    if width != dc + dr:
        raise ValueError("q has %d channels, the cache %d" % (width, dc + dr))
    desc = make_desc(block_table, ctx_lens, cu_q_lens, total, max_q_len, max_kv_len, need)
    want = (total, H, dc)
    if out is None:
        out = torch.empty(want, dtype=torch.bfloat16, device=q.device)
    else:
        need(out, "out", torch.bfloat16)
        if out.shape != want:
            raise ValueError("out must have shape %s" % (want,))
    if lse is not None:
        need(lse, "lse", torch.float32)
        if lse.shape != (total, H):
            raise ValueError("lse must be [total_q][num_q_heads]")
    elif return_lse:
        lse = torch.empty((total, H), dtype=torch.float32, device=q.device)
    if workspace is None:
        workspace = torch.empty(workspace_bytes_latent(H, cache, desc), dtype=torch.uint8, device=q.device)
    else:
        need(workspace, "workspace", torch.uint8)    # the library checks its size
    st = getattr(load(), fname)(_latent_shape_ref(*sizes), ctypes.byref(desc), q.data_ptr(), cache.data_ptr(), float(scale),
                                out.data_ptr(), _ptr(lse), workspace.data_ptr(), workspace.numel(), _stream_on(dev))
    _check(st, fname)
    return (out, lse) if lse is not None else out


def latent_decode(q, cache, block_table, ctx_lens, max_kv_len, scale, return_lse=False, out=None, lse=None, workspace=None):
    """Single-token decode over a cache of latent rows (pearl_attn_latent_decode): q [batch][H][latent_dim + rope_dim] absorbed
    queries, out [batch][H][latent_dim].  `scale` has no default: it goes by the head's width before absorption."""
    return _attention_latent("pearl_attn_latent_decode", q, cache, block_table, ctx_lens, None, 1, max_kv_len, scale, return_lse,
                             out, lse, workspace)


def latent_prefill_append(q, cache, block_table, ctx_lens, cu_q_lens, max_q_len, max_kv_len, scale, return_lse=False, out=None,
                          lse=None, workspace=None):
    """Causal prefill-append attention over a cache of latent rows that holds the new tokens
    (pearl_attn_latent_prefill_append)."""
    return _attention_latent("pearl_attn_latent_prefill_append", q, cache, block_table, ctx_lens, cu_q_lens, max_q_len,
                             max_kv_len, scale, return_lse, out, lse, workspace)


# ------------------------------------------------------------------------------------------------
# measurement tooling (include/pearl_bench.h): bandwidth probes and the cache flush
# ------------------------------------------------------------------------------------------------

def hbm_copy(src: torch.Tensor, dst: torch.Tensor) -> None:
    """dst <- src, byte for byte (both contiguous GPU tensors of the same byte size)."""
    if not (src.is_cuda and dst.is_cuda and src.is_contiguous() and dst.is_contiguous()):
        raise ValueError("hbm_copy needs contiguous GPU tensors")
    n = src.numel() * src.element_size()
    if dst.numel() * dst.element_size() != n:
        raise ValueError("hbm_copy: byte sizes differ")
    _check(load().pearl_hbm_copy(src.data_ptr(), dst.data_ptr(), n, _stream()), "pearl_hbm_copy")


def hbm_read(src: torch.Tensor, sink: torch.Tensor, nontemporal: bool = False) -> None:
    """Stream-read src; `sink` is a 16-byte (or larger) GPU tensor the kernel may overwrite.  Over
    >= 1 GiB the plain read is the cache flush (it leaves no dirty lines behind); nontemporal=True
    is pearl_hbm_read_nt, the faster read mode, which is no flush."""
    if not (src.is_cuda and src.is_contiguous() and sink.is_cuda and sink.numel() * sink.element_size() >= 16):
        raise ValueError("hbm_read needs a contiguous GPU source and a 16-byte GPU sink")
    name = "pearl_hbm_read_nt" if nontemporal else "pearl_hbm_read"
    _check(getattr(load(), name)(src.data_ptr(), src.numel() * src.element_size(), sink.data_ptr(), _stream()),
           name)


def hbm_fill(dst: torch.Tensor, pattern: int = 0) -> None:
    """Write a 32-bit pattern over dst."""
    if not (dst.is_cuda and dst.is_contiguous()):
        raise ValueError("hbm_fill needs a contiguous GPU tensor")
    _check(load().pearl_hbm_fill(dst.data_ptr(), dst.numel() * dst.element_size(), pattern & 0xFFFFFFFF,
                                 _stream()), "pearl_hbm_fill")
