"""MI355X (gfx950) paged-KV attention for multi-turn rollout: kv_append, prefill-append, decode,
colocated mixed batches and KV transfer pack/unpack between pools, and a KV cache in MX blocks of 4 or 8
bits an element, as hand-written HIP kernels behind a C ABI (include/pearl_attn.h).

The Python layer only marshals arguments (see ``binding``); it has no compute fallback."""
from .binding import (  # noqa: F401
    LIB_PATH, MXFP4, MXFP8, PearlError, abi_version, decode, decode_append, decode_append_mx, decode_mx, kv_append,
    kv_append_mx, kv_pack, kv_pack_mx, kv_unpack, last_error, load, mixed, mx_block_bytes, mx_cache, prefill_append,
    prefill_append_mx, workspace_bytes, workspace_bytes_mx,
)

__all__ = ["kv_append", "kv_pack", "kv_unpack", "prefill_append", "decode", "decode_append", "mixed", "workspace_bytes",
           "mx_cache", "mx_block_bytes", "MXFP4", "MXFP8", "kv_append_mx", "kv_pack_mx", "decode_mx",
           "decode_append_mx", "prefill_append_mx", "workspace_bytes_mx", "abi_version", "last_error", "load", "PearlError", "LIB_PATH"]
