"""MI355X (gfx950) paged-KV attention for multi-turn rollout: kv_append, prefill-append, decode,
colocated mixed batches and KV transfer pack/unpack between pools, a KV cache in MX blocks of 4 or 8
bits an element, rotary position embedding with or without the append, and appends and attention over a
cache of latent vectors, as hand-written HIP kernels behind a C ABI (include/pearl_attn.h, pearl_latent.h).

The Python layer only marshals arguments (see ``binding``); it has no compute fallback."""
from .binding import (  # noqa: F401
    LIB_PATH, MXFP4, MXFP8, PearlError, Rope, abi_version, decode, decode_append, decode_append_mx, decode_mx, kv_append,
    kv_append_mx, kv_pack, kv_pack_mx, kv_unpack, last_error, load, mixed, mx_block_bytes, mx_cache, prefill_append,
    prefill_append_mx, workspace_bytes, workspace_bytes_mx, rope_rows, kv_append_rope, latent_cache, latent_append,
    latent_decode, latent_prefill_append, workspace_bytes_latent,
)

__all__ = ["kv_append", "kv_pack", "kv_unpack", "prefill_append", "decode", "decode_append", "mixed", "workspace_bytes",
           "mx_cache", "mx_block_bytes", "MXFP4", "MXFP8", "kv_append_mx", "kv_pack_mx", "decode_mx",
           "decode_append_mx", "prefill_append_mx", "workspace_bytes_mx", "Rope", "rope_rows", "kv_append_rope",
           "latent_cache", "latent_append", "latent_decode", "latent_prefill_append", "workspace_bytes_latent",
           "abi_version", "last_error", "load", "PearlError", "LIB_PATH"]
