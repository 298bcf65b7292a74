"""CPU oracle (test infrastructure only): plain float64 paged-KV attention written from the
definition.  Imported only by tests, the smoke check and the benchmark's CPU baseline."""
from .paged_attention import (  # noqa: F401
    PAGE, attention, attention_scalar_loops, attention_split, attention_unit, bf16_bits_to_f64,
    compare, f64_to_bf16_bits, gather_kv, kv_append, kv_pack, kv_unpack, merge_states, partial_state,
)
from .mx_cache import (  # noqa: F401
    mx_append, mx_block_bytes, mx_element_values, mx_pack, mx_pools, mx_quantise, mx_values,
)
from .rotary import norm_rows, positions, rope_rows, rotate  # noqa: F401
from .latent import latent_attention, latent_rows  # noqa: F401
