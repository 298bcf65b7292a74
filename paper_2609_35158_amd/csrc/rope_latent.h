// Internal interface between the C-ABI host layer (api.cpp) and the gfx950 kernels of rotation, appends with rotation and
// attention over a cache of latent vectors (rope.hip, latent16.hip, latent64.hip).  Not installed; callers use include/pearl_attn.h and
// pearl_latent.h.  Apart from pearl_internal.h, whose bytes the committed counters of the attention kernels are tied to.
#pragma once

#include "pearl_internal.h"

namespace pearl {

// Query heads of an attention call over a cache of latent vectors, at most.
constexpr int kLatentMaxHeads = 128;
// Workgroups of such a call: one a compute unit (a fixed number, which sizes the workspace).
constexpr int kLatentGrid = kPlanComputeUnits;

// Rotary position embedding (rope.hip).
struct RopeArgs {
  const float* inv_freq;
  const uint16_t* q_weight;  // RMS norm weights, or null: none
  const uint16_t* k_weight;
  int rotary_dim;
  int next;                  // pairs (2n, 2n + 1); 0: (n, n + rotary_dim / 2)
  float factor, eps;
};
struct RopeSeqs {
  const int32_t* block_table;
  const int32_t* ctx_lens;
  const int32_t* cu;         // may be null: one token a sequence
  int bt_stride, num_pages, batch, total_q;
};
// Strides are elements from one token's rows to the next one's.
struct RopeRows {
  const uint16_t *q, *k, *v;
  uint16_t *q_out, *k_out, *v_out;  // k_out and v_out: the pools, or k_out the row buffer
  int64_t q_stride, k_stride, v_stride;
  int num_q_heads, num_kv_heads;
};
struct LatentRows {
  const uint16_t *q_rope, *rows;
  uint16_t *q, *cache;
  int64_t q_rope_stride;     // from one head's row to the next one's
  int64_t rows_stride;
  int num_q_heads;
};
hipError_t launch_rope(const RopeArgs& r, const RopeSeqs& seqs, const RopeRows& rows, int head_dim, bool to_pool, hipStream_t stream);
hipError_t launch_latent_append(const RopeArgs& r, const RopeSeqs& seqs, const LatentRows& rows, int latent_dim, int rope_dim,
                                hipStream_t stream);

// Attention over a cache of latent vectors (latent16.hip, latent64.hip).
struct LatentArgs {
  const uint16_t* q;
  const uint16_t* cache;
  const int32_t* block_table;
  const int32_t* ctx_lens;
  const int32_t* cu;         // may be null: one token a sequence
  uint16_t* out;
  float* lse;                // may be null
  int32_t* ws_hdr;
  int4* jobs;                // [kLatentGrid]: cut tiles to be joined
  float* part_o;             // [2 kLatentGrid][tile][latent_dim] unnormalised partial outputs
  float* part_ml;            // [2 kLatentGrid][tile][2] running max (log2 units) and sum
  int bt_stride, num_pages, batch, total_q, max_q_len, max_kv_len;
  int heads;
  unsigned long long per_head;  // 2^35 / heads, rounded up
  int group;                 // workgroups that take neighbouring tiles of one share
  int slope;                 // 128 group * tile / heads
  int min_share_shift;       // a share has 2^this keys, at least
  float scale_log2;
};
// merge: the join of cut tiles, launched after the attention itself.
hipError_t launch_latent(const LatentArgs& a, int latent_dim, int tile, bool merge, hipStream_t stream);
hipError_t launch_latent64(const LatentArgs& a, int latent_dim, hipStream_t stream);

}  // namespace pearl
