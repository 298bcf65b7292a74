// gfx950 kernels of the rotary position embedding: query and key rows normalised per head (RMS norm,
// optional) and rotated by their tokens' positions, on their way into row buffers or, for keys with
// their values, into the paged pools; and the append of latent rows, whose shared key part is rotated.
// (Paper, Background: the context grows by each turn's tokens; a token's position is its place in it.)
//
// Token at position p, channel pair (i, j) of a head, n = 0 .. rotary_dim / 2 - 1 its number:
//   a = p inv_freq[n];   y_i = f (x_i cos a - x_j sin a),   y_j = f (x_j cos a + x_i sin a),
// (i, j) = (n, n + rotary_dim / 2) or (2n, 2n + 1); x = head * rsqrt(mean head^2 + eps) * weight where a
// weight is given.  32 bits throughout, rounded once; the angle is taken in 64 bits, as turns less the nearest whole
// number of them (p inv_freq has up to 49 bits), and goes to the sine and cosine instructions in turns: off by 2^-25 turns.
//
// A lane holds one 16-byte chunk of a row, D / 8 lanes a row, a wave 512 / D rows of one token.  A lane's cosines and
// sines are the same for all of the token's rows, with the norm's weights folded in: y = r (x cw + x' sw), x' the
// pair's other element, which is in the same chunk or comes over from another lane of the row as the raw 16 bytes.
// Bound by HBM where tokens are many (rows in, rows out): 19.4K tokens of 32 + 4 + 4 heads of 128 channels, 397 MB, take 82.5 us with norms and
// append (4.8 TB/s; a copy of as many bytes 74), 18K latent rows with 16 query heads, 115 MB, 30 us.  Where few, by the latency of lengths, page
// id and rows one after the other: 64 tokens 4.1 to 4.4 us, 32 latent rows 3.8.  Tried: the rows' loads before the place is looked up
// (registers for fewer waves: 83 -> 110 us).

#include "rope_latent.h"

namespace pearl {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr int kRopeThreads = 256;
constexpr int kRopeWaves = kRopeThreads / 64;

template <int kCtrl> __device__ __forceinline__ float dpp_add(float x) {
  return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), kCtrl, 0xf, 0xf, false));
}

// The sum over each run of N lanes, the same in all of them.
template <int N> __device__ __forceinline__ float lanes_sum(float x) {
  x = dpp_add<0xB1>(x);                             // lane ^ 1
  x = dpp_add<0x4E>(x);                             // lane ^ 2
  if constexpr (N >= 8) x = dpp_add<0x141>(x);      // mirrored in 8 lanes
  if constexpr (N >= 16) x = dpp_add<0x140>(x);     // mirrored in 16
  if constexpr (N >= 32) {
    const unsigned u = __builtin_bit_cast(unsigned, x);
    const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    x = __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
  }
  if constexpr (N >= 64) {
    const unsigned u = __builtin_bit_cast(unsigned, x);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    x = __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
  }
  return x;
}

__device__ __forceinline__ float low(uint32_t w) { return __builtin_bit_cast(float, w << 16); }
__device__ __forceinline__ float high(uint32_t w) { return __builtin_bit_cast(float, w & 0xffff0000u); }
__device__ __forceinline__ float element(const u32x4& w, int e) { return e & 1 ? high(w[e >> 1]) : low(w[e >> 1]); }
__device__ __forceinline__ u32x4 rounded(const float* y) {
  typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
  bf16x8 v;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = (__bf16)y[e];
  return __builtin_bit_cast(u32x4, v);
}
__device__ __forceinline__ u32x4 load16(const uint16_t* p) { return *reinterpret_cast<const u32x4*>(p); }
__device__ __forceinline__ void store16(uint16_t* p, const u32x4& v) { *reinterpret_cast<u32x4*>(p) = v; }

// A token's row of the call and its place.
struct Token {
  int seq;
  long long pos;
  bool ok;
};

// The sequence that a row belongs to is found by counting, with ballots, the starts that are not behind it: 64 evenly
// spaced ones, then 64 in the gap between two, until there is none.  Rows behind the last sequence have none.
__device__ __forceinline__ Token token_of(int row, const RopeSeqs& s) {
  int b = row;
  long long t = 0;
  if (s.cu) {
    const int lane = threadIdx.x & 63;
    int n = s.batch;
    b = 0;
    while (n > 1) {
      const int gap = (n + 63) / 64, probe = lane * gap;
      const int at = max(__popcll(__ballot(probe < n && s.cu[b + min(probe, n - 1)] <= row)) - 1, 0) * gap;
      b += at;
      n = min(gap, n - at);
    }
    b = __builtin_amdgcn_readfirstlane(b);
    const int start = s.cu[b];
    if (start < 0 || start > row || s.cu[b + 1] <= row) return Token{0, 0, false};
    t = row - start;
  }
  const int ctx = s.ctx_lens[b];
  return Token{b, ctx + t, ctx >= 0};
}

// The slot of the token in a pool, as page * kPage + slot, or -1 where it has none.
__device__ __forceinline__ long long slot_of(const Token& t, const RopeSeqs& s) {
  const long long lp = t.pos / kPage;
  if (lp >= s.bt_stride) return -1;
  const int page = s.block_table[(size_t)t.seq * s.bt_stride + lp];
  return page >= 0 && page < s.num_pages ? (long long)page * kPage + t.pos % kPage : -1;
}

// A lane's part of the rotation of rows of D channels: chunk kc of its row.
template <int D> struct RopeLane {
  static constexpr int kLanes = D / 8;              // of a row
  static constexpr int kRows = 64 / kLanes;         // of a wave
  int kc, sub;                                      // the lane's chunk, and its row of the wave's
  bool turns;                                       // the chunk is rotated
  int other;                                        // byte index of the lane that holds the pairs' other elements
  float c[8], s[8];                                 // y[e] = x[e] c[e] + x'[e] s[e]

  __device__ __forceinline__ RopeLane(const RopeArgs& r, long long pos) {
    const int lane = threadIdx.x & 63;
    kc = lane % kLanes;
    sub = lane / kLanes;
    const int half = r.rotary_dim / 2;
    turns = 8 * kc < r.rotary_dim;
    const bool second = 8 * kc >= half;
    other = 4 * (r.next || !turns ? lane : second ? lane - half / 8 : lane + half / 8);
    const float* freq = r.inv_freq + (!turns ? 0 : r.next ? 4 * kc : 8 * kc - (second ? half : 0));
    auto turn = [&](int n, float& cosine, float& sine) {
      const double a = (double)pos * ((double)freq[n] * 0.15915494309189533577);   // 1 / (2 pi)
      const float x = (float)(a - __builtin_rint(a));
      cosine = r.factor * __builtin_amdgcn_cosf(x);
      sine = r.factor * __builtin_amdgcn_sinf(x);
    };
    if (r.next) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float cosine, sine;
        turn(e, cosine, sine);
        c[2 * e] = c[2 * e + 1] = cosine;
        s[2 * e] = -sine;
        s[2 * e + 1] = sine;
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        turn(e, c[e], s[e]);
        if (!second) s[e] = -s[e];
      }
    }
    if (!turns) {
#pragma unroll
      for (int e = 0; e < 8; ++e) { c[e] = 1.f; s[e] = 0.f; }
    }
  }

  // The pairs' other elements.
  __device__ __forceinline__ u32x4 partner(const u32x4& x, bool next) const {
    u32x4 p;
#pragma unroll
    for (int w = 0; w < 4; ++w)
      p[w] = next ? x[w] >> 16 | x[w] << 16 : (uint32_t)__builtin_amdgcn_ds_bpermute(other, (int)x[w]);
    return p;
  }

  // weights: the norm's, or null; cw, sw: the coefficients with them.
  __device__ __forceinline__ void fold(const uint16_t* weights, bool next, float* cw, float* sw) const {
    u32x4 w = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
    if (weights) w = load16(weights + 8 * kc);
    const u32x4 p = partner(w, next);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      cw[e] = c[e] * element(w, e);
      sw[e] = s[e] * element(p, e);
    }
  }

  __device__ __forceinline__ u32x4 apply(const u32x4& x, bool next, bool norm, float eps, const float* cw, const float* sw) const {
    const u32x4 p = partner(x, next);
    float r = 1.f, y[8];
    if (norm) {
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) sum = fmaf(element(x, e), element(x, e), sum);
      r = rsqrtf(lanes_sum<kLanes>(sum) * (1.f / D) + eps);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      // an unrotated channel takes nothing of another, not even an infinity times 0
      const float v = turns ? fmaf(element(x, e), cw[e], element(p, e) * sw[e]) : element(x, e) * cw[e];
      y[e] = norm ? r * v : v;
    }
    return turns || norm ? rounded(y) : x;
  }
};

// Wave w of a token's `waves` takes groups w, w + waves, .. of RopeLane::kRows rows: queries, then keys, then (into the
// pools) values.
template <int D, bool kToPool>
__global__ __launch_bounds__(kRopeThreads) void rope_kernel(RopeArgs r, RopeSeqs seqs, RopeRows a, int waves) {
  using Lane = RopeLane<D>;
  // groups asked for at once: 2 leave registers for more waves (64 channels, in a graph: 14.5K tokens of 16 + 8 heads 22.4 us, with 4 23.7; 128 channels: 19.4K
  // tokens of 32 + 4 + 4 heads 85.7, with 4 85.2)
  constexpr int kUnroll = D == 64 ? 2 : 4;
  const int id = __builtin_amdgcn_readfirstlane(blockIdx.x * kRopeWaves + (int)(threadIdx.x >> 6));
  const int row = id / waves, w = id - row * waves;
  if (row >= seqs.total_q) return;
  const Token t = token_of(row, seqs);
  if (!t.ok) return;
  const long long slot = kToPool ? slot_of(t, seqs) : 0;
  const int kv = a.num_kv_heads;
  const int nq = (a.num_q_heads + Lane::kRows - 1) / Lane::kRows, nk = (kv + Lane::kRows - 1) / Lane::kRows;
  const Lane lane(r, t.pos);
  const bool next = r.next != 0;
  const uint16_t* const q = a.q + (size_t)row * a.q_stride + 8 * lane.kc;
  const uint16_t* const k = a.k + (size_t)row * a.k_stride + 8 * lane.kc;
  const uint16_t* const v = a.v + (size_t)row * a.v_stride + 8 * lane.kc;
  uint16_t* const q_out = a.q_out + (size_t)row * a.num_q_heads * D + 8 * lane.kc;
  // a key's or value's next head is one row further in the buffer, or kPage rows in the pool
  const size_t head = (size_t)(kToPool ? kPage : 1) * D;
  const size_t at = (kToPool ? ((size_t)(slot < 0 ? 0 : slot / kPage) * kv * kPage + (slot < 0 ? 0 : slot % kPage)) : (size_t)row * kv) * D + 8 * lane.kc;
  float cw[8], sw[8];
  // rows of one kind: their groups from g0 on among all of the token's
  auto rows = [&](int g0, int groups, int heads, const uint16_t* src, uint16_t* dst, size_t step, auto&& f) {
    int g = w - g0;
    if (g < 0) g += (-g + waves - 1) / waves * waves;
    for (; g < groups; g += kUnroll * waves) {
      u32x4 x[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int h = (g + u * waves) * Lane::kRows + lane.sub;
        x[u] = h < heads ? load16(src + (size_t)h * D) : u32x4{0u, 0u, 0u, 0u};
      }
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        if (g + u * waves >= groups) break;
        const int h = (g + u * waves) * Lane::kRows + lane.sub;
        const u32x4 y = f(x[u]);
        if (h < heads) store16(dst + (size_t)h * step, y);
      }
    }
  };
  const uint16_t* weights = r.q_weight;
  bool norm = weights != nullptr;
  auto turned = [&](const u32x4& x) { return lane.apply(x, next, norm, r.eps, cw, sw); };
  lane.fold(weights, next, cw, sw);
  rows(0, nq, a.num_q_heads, q, q_out, D, turned);
  if (kToPool && slot < 0) return;
  weights = r.k_weight;
  norm = weights != nullptr;
  lane.fold(weights, next, cw, sw);
  rows(nq, nk, kv, k, a.k_out + at, head, turned);
  if (kToPool) rows(nq + nk, nk, kv, v, a.v_out + at, head, [](const u32x4& x) { return x; });
}

// Latent rows.  Group 0 of a token is its latent vector, DC / 8 lanes; the others hold the rows that are rotated: the
// queries' and, as one head more, the key's.
template <int DC, int DR>
__global__ __launch_bounds__(kRopeThreads) void latent_append_kernel(RopeArgs r, RopeSeqs seqs, LatentRows a, int waves) {
  using Lane = RopeLane<DR>;
  constexpr int kUnroll = 4, kWidth = DC + DR;
  const int id = __builtin_amdgcn_readfirstlane(blockIdx.x * kRopeWaves + (int)(threadIdx.x >> 6));
  const int row = id / waves, w = id - row * waves;
  if (row >= seqs.total_q) return;
  const Token t = token_of(row, seqs);
  if (!t.ok) return;
  const long long slot = slot_of(t, seqs);
  uint16_t* const dst = a.cache + (size_t)(slot < 0 ? 0 : slot) * kWidth;
  const uint16_t* const src = a.rows + (size_t)row * a.rows_stride;
  const int groups = (a.num_q_heads + 1 + Lane::kRows - 1) / Lane::kRows;
  if (w == 0) {
    const int l = threadIdx.x & 63;
    const bool in = l < DC / 8;
    u32x4 x = in ? load16(src + 8 * l) : u32x4{0u, 0u, 0u, 0u};
    if (r.k_weight) {
      const u32x4 wt = in ? load16(r.k_weight + 8 * l) : u32x4{0u, 0u, 0u, 0u};
      float sum = 0.f, y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) sum = fmaf(element(x, e), element(x, e), sum);
      const float inv = rsqrtf(lanes_sum<64>(sum) * (1.f / DC) + r.eps);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = element(x, e) * inv * element(wt, e);
      x = rounded(y);
    }
    if (in && slot >= 0) store16(dst + 8 * l, x);
  }
  const int first = w == 0 ? waves : w;
  if (first > groups) return;
  const Lane lane(r, t.pos);
  const bool next = r.next != 0;
  const uint16_t* const q = a.q_rope + (size_t)row * a.num_q_heads * a.q_rope_stride + 8 * lane.kc;
  uint16_t* const q_out = a.q + (size_t)row * a.num_q_heads * kWidth + DC + 8 * lane.kc;
  for (int g = first - 1; g < groups; g += kUnroll * waves) {
    u32x4 x[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int h = (g + u * waves) * Lane::kRows + lane.sub;
      x[u] = h < a.num_q_heads ? load16(q + (size_t)h * a.q_rope_stride)
             : h == a.num_q_heads ? load16(src + DC + 8 * lane.kc) : u32x4{0u, 0u, 0u, 0u};
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      if (g + u * waves >= groups) break;
      const int h = (g + u * waves) * Lane::kRows + lane.sub;
      const u32x4 y = lane.apply(x[u], next, false, 0.f, lane.c, lane.s);
      if (h < a.num_q_heads) store16(q_out + (size_t)h * kWidth, y);
      else if (h == a.num_q_heads && slot >= 0) store16(dst + DC + 8 * lane.kc, y);
    }
  }
}

// Waves a token: one a group while the launch is small, fewer where tokens alone fill the card.  One for all groups, this rule, with four times as
// many, one a group: appends of 64 tokens 9.4, 4.0, 4.0, 4.0 us, of 2048 14.7, 14.6, 20.0, 19.9, of 4800 22.0, 22.5, 33.4, 40.1; more waves look up the
// token's place and make its cosines more often.
constexpr int64_t kRopeFill = 8192;
int waves_per_token(int total_q, int groups) {
  return (int)(total_q * (int64_t)groups <= kRopeFill ? groups : kRopeFill > total_q ? (kRopeFill + total_q - 1) / total_q : 1);
}

}  // namespace

int rope_groups(int head_dim, int num_q_heads, int num_kv_heads, bool to_pool) {
  const int rows = 512 / head_dim;
  return (num_q_heads + rows - 1) / rows + (num_kv_heads + rows - 1) / rows * (to_pool ? 2 : 1);
}

hipError_t launch_rope(const RopeArgs& r, const RopeSeqs& seqs, const RopeRows& rows, int head_dim, bool to_pool, hipStream_t stream) {
  const int waves = waves_per_token(seqs.total_q, rope_groups(head_dim, rows.num_q_heads, rows.num_kv_heads, to_pool));
  const int64_t blocks = ((int64_t)seqs.total_q * waves + kRopeWaves - 1) / kRopeWaves;
  if (blocks * kRopeWaves > INT32_MAX) return hipErrorInvalidValue;
  const dim3 grid((unsigned)blocks), block(kRopeThreads);
  if (head_dim == 128) {
    if (to_pool) hipLaunchKernelGGL((rope_kernel<128, true>), grid, block, 0, stream, r, seqs, rows, waves);
    else hipLaunchKernelGGL((rope_kernel<128, false>), grid, block, 0, stream, r, seqs, rows, waves);
  } else {
    if (to_pool) hipLaunchKernelGGL((rope_kernel<64, true>), grid, block, 0, stream, r, seqs, rows, waves);
    else hipLaunchKernelGGL((rope_kernel<64, false>), grid, block, 0, stream, r, seqs, rows, waves);
  }
  return hipGetLastError();
}

hipError_t launch_latent_append(const RopeArgs& r, const RopeSeqs& seqs, const LatentRows& rows, int latent_dim, int rope_dim,
                                hipStream_t stream) {
  const int per_group = 512 / rope_dim;
  const int waves = waves_per_token(seqs.total_q, 1 + (rows.num_q_heads + per_group) / per_group);
  const int64_t blocks = ((int64_t)seqs.total_q * waves + kRopeWaves - 1) / kRopeWaves;
  if (blocks * kRopeWaves > INT32_MAX) return hipErrorInvalidValue;
  const dim3 grid((unsigned)blocks), block(kRopeThreads);
  if (latent_dim == 512) hipLaunchKernelGGL((latent_append_kernel<512, 64>), grid, block, 0, stream, r, seqs, rows, waves);
  else hipLaunchKernelGGL((latent_append_kernel<256, 32>), grid, block, 0, stream, r, seqs, rows, waves);
  return hipGetLastError();
}

}  // namespace pearl
