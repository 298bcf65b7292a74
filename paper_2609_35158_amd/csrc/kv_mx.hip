// gfx950 kernels that write K/V rows into a cache of MX blocks and read them back: kv_append_mx (the
// append of a turn's new tokens; paper, Background: the context grows by each turn's tokens) and
// kv_pack_mx (the token ranges of a transfer between workers; section 4.3, Eq. 3).
//
// Quantisation of a block of 32 channels: with amax its largest magnitude, s is the least scale that
// keeps amax <= 1.75 * 2^emax * 2^(s - 127) (emax = 2 at 4 bits, 8 at 8), at least 1, and every element is
// x 2^(127 - s) rounded to nearest, ties to even.  At 8 bits 1.75 * 2^8 = 448 is the largest element, so
// none is clipped.  At 4 bits the largest is 6, and amax of 6 to 7 units becomes 6: at most a unit off,
// half the step from 4 to 6, as everywhere else on that step.  (Root mean square error over the signal's, 32 normal numbers a
// block: bound 6 0.1154, 7 0.1119, 8 0.1150; Laplace 0.132, 0.124, 0.127.)  1.75 is read off amax's bf16
// bits, and scaling by a power of two is exact, so the bytes are a function of the bf16 inputs alone.
// Reading back and quantising again gives the same values: the block's largest element is over 3.5
// units at 4 bits, hence s again, and at 8 bits s may drop by one where every element is twice as many units.
// A block holding a NaN or an infinity gets scale 255 and codes 0: all its elements read as NaN.
//
// A workgroup of D threads takes one (page, kv-head).  K: a thread quantises 8 channels of a
// token, four threads share a block (a maximum over a quad).  V: a thread takes one channel pair for 8 tokens and
// 16 neighbouring threads are a block, so the transposed unit is complete in the thread's registers.
// Bound by HBM: bf16 rows one way (512 bytes a token and kv-head at D = 128), MX blocks the other (136 or 264).  80K tokens
// of 8 kv-heads in 4 bits: append 76 us (5.6 TB/s of rows and blocks), read-back 78 us (5.4).

#include "mx_format.h"

namespace pearl {

namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ u16x2 as_u16x2(uint32_t x) { return __builtin_bit_cast(u16x2, x); }
__device__ __forceinline__ uint32_t as_u32(u16x2 x) { return __builtin_bit_cast(uint32_t, x); }
__device__ __forceinline__ uint32_t pk_max(uint32_t a, uint32_t b) { return as_u32(__builtin_elementwise_max(as_u16x2(a), as_u16x2(b))); }

// The maximum, in each half of a dword, with the lane that a DPP control names.
template <int kCtrl> __device__ __forceinline__ uint32_t dpp_max(uint32_t x) {
  return pk_max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kCtrl, 0xf, 0xf, false));
}
constexpr int kQuadXor1 = 0xB1, kQuadXor2 = 0x4E, kRowRor = 0x120;

// The magnitudes of a dword's two bf16, as bits: NaN and infinity are the largest.
__device__ __forceinline__ uint32_t mags(uint32_t w) { return w & 0x7fff7fffu; }

// The scale bytes of two blocks, in the halves of a dword, from the bits of their largest magnitudes: the exponent, one
// more if the 7 mantissa bits are over 96 (1.75 = 1 + 96 / 128; adding 31 carries then), less emax, at least 1; 0xffff
// (byte 255) from infinity on.
template <int kBits> __device__ __forceinline__ uint32_t scale_bytes(uint32_t amax) {
  const u16x2 m = as_u16x2(amax);
  const u16x2 e = (m + (u16x2){31, 31}) >> (u16x2){7, 7};
  constexpr unsigned short least = kBits == 4 ? 3 : 9;      // emax + 1
  const u16x2 s = __builtin_elementwise_max(e, (u16x2){least, least}) - (u16x2){least - 1, least - 1};
  typedef short s16x2_ __attribute__((ext_vector_type(2)));
  const s16x2_ bad = __builtin_bit_cast(s16x2_, m + (u16x2){0x80, 0x80}) >> (s16x2_){15, 15};
  return as_u32(s) | __builtin_bit_cast(uint32_t, bad);
}

// Two bf16 as codes into part kSel of a dword: a byte of four (4 bits), or a half (8 bits).
template <int kBits, int kSel> __device__ __forceinline__ uint32_t mx_down(uint32_t old, uint32_t w, float scale) {
  if constexpr (kBits == 4)
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(old, __builtin_bit_cast(bf16x2, w), scale, kSel);
  else
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(
        __builtin_bit_cast(s16x2, old), __builtin_bit_cast(bf16x2, w), scale, kSel != 0));
}

// How a launch's items, (sequence, logical page) pairs, are counted: per_seq a sequence, or, if that is 0, as
// many as `batch` sequences' token counts can give.
struct PageItems {
  int per_seq, batch;
};

// The (page, kv-head) of a workgroup: its slots [s0, s1) hold the rows row0 .. of this call.
struct PageRows {
  int s0, s1, page;                                 // s0 >= s1: nothing to do
  size_t row0;
};

// Where items are not pages_per_seq a sequence (PageItems), sequence b's start at cu[b] / 16 + 2 b: n tokens
// starting anywhere touch at most n / 16 + 2 pages.  The sequence of an item is found by counting these
// starts with ballots: 64 evenly spaced probes, then 64 in the gap between two, until there is none.
__device__ __forceinline__ int first_item(const int32_t* cu, int b) { return max(cu[b], 0) / kPage + 2 * b; }
__device__ __forceinline__ int seq_of(int item, const int32_t* cu, int batch) {
  const int lane = threadIdx.x & 63;
  int b = 0, n = batch;                             // it is one of b .. b + n - 1
  while (n > 1) {
    const int gap = (n + 63) / 64, probe = lane * gap;
    const int at = max(__popcll(__ballot(probe < n && first_item(cu, b + min(probe, n - 1)) <= item)) - 1, 0) * gap;
    b += at;
    n = min(gap, n - at);
  }
  return __builtin_amdgcn_readfirstlane(b);
}

// The rel-th page that sequence b's new tokens touch.
__device__ __forceinline__ PageRows rows_of(int b, int rel, const int32_t* bt, int bt_stride, const int32_t* ctx_lens,
                                            const int32_t* cu, int total_q) {
  const int q_start = cu ? cu[b] : b;
  const int ctx = ctx_lens[b];
  const int q_len = min(cu ? cu[b + 1] - q_start : 1, total_q - q_start);
  if (q_len <= 0 || q_start < 0 || ctx < 0) return PageRows{0, 0, -1, 0};
  const int lp = ctx / kPage + rel;
  const long long first = max((long long)ctx, (long long)lp * kPage);
  const long long end = min((long long)ctx + q_len, ((long long)lp + 1) * kPage);
  if (first >= end || lp >= bt_stride) return PageRows{0, 0, -1, 0};
  return PageRows{(int)(first - (long long)lp * kPage), (int)(end - (long long)lp * kPage),
                  bt[(size_t)b * bt_stride + lp], (size_t)(q_start + first - ctx)};
}

__device__ __forceinline__ PageRows page_rows(int item, const int32_t* bt, int bt_stride, const int32_t* ctx_lens,
                                              const int32_t* cu, const PageItems& it, int total_q) {
  int b, rel;
  if (it.per_seq > 0) {
    b = item / it.per_seq;
    rel = item - b * it.per_seq;
  } else {
    b = seq_of(item, cu, it.batch);
    rel = item - first_item(cu, b);
    if (rel < 0) return PageRows{0, 0, -1, 0};
  }
  return rows_of(b, rel, bt, bt_stride, ctx_lens, cu, total_q);
}

template <bool kOnce, typename T> __device__ __forceinline__ T read_row(const uint16_t* p) {
  const T* q = reinterpret_cast<const T*>(p);
  if constexpr (kOnce) return __builtin_nontemporal_load(q);
  else return *q;
}

// One page of a kv-head: its slots [s0, s1), all of them if kWhole.
template <int D, int kBits, bool kOnce, bool kWhole>
__device__ __forceinline__ void append_page(const uint16_t* __restrict__ k_new, const uint16_t* __restrict__ v_new,
                                            uint8_t* __restrict__ blk, const PageRows& p, int h, int num_kv_heads) {
  using MX = MxBlock<D, kBits>;
  constexpr int kRowThreads = D / 8, kIters = kPage / 8;    // 8 rows of K at once
  const int tid = threadIdx.x;
  const int row_len = num_kv_heads * D;
  // slot 0's row (of slots before s0 none is read): a uniform base, and a lane's 32-bit offsets from it
  const long long base = ((long long)p.row0 - p.s0) * row_len + (long long)h * D;
  auto holds = [&](int slot) { return kWhole || (slot >= p.s0 && slot < p.s1); };
  // all loads first: K 16 bytes of rows tid / kRowThreads + {0, 8}, V 4 bytes of 8 tokens
  const int kr = tid / kRowThreads, kc = tid % kRowThreads;
  const int pair = tid % (D / 2), half = tid / (D / 2);
  u32x4 k[kIters];
  uint32_t v[8];
#pragma unroll
  for (int i = 0; i < kIters; ++i)
    k[i] = holds(kr + 8 * i) ? read_row<kOnce, u32x4>(k_new + (base + (long long)8 * i * row_len) + (unsigned)(kr * row_len + 8 * kc))
                             : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
  for (int t = 0; t < 8; ++t)
    v[t] = holds(8 * half + t)
               ? read_row<kOnce, uint32_t>(v_new + (base + (long long)t * row_len) + (unsigned)(8 * half * row_len + 2 * pair))
               : 0u;
#pragma unroll
  for (int i = 0; i < kIters; ++i) {
    const int slot = kr + 8 * i;
    uint32_t m = pk_max(pk_max(mags(k[i][0]), mags(k[i][1])), pk_max(mags(k[i][2]), mags(k[i][3])));
    m = pk_max(m, m >> 16 | m << 16);
    m = dpp_max<kQuadXor2>(dpp_max<kQuadXor1>(m));
    const uint32_t s = scale_bytes<kBits>(m) & 0xffu;
    const float f = mx_scale(s);
    u32x2 c;
    if constexpr (kBits == 4)
      c = u32x2{mx_down<4, 3>(mx_down<4, 2>(mx_down<4, 1>(mx_down<4, 0>(0u, k[i][0], f), k[i][1], f), k[i][2], f), k[i][3], f), 0u};
    else
      c = u32x2{mx_down<8, 1>(mx_down<8, 0>(0u, k[i][0], f), k[i][1], f), mx_down<8, 1>(mx_down<8, 0>(0u, k[i][2], f), k[i][3], f)};
    if (s == 255u) c = u32x2{0u, 0u};
    if (holds(slot)) {
      if constexpr (kBits == 4) *reinterpret_cast<uint32_t*>(blk + slot * MX::kRow + 4 * kc) = c[0];
      else *reinterpret_cast<u32x2*>(blk + slot * MX::kRow + 8 * kc) = c;
      if ((kc & 3) == 0) blk[MX::k_scale(slot, kc >> 2)] = (uint8_t)s;
    }
  }
  // V: tokens 2 x and 2 x + 1 side by side in the halves of a dword, from their maxima to their scales
  uint32_t s2[4], c[kBits / 2];
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    const uint32_t a = mags(v[2 * x]), b = mags(v[2 * x + 1]);
    uint32_t m = pk_max(__builtin_amdgcn_perm(b, a, 0x05040100u), __builtin_amdgcn_perm(b, a, 0x07060302u));
    m = dpp_max<kRowRor + 8>(m);
    m = dpp_max<kRowRor + 4>(m);
    m = dpp_max<kRowRor + 2>(m);
    m = dpp_max<kRowRor + 1>(m);
    s2[x] = scale_bytes<kBits>(m);
    const float f0 = mx_scale(s2[x] & 0xffu), f1 = mx_scale(s2[x] >> 16 & 0xffu);
    if constexpr (kBits == 4) {
      if (x % 2 == 0) c[x / 2] = mx_down<4, 1>(mx_down<4, 0>(0u, v[2 * x], f0), v[2 * x + 1], f1);
      else c[x / 2] = mx_down<4, 3>(mx_down<4, 2>(c[x / 2], v[2 * x], f0), v[2 * x + 1], f1);
    } else {
      c[x] = mx_down<8, 1>(mx_down<8, 0>(0u, v[2 * x], f0), v[2 * x + 1], f1);
    }
  }
  if (__ballot(((s2[0] | s2[1] | s2[2] | s2[3]) & 0xff00ff00u) != 0u)) {   // some block has no scale: codes 0
#pragma unroll
    for (int t = 0; t < 8; ++t)
      if (s2[t / 2] >> (16 * (t % 2) + 8) & 1u) {
        if constexpr (kBits == 4) c[t / 4] &= ~(0xffu << (8 * (t % 4)));
        else c[t / 2] &= ~(0xffffu << (16 * (t % 2)));
      }
  }
  const u32x2 s8 = {__builtin_amdgcn_perm(s2[1], s2[0], 0x06040200u), __builtin_amdgcn_perm(s2[3], s2[2], 0x06040200u)};
  const bool scales = (pair & 15) == 0;
  uint8_t* const vc = blk + MX::v_code(8 * half, pair);
  uint8_t* const vs = blk + MX::v_scale(8 * half, pair >> 4);
  const int lo = p.s0 - 8 * half, hi = p.s1 - 8 * half;       // this thread's tokens are lo <= t < hi
  if (kWhole || (lo <= 0 && hi >= 8)) {
    if constexpr (kBits == 4) *reinterpret_cast<u32x2*>(vc) = u32x2{c[0], c[1]};
    else *reinterpret_cast<u32x4*>(vc) = u32x4{c[0], c[1], c[2], c[3]};
    if (scales) *reinterpret_cast<u32x2*>(vs) = s8;
  } else {
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      if (t < lo || t >= hi) continue;
      if constexpr (kBits == 4) vc[t] = (uint8_t)(c[t / 4] >> (8 * (t % 4)));
      else reinterpret_cast<uint16_t*>(vc)[t] = (uint16_t)(c[t / 2] >> (16 * (t % 2)));
      if (scales) vs[t] = (uint8_t)(s8[t / 4] >> (8 * (t % 4)));
    }
  }
}

}  // namespace

// blockIdx.x = item * num_kv_heads + h.  Rows of a page id outside [0, num_pages) are skipped.
// kOnce: the rows are read past the caches.
template <int D, int kBits, bool kOnce>
__global__ __launch_bounds__(D) void kv_append_mx_kernel(
    const uint16_t* __restrict__ k_new, const uint16_t* __restrict__ v_new, uint8_t* __restrict__ cache,
    const int32_t* __restrict__ bt, int bt_stride, const int32_t* __restrict__ ctx_lens,
    const int32_t* __restrict__ cu, PageItems items, int num_kv_heads, int num_pages, int total_q) {
  using MX = MxBlock<D, kBits>;
  const int item = blockIdx.x / num_kv_heads, h = blockIdx.x - item * num_kv_heads;
  const PageRows p = page_rows(item, bt, bt_stride, ctx_lens, cu, items, total_q);
  if (p.s0 >= p.s1 || p.page < 0 || p.page >= num_pages) return;
  uint8_t* const blk = cache + ((size_t)p.page * num_kv_heads + h) * MX::kBytes;
  if (p.s0 == 0 && p.s1 == kPage)
    append_page<D, kBits, kOnce, true>(k_new, v_new, blk, p, h, num_kv_heads);
  else
    append_page<D, kBits, kOnce, false>(k_new, v_new, blk, p, h, num_kv_heads);
}

// The rows of the same token ranges, as bf16: zeros for a page id outside [0, num_pages).
template <int D, int kBits>
__global__ __launch_bounds__(D) void kv_pack_mx_kernel(
    const uint8_t* __restrict__ cache, uint16_t* __restrict__ k_rows, uint16_t* __restrict__ v_rows,
    const int32_t* __restrict__ bt, int bt_stride, const int32_t* __restrict__ ctx_lens,
    const int32_t* __restrict__ cu, PageItems items, int num_kv_heads, int num_pages, int total_q) {
  using MX = MxBlock<D, kBits>;
  constexpr int kRowThreads = D / 8, kRowsAtOnce = D / kRowThreads, kIters = kPage / kRowsAtOnce;
  const int item = blockIdx.x / num_kv_heads, h = blockIdx.x - item * num_kv_heads;
  const PageRows p = page_rows(item, bt, bt_stride, ctx_lens, cu, items, total_q);
  if (p.s0 >= p.s1) return;
  const bool ok = p.page >= 0 && p.page < num_pages;
  const int tid = threadIdx.x;
  const uint8_t* const blk = cache + ((size_t)(ok ? p.page : 0) * num_kv_heads + h) * MX::kBytes;
  auto row = [&](uint16_t* rows, int slot) {
    return rows + ((p.row0 + (slot - p.s0)) * num_kv_heads + h) * D;
  };
  const int kr = tid / kRowThreads, kc = tid % kRowThreads;
  u32x2 k[kIters];
  uint32_t ks[kIters];
#pragma unroll
  for (int i = 0; i < kIters; ++i) {
    const int slot = kr + i * kRowsAtOnce;
    if constexpr (kBits == 4) k[i] = u32x2{*reinterpret_cast<const uint32_t*>(blk + slot * MX::kRow + 4 * kc), 0u};
    else k[i] = *reinterpret_cast<const u32x2*>(blk + slot * MX::kRow + 8 * kc);
    ks[i] = blk[MX::k_scale(slot, kc >> 2)];
  }
  const int pair = tid % (D / 2), half = tid / (D / 2);
  const uint8_t* const vc = blk + MX::v_code(8 * half, pair);
  u32x4 v;
  if constexpr (kBits == 4) {
    const u32x2 w = *reinterpret_cast<const u32x2*>(vc);
    v = u32x4{w[0], w[1], 0u, 0u};
  } else {
    v = *reinterpret_cast<const u32x4*>(vc);
  }
  const u32x2 vs = *reinterpret_cast<const u32x2*>(blk + MX::v_scale(8 * half, pair >> 4));
#pragma unroll
  for (int i = 0; i < kIters; ++i) {
    const int slot = kr + i * kRowsAtOnce;
    const float f = mx_scale(ks[i]);
    u32x4 x;
    if constexpr (kBits == 4)
      x = u32x4{mx_up<4, 0>(k[i][0], f), mx_up<4, 1>(k[i][0], f), mx_up<4, 2>(k[i][0], f), mx_up<4, 3>(k[i][0], f)};
    else
      x = u32x4{mx_up<8, 0>(k[i][0], f), mx_up<8, 1>(k[i][0], f), mx_up<8, 0>(k[i][1], f), mx_up<8, 1>(k[i][1], f)};
    if (slot >= p.s0 && slot < p.s1)
      *reinterpret_cast<u32x4*>(row(k_rows, slot) + 8 * kc) = ok ? x : u32x4{0u, 0u, 0u, 0u};
  }
  auto token = [&](auto t_c) {                      // token 8 half + t: 4 bytes a thread, a row together
    constexpr int t = decltype(t_c)::value;
    const int slot = 8 * half + t;
    if (slot < p.s0 || slot >= p.s1) return;
    const float f = mx_scale_of<t % 4>(vs[t / 4]);
    const uint32_t x = kBits == 4 ? mx_up<kBits, t % 4>(v[t / 4], f) : mx_up<kBits, t % 2>(v[t / 2], f);
    *reinterpret_cast<uint32_t*>(row(v_rows, slot) + 2 * pair) = ok ? x : 0u;
  };
  token(std::integral_constant<int, 0>{});
  token(std::integral_constant<int, 1>{});
  token(std::integral_constant<int, 2>{});
  token(std::integral_constant<int, 3>{});
  token(std::integral_constant<int, 4>{});
  token(std::integral_constant<int, 5>{});
  token(std::integral_constant<int, 6>{});
  token(std::integral_constant<int, 7>{});
}

// Up to one token a sequence, as in a decode step: a wave takes a (sequence, kv-head), a lane a channel pair of K and of V
// (at D = 64 the half-waves take one each).  The rows are on their way while the page is looked up, and no vector work goes
// into the 15 other slots.  The append's first workgroup also clears `zero` (a decode step's append and its decode are then
// two launches, as decode alone).  us of an append and of a read-back, 8 kv-heads, d = 128, 4 bits, by the kernels above
// and so: one sequence 2.9 and 2.0, so 2.1 and 1.9; 64 3.4 and 2.4, so 2.2 and 2.1; 512 7.2 and 4.4, so 3.7 and 2.9; 4096 34 and
// 21, so 13 and 11.
constexpr int kTokenWaves = 4;                      // of a workgroup

namespace {
// A lane's dwords of a token: which of K (0) and V (1) they are of, where its codes and, in a block's first lane, its scale
// are in the MX block.
template <int D, int kBits> struct TokenLane {
  using MX = MxBlock<D, kBits>;
  static constexpr int kWords = D / 64, kCodeBytes = kBits / 4;
  int lane, pair;
  __device__ __forceinline__ TokenLane() : lane(threadIdx.x & 63), pair(lane % (D / 2)) {}
  __device__ __forceinline__ int is_v(int i) const { return kWords == 2 ? i : lane >> 5; }
  __device__ __forceinline__ int code(int i, int slot) const { return is_v(i) ? MX::v_code(slot, pair) : slot * MX::kRow + pair * kCodeBytes; }
  __device__ __forceinline__ int scale(int i, int slot) const { return is_v(i) ? MX::v_scale(slot, pair >> 4) : MX::k_scale(slot, pair >> 4); }
};
}  // namespace

template <int D, int kBits>
__global__ __launch_bounds__(64 * kTokenWaves) void kv_append_token_mx_kernel(
    const uint16_t* __restrict__ k_new, const uint16_t* __restrict__ v_new, uint8_t* __restrict__ cache,
    const int32_t* __restrict__ bt, int bt_stride, const int32_t* __restrict__ ctx_lens,
    const int32_t* __restrict__ cu, int batch, int num_kv_heads, int num_pages, int total_q, ZeroWords zero) {
  using MX = MxBlock<D, kBits>;
  using T = TokenLane<D, kBits>;
  if (blockIdx.x == 0) {
    if (zero.hdr && threadIdx.x < kHdrWords) zero.hdr[threadIdx.x] = 0;
    for (int i = threadIdx.x; i < zero.n_cnt; i += 64 * kTokenWaves) zero.cnt[i] = 0;
  }
  const int item = __builtin_amdgcn_readfirstlane((int)blockIdx.x * kTokenWaves + (int)(threadIdx.x >> 6));
  if (item >= batch * num_kv_heads) return;
  const int b = item / num_kv_heads, h = item - b * num_kv_heads;
  const T t;
  const size_t at = ((size_t)min(max(cu ? cu[b] : b, 0), total_q - 1) * num_kv_heads + h) * D + 2 * t.pair;
  uint32_t x[T::kWords];
#pragma unroll
  for (int i = 0; i < T::kWords; ++i) x[i] = *reinterpret_cast<const uint32_t*>((t.is_v(i) ? v_new : k_new) + at);
  const PageRows p = rows_of(b, 0, bt, bt_stride, ctx_lens, cu, total_q);
  if (p.s0 >= p.s1 || p.page < 0 || p.page >= num_pages) return;
  uint8_t* const blk = cache + ((size_t)p.page * num_kv_heads + h) * MX::kBytes;
  uint32_t m = mags(x[0]);                          // the larger magnitude, or K's and V's
  if constexpr (T::kWords == 2) m = pk_max(__builtin_amdgcn_perm(mags(x[1]), m, 0x05040100u), __builtin_amdgcn_perm(mags(x[1]), m, 0x07060302u));
  else m = pk_max(m, m >> 16 | m << 16);
  m = dpp_max<kRowRor + 8>(m);
  m = dpp_max<kRowRor + 4>(m);
  m = dpp_max<kRowRor + 2>(m);
  m = dpp_max<kRowRor + 1>(m);
  const uint32_t s2 = scale_bytes<kBits>(m);
#pragma unroll
  for (int i = 0; i < T::kWords; ++i) {
    const uint32_t s = s2 >> (16 * i) & 0xffu;
    const uint32_t c = s == 255u ? 0u : mx_down<kBits, 0>(0u, x[i], mx_scale(s));
    uint8_t* const to = blk + t.code(i, p.s0);
    if constexpr (kBits == 4) *to = (uint8_t)c;
    else *reinterpret_cast<uint16_t*>(to) = (uint16_t)c;
    if ((t.lane & 15) == 0) blk[t.scale(i, p.s0)] = (uint8_t)s;
  }
}

template <int D, int kBits>
__global__ __launch_bounds__(64 * kTokenWaves) void kv_pack_token_mx_kernel(
    const uint8_t* __restrict__ cache, uint16_t* __restrict__ k_rows, uint16_t* __restrict__ v_rows,
    const int32_t* __restrict__ bt, int bt_stride, const int32_t* __restrict__ ctx_lens,
    const int32_t* __restrict__ cu, int batch, int num_kv_heads, int num_pages, int total_q) {
  using MX = MxBlock<D, kBits>;
  using T = TokenLane<D, kBits>;
  const int item = __builtin_amdgcn_readfirstlane((int)blockIdx.x * kTokenWaves + (int)(threadIdx.x >> 6));
  if (item >= batch * num_kv_heads) return;
  const int b = item / num_kv_heads, h = item - b * num_kv_heads;
  const PageRows p = rows_of(b, 0, bt, bt_stride, ctx_lens, cu, total_q);
  if (p.s0 >= p.s1) return;
  const bool ok = p.page >= 0 && p.page < num_pages;
  const uint8_t* const blk = cache + ((size_t)(ok ? p.page : 0) * num_kv_heads + h) * MX::kBytes;
  const T t;
  const size_t at = (p.row0 * num_kv_heads + h) * D + 2 * t.pair;
#pragma unroll
  for (int i = 0; i < T::kWords; ++i) {
    const uint8_t* const from = blk + t.code(i, p.s0);
    const uint32_t c = kBits == 4 ? *from : *reinterpret_cast<const uint16_t*>(from);
    const uint32_t x = mx_up<kBits, 0>(c, mx_scale(blk[t.scale(i, p.s0)]));
    *reinterpret_cast<uint32_t*>((t.is_v(i) ? v_rows : k_rows) + at) = ok ? x : 0u;
  }
}

namespace {
// Workgroups of a launch over the token ranges, or -1 if they pass the grid's limit of 2^32 threads.  A sequence of up
// to max_q_len tokens touches at most ceil((max_q_len + 15) / 16) pages.  As many items for each sequence are found without
// a search, but where few are as long as the longest most items hold nothing.  us of an append, 8 kv-heads, d = 128, 4 bits,
// with as many for each and by the token counts, and how many times more items the first gives: 256 sequences of 20 new
// tokens (0.92) 9.0 and 10.0; 200 of 1-64 (1.23) 9.7 and 10.4; 32 of 1-4096 (1.89) 63.7 and 60.5; 63 of 100 and one of 330
// (2.60) 10.0 and 8.5; 255 of one and one of 8192 (126) 376 and 12.
int64_t page_items(int batch, int max_q_len, int total_q, int num_kv_heads, int head_dim, PageItems* items) {
  const int64_t per_seq = (max_q_len + 2 * kPage - 2) / kPage;
  const int64_t even = batch * per_seq, least = (int64_t)total_q / kPage + 2 * (int64_t)batch;
  const bool by_count = 2 * even > 3 * least;
  *items = PageItems{by_count ? 0 : (int)per_seq, batch};
  const int64_t blocks = (by_count ? least : even) * num_kv_heads;
  return blocks * head_dim > UINT32_MAX ? -1 : blocks;
}
int64_t token_blocks(int batch, int num_kv_heads) {
  const int64_t blocks = ((int64_t)batch * num_kv_heads + kTokenWaves - 1) / kTokenWaves;
  return blocks * 64 * kTokenWaves > UINT32_MAX ? -1 : blocks;
}

template <bool kOnce> auto append_kernel_of(int head_dim, int bits) {
  return head_dim == 64 ? (bits == 4 ? kv_append_mx_kernel<64, 4, kOnce> : kv_append_mx_kernel<64, 8, kOnce>)
                        : (bits == 4 ? kv_append_mx_kernel<128, 4, kOnce> : kv_append_mx_kernel<128, 8, kOnce>);
}
}  // namespace

hipError_t launch_kv_append_mx(int bits, const uint16_t* k_new, const uint16_t* v_new, uint8_t* cache,
                               const int32_t* block_table, int bt_stride, const int32_t* ctx_lens,
                               const int32_t* cu_q_lens, int batch, int max_q_len, int num_kv_heads, int head_dim,
                               int num_pages, int total_q, const ZeroWords& zero, hipStream_t stream) {
  if (max_q_len <= 0 || batch <= 0 || total_q <= 0) return hipSuccess;
  if (max_q_len == 1 || !cu_q_lens) {
    const int64_t blocks = token_blocks(batch, num_kv_heads);
    if (blocks < 0) return hipErrorInvalidValue;
    auto kernel = head_dim == 64 ? (bits == 4 ? kv_append_token_mx_kernel<64, 4> : kv_append_token_mx_kernel<64, 8>)
                                 : (bits == 4 ? kv_append_token_mx_kernel<128, 4> : kv_append_token_mx_kernel<128, 8>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(64 * kTokenWaves), 0, stream, k_new, v_new, cache, block_table,
                       bt_stride, ctx_lens, cu_q_lens, batch, num_kv_heads, num_pages, total_q, zero);
    return hipGetLastError();
  }
  PageItems items;
  const int64_t blocks = page_items(batch, max_q_len, total_q, num_kv_heads, head_dim, &items);
  if (blocks < 0) return hipErrorInvalidValue;
  // Rows of 48 MiB on are read with non-temporal loads: they would only push each other out of the caches.  us of an append
  // and its read-back without and with them, 8 kv-heads, d = 128: 8K tokens (34 MB of rows) in 4 bits 17.5 and 18.0, in 8
  // bits 19.4 and 20.5; 16K 38.0 and 32.5; 33K 68.7 and 61.1, in 8 bits 81.7 and 72.4; 66K 150 and 125.
  const bool once = 4 * (int64_t)total_q * num_kv_heads * head_dim >= (int64_t)48 << 20;
  auto kernel = once ? append_kernel_of<true>(head_dim, bits) : append_kernel_of<false>(head_dim, bits);
  hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(head_dim), 0, stream, k_new, v_new, cache, block_table,
                     bt_stride, ctx_lens, cu_q_lens, items, num_kv_heads, num_pages, total_q);
  return hipGetLastError();
}

hipError_t launch_kv_pack_mx(int bits, const uint8_t* cache, uint16_t* k_rows, uint16_t* v_rows,
                             const int32_t* block_table, int bt_stride, const int32_t* ctx_lens,
                             const int32_t* cu_q_lens, int batch, int max_q_len, int num_kv_heads, int head_dim,
                             int num_pages, int total_q, hipStream_t stream) {
  if (max_q_len <= 0 || batch <= 0 || total_q <= 0) return hipSuccess;
  if (max_q_len == 1 || !cu_q_lens) {
    const int64_t blocks = token_blocks(batch, num_kv_heads);
    if (blocks < 0) return hipErrorInvalidValue;
    auto kernel = head_dim == 64 ? (bits == 4 ? kv_pack_token_mx_kernel<64, 4> : kv_pack_token_mx_kernel<64, 8>)
                                 : (bits == 4 ? kv_pack_token_mx_kernel<128, 4> : kv_pack_token_mx_kernel<128, 8>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(64 * kTokenWaves), 0, stream, cache, k_rows, v_rows, block_table,
                       bt_stride, ctx_lens, cu_q_lens, batch, num_kv_heads, num_pages, total_q);
    return hipGetLastError();
  }
  PageItems items;
  const int64_t blocks = page_items(batch, max_q_len, total_q, num_kv_heads, head_dim, &items);
  if (blocks < 0) return hipErrorInvalidValue;
  auto kernel = head_dim == 64 ? (bits == 4 ? kv_pack_mx_kernel<64, 4> : kv_pack_mx_kernel<64, 8>)
                               : (bits == 4 ? kv_pack_mx_kernel<128, 4> : kv_pack_mx_kernel<128, 8>);
  hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(head_dim), 0, stream, cache, k_rows, v_rows, block_table,
                     bt_stride, ctx_lens, cu_q_lens, items, num_kv_heads, num_pages, total_q);
  return hipGetLastError();
}

}  // namespace pearl
