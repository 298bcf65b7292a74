// gfx950 decode attention over a cache of MX blocks (mx_format.h): one new token per sequence, each query
// head over the cached keys of its kv-head (paper, section 4.3, Eq. 1: the KV-cache read per
// sequence is what a decode step costs).
//
// The launch is cut as decode_kernel's (decode_shares.h): every wave streams an equal run of the batch's
// pages, whatever the lengths.  A wave takes a unit of kPages pages of a sequence at a time:
//   S^T (keys x heads)   = K . Q^T      16x16x32 MFMA, A = K rows, B = the group's queries
//   O^T (pairs x heads) += V^T . P^T    16x16x32 MFMA, A = channel pairs of V, B = the weights
// A unit travels by LDS-DMA, block by block as it lies in memory (1 KiB an instruction), into the wave's two
// buffers; the next unit's copies are in flight while one is attended.
//   * Lane group g = l / 16 of the products holds the unit's tokens TG g .. TG g + TG - 1 (TG = 4 kPages).
//     Row 4 g + i of K tile t is token 4 t + i of group g, so the scores of tile t come out, in the lanes of
//     group g, as those of the tokens whose V those lanes hold: the weights are P.V's operand as they are.
//   * Elements are turned into bf16 by the conversion instructions, which apply the scale: exact.  A K
//     conversion gives two neighbouring channels, an operand's dword.  A V conversion gives the two
//     channels of a pair for one token, and goes into the product as it is, as two contraction indices (token, even)
//     and (token, odd): the products have 16 columns for at most 8 heads, so columns 0..7 hold the weights
//     at the even indices and columns 8..15 at the odd ones (zeros at the others), and give the even and
//     the odd channels.  (Sorted by channel first, with a byte permute per two tokens, the conversion of V
//     took 192 instructions a unit instead of 128.)
// Weights enter P.V in two bf16 parts, the nearest bf16 and the rest, in a product each: 16 bits of a weight.  One
// part alone is 2-6% faster (64 sequences of 2K-16K tokens 122.4 us, with both 125.9) but off by up to 2^-8 a
// weight, as much as rounding the outputs to bf16 is.
// The other channel of a pair meets a weight of 0 in each column half, and 0 times an infinity or NaN is NaN.  So every
// unit is tested for scales and codes that stand for such elements of V; where there are any, they are counted in a
// product of their own and added to the outputs, and become zeros for the weights' product: an infinite element of an
// attended token makes its own channel infinite, and no other one anything.  (The test: 64 sequences of 2K-16K tokens in
// 4 bits 113.0 us for 112.9, at d = 64 256 of 200-3000 59.0 for 58.2; in 8 bits, with all codes, 64 of 2K-16K 189.7 for
// 188.9, at d = 64 48 of 500-6000 34.9 for 33.9.)
// The running maximum may lag the true one by 8 (log2 units), as in the prefill kernel: most units look for none.

#include "decode_shares.h"
#include "mx_format.h"

#include <algorithm>
#include <atomic>

namespace pearl {

namespace {

// 2176 bytes of K and V a page and kv-head at 4 bits, d = 128.  Each line is drawn by type, where the times of batches on
// both sides of it say so (us a call, 8 kv-heads unless said).
// kPieceCost, several kv-heads a workgroup, 8 and 3: d = 64 in 8 bits 48 sequences of 500-6000 tokens 35.9 and 34.0, 32 of
//   2K-8K 37.4 and 36.0, 200 of 1K-5K at 2 kv-heads 38.0 and 36.9; but in 4 bits 64 of 2K-6K 38.7 and 41.3; d = 128 in 8 bits
//   48 of 2K-6K 67.8 and 70.8, 32 of 2K-8K 58.8 and 64.4, 200 of 500-2000 at 4 kv-heads 53.6 and 57.6; in 4 bits, 8 and
//   4, 48 of 2K-6K 44.8 and 47.7, 200 of 500-2000 at 4 kv-heads 38.5 and 42.3.  (Why d = 64 in 8 bits differs is not known.)
// kWholePages, no runs of whole sequences, and with 28, 56 and 112: 4 bits, 24 of 500-1000 16.1 / 13.6 / 13.4 / 13.6, 24 of
//   500-1200 16.1 / 16.1 / 15.7 / 15.7, 300 of 100-500 at 2 kv-heads 21.0 / 21.0 / 20.0 / 20.2, at d = 64 100 of 200-1500 at 2
//   16.8 / 16.9 / 16.8 / 15.1; 8 bits, 24 of 500-1200 17.4 / 17.3 / 16.8 / 16.9, at d = 64 40 of 200-1200 17.3 / 17.3 / 17.1 / 19.0.
// kSeqCost, 0, 4 and 8: shares of 70 pages of 512 sequences (64-1024 tokens) took 2.2 us a unit and 2.0 a sequence more, so
//   those with 5 or 6 sequences ended last: 65.8 / 62.9 / 63.5; 900 of 1-400 57.9 / 53.2 / 53.2, 64 of 2K-16K 109.5 / 108.0 /
//   106.9; at d = 64 700 of 64-1024 59.2 / 58.0 / 59.6, in 8 bits 900 of 64-512 61.0 / 56.1 / 57.3; d = 128 in 8 bits 512 of
//   64-1024 105.0 / 106.3 / 108.5.
template <int D, int kBits, int kPages> struct MxCut {
  static constexpr int kPieceCost = D == 64 && kBits == 8 ? 3 : 8, kWholePages = 56, kSeqCost = kMxSeqCost, kUnit = kPages;
};

// A unit: kPages pages of one (sequence, kv-head) and how they lie in a wave's buffer.
template <int D, int kBits> struct Unit {
  using MX = MxBlock<D, kBits>;
  // Two buffers of 8 waves in LDS: 4 pages at D = 128 and 4 bits, 2 at 8 bits.  At D = 64 and 4 bits 2 pages leave room for
  // a second workgroup (us a call with 4 pages and with 2, 8 kv-heads: 100 sequences of 300-3000 tokens 33.9 and 30.8, 16
  // of 2K-30K 40.5 and 38.8); at 8 bits that loses more at large batches (256 of 200-3000: 79.4 and 83.8) than it gains at
  // small ones (40 of 300-6000: 32.0 and 31.2).
  static constexpr int kPages = D * kBits == 512 ? 4 : 2;
  static constexpr int TG = 4 * kPages;             // tokens of a lane group
  static constexpr int KB = D / 32;                 // 32-channel steps of the Q.K product
  static constexpr int TP = D / 32;                 // groups of 16 channel pairs
  static constexpr int kCopies = 2 * MX::kCodes / 1024;   // 1 KiB copies of a page's codes
  static constexpr int kPageBytes = 2 * MX::kCodes + 16;  // 16 bytes apart mod 256: K rows of 4 pages on other banks
  static constexpr int kScaleBytes = MX::kBytes - 2 * MX::kCodes;
  static constexpr int kScales = kPages * kPageBytes;     // offset of the pages' scales
  static constexpr int kBytes = kScales + kPages * kScaleBytes;
  static_assert(kCopies >= 1 && kCopies * 1024 == 2 * MX::kCodes && kPages * kScaleBytes <= 1024, "copies");
};

// The first channel of k-step ks of a lane group: 16-byte pieces of a row where a group holds more.
template <int D, int kBits> __device__ __forceinline__ int k_channel(int group, int ks) {
  if constexpr (D == 128 && kBits == 8) return 64 * (ks >> 1) + 16 * group + 8 * (ks & 1);
  else return D / 4 * group + 8 * ks;
}

// 1 KiB from base + 16 lane (+ 1024 i) to LDS at lds + 16 lane (+ 1024 i), i < N: as lds_dma16 in the bf16 kernels.
template <int N> __device__ __forceinline__ void copy_codes(const uint8_t* base, int lane16, unsigned lds) {
  unsigned saved;
  if constexpr (N == 1)
    __asm__ volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\t"
                     "global_load_lds_dwordx4 %3, %2 nt\n\t"
                     "s_mov_b32 m0, %0"
                     : "=&s"(saved) : "s"(lds), "s"(base), "v"(lane16) : "memory");
  else if constexpr (N == 2)
    __asm__ volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\t"
                     "global_load_lds_dwordx4 %3, %2 nt\n\t"
                     "global_load_lds_dwordx4 %3, %2 offset:1024 nt\n\t"
                     "s_mov_b32 m0, %0"
                     : "=&s"(saved) : "s"(lds), "s"(base), "v"(lane16) : "memory");
  else
    __asm__ volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\t"
                     "global_load_lds_dwordx4 %3, %2 nt\n\t"
                     "global_load_lds_dwordx4 %3, %2 offset:1024 nt\n\t"
                     "global_load_lds_dwordx4 %3, %2 offset:2048 nt\n\t"
                     "global_load_lds_dwordx4 %3, %2 offset:3*1024 nt\n\t"
                     "s_mov_b32 m0, %0"
                     : "=&s"(saved) : "s"(lds), "s"(base), "v"(lane16) : "memory");
}
__device__ __forceinline__ void copy_scales(const uint8_t* at, unsigned lds) {   // 16 bytes a lane from its own address
  unsigned saved;
  __asm__ volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\t"
                   "global_load_lds_dwordx4 %1, off nt\n\t"
                   "s_mov_b32 m0, %0"
                   : "=&s"(saved) : "v"(at), "s"(lds) : "memory");
}

template <int N> __device__ __forceinline__ void lds_words(uint32_t* x, const char* p) {
  if constexpr (N == 1) {
    x[0] = *reinterpret_cast<const uint32_t*>(p);
  } else if constexpr (N == 2) {
    const u32x2 y = *reinterpret_cast<const u32x2*>(p);
    x[0] = y[0];
    x[1] = y[1];
  } else {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const u32x4 y = *reinterpret_cast<const u32x4*>(p + 4 * i);
#pragma unroll
      for (int j = 0; j < 4; ++j) x[i + j] = y[j];
    }
  }
}

template <int kBits> __device__ __forceinline__ bf16x8 eight_up(const uint32_t* w, float f) {
  if constexpr (kBits == 4)
    return as_bf16x8(u32x4{mx_up<4, 0>(w[0], f), mx_up<4, 1>(w[0], f), mx_up<4, 2>(w[0], f), mx_up<4, 3>(w[0], f)});
  else
    return as_bf16x8(u32x4{mx_up<8, 0>(w[0], f), mx_up<8, 1>(w[0], f), mx_up<8, 0>(w[1], f), mx_up<8, 1>(w[1], f)});
}

// Of a pair of V in bf16: 1 for an infinite element, 2^8 for minus infinity, 2^16 for NaN (in bf16), so that a sum over a
// unit's up to 64 tokens counts each kind exactly; `mask` covers these elements.
__device__ __forceinline__ uint32_t odd_kinds(uint32_t x, uint32_t& mask) {
  mask = (mx_low_not_finite(x) ? 0x0000ffffu : 0u) | (mx_high_not_finite(x) ? 0xffff0000u : 0u);
  auto kind = [](uint32_t b) -> uint32_t { return (b & 0x7fu) ? 0x4780u : (b & 0x8000u) ? 0x4380u : 0x3f80u; };
  return (kind(x & 0xffffu) | kind(x >> 16) << 16) & mask;
}
// x and the elements that were so counted in n.
__device__ __forceinline__ float with_odd(float x, float n) {
  const int k = (int)n;
  if (k == 0) return x;
  const bool nan = k >= 1 << 16 || ((k & 255) != 0 && k >= 1 << 8);
  return x + (nan ? __builtin_nanf("") : k >= 1 << 8 ? -INFINITY : INFINITY);
}

// x in bf16 in both halves of a dword.
__device__ __forceinline__ uint32_t twice_bf16(float x) {
  const bf16x2 y = {(__bf16)x, (__bf16)x};
  return __builtin_bit_cast(uint32_t, y);
}

// A lane's places in a buffer, and the products of a unit.
template <int D, int kBits> struct Attend {
  using MX = MxBlock<D, kBits>;
  using U = Unit<D, kBits>;
  static constexpr int TG = U::TG, NT = U::kPages;  // NT: tiles of 16 keys
  static constexpr int kPieces = D * kBits / 8 >= 128 ? 2 : 1;   // of a lane's K row: 16 bytes (8 at 64 x 4)
  static constexpr int KW = D * kBits / 128;        // dwords of it
  static constexpr int VW = TG * kBits / 16;        // dwords of a channel pair's tokens
  int k, ks, v, vs;
  int vs_any, vs_tok;                               // this lane's word of all of the unit's V scales, and its first token
  int k_shift;                                      // of the scale word: tile t's byte becomes byte t
  __device__ __forceinline__ explicit Attend(int lane) {
    const int row = lane & 15, group = lane >> 4;
    const int tok = row / 4 * TG + (row & 3);       // of tile 0; tile t is 4 t further, on the same page
    k = tok / kPage * U::kPageBytes + tok % kPage * MX::kRow + group * (KW >= 4 ? 16 : 8);
    const int blk = D == 128 && kBits == 4 ? group : group >> 1;   // of piece 0; piece 1 is two blocks on
    ks = U::kScales + tok / kPage * U::kScaleBytes + ((tok & 3) * MX::kBlocks + blk) * 4;
    k_shift = tok % kPage / 4 * 8;
    const int vt = group * TG;
    v = vt / kPage * U::kPageBytes + MX::v_code(vt % kPage, row);
    vs = U::kScales + vt / kPage * U::kScaleBytes + MX::kVScales - 2 * MX::kCodes + vt % kPage;
    constexpr int kWords = kPage * MX::kBlocks / 4;  // of a page
    const int word = lane % (U::kPages * kWords), page = word / kWords, at = word % kWords * 4;
    vs_any = U::kScales + page * U::kScaleBytes + MX::kVScales - 2 * MX::kCodes + at;
    vs_tok = page * kPage + at % kPage - group * TG;
  }

  // The first `left` (0 to 4) bytes of a word.
  __device__ static __forceinline__ uint32_t bytes(int left) { return left >= 4 ? 0xffffffffu : (1u << (8 * max(left, 0))) - 1u; }

  // Adds the unit's infinite and NaN elements of V to the outputs, and makes them zeros in buf (a scale of 255 becomes 0).
  // Rare: a token at a time, in few registers.
  __device__ __forceinline__ void take_odd(char* buf, f32x4* oacc, int lim, uint32_t half) const {
    const uint32_t one = 0x3f803f80u & half;
    int codes = v, scales = vs;
    __asm__ volatile("" : "+v"(codes), "+v"(scales));   // (else the addresses below are kept in registers all along)
#pragma unroll
    for (int q = 0; q < U::TP; ++q) {
      f32x4 n = {0.f, 0.f, 0.f, 0.f};               // counts of each channel
#pragma unroll 1
      for (int j = 0; j < TG; ++j) {
        char* const code = buf + codes + 256 * q + (kBits == 4 ? j : j / 8 * (D / 2 * 16) + j % 8 * 2);
        uint8_t* const scale = reinterpret_cast<uint8_t*>(buf + scales + kPage * q + j);
        const uint32_t w = kBits == 4 ? *reinterpret_cast<const uint8_t*>(code) : *reinterpret_cast<const u16_any*>(code);
        uint32_t m, kinds = odd_kinds(mx_up<kBits, 0>(w, mx_scale(*scale)), m);
        kinds = j < lim ? kinds : 0u;
        n = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(u32x4{kinds, 0u, 0u, 0u}), as_bf16x8(u32x4{one, 0u, 0u, 0u}), n, 0, 0, 0);
        if constexpr (kBits == 4) *reinterpret_cast<uint8_t*>(code) = (uint8_t)(w & ~((m & 0x0fu) | (m >> 16 & 0xf0u)));
        else *reinterpret_cast<u16_any*>(code) = (uint16_t)(w & ~((m & 0xffu) | (m >> 16 & 0xff00u)));
        if (*scale == 255) *scale = 0;              // (of all 16 lanes alike)
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) oacc[q][i] = with_odd(oacc[q][i], n[i]);
    }
  }

  // Attends the heads to the unit in buf.  lim: how many of this lane group's tokens count (TG unless kTail).
  template <bool kTail>
  __device__ __forceinline__ void unit(char* buf, const bf16x8* qop, f32x4* oacc, float& m_run, float& l_run, float c,
                                       int lim, uint32_t half) const {
    // All of the unit's operands are read before the first is used, so that one LDS latency passes and not one a
    // tile (the barrier keeps the compiler from moving each read to its use).
    uint32_t scale[kPieces], kw[NT][KW], vw[U::TP][VW], vsc[U::TP][TG / 4], large;
    lds_words<1>(&large, buf + vs_any);
#pragma unroll
    for (int p = 0; p < kPieces; ++p) lds_words<1>(&scale[p], buf + ks + 8 * p);
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int p = 0; p < kPieces; ++p) lds_words<KW / kPieces>(&kw[t][p * (KW / kPieces)], buf + k + 4 * t * MX::kRow + 64 * p);
    auto read_v = [&]() {
#pragma unroll
      for (int q = 0; q < U::TP; ++q) {
        lds_words<TG / 4>(vsc[q], buf + vs + kPage * q);
#pragma unroll
        for (int x = 0; x < VW; x += 4)             // (8 words: tokens 0-7 and 8-15, a unit each)
          lds_words<VW < 4 ? VW : 4>(&vw[q][x], buf + v + 256 * q + x / 4 * (D / 2 * 16));
      }
    };
    read_v();
    __builtin_amdgcn_sched_barrier(0);
    f32x4 s[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    if constexpr (TG < 16) {
#pragma unroll
      for (int p = 0; p < kPieces; ++p) scale[p] >>= k_shift;
    }
#pragma unroll
    for (int kb = 0; kb < U::KB; ++kb) {            // the tiles in turn: no product waits for the one before it
      auto tile = [&](auto t_c) {
        constexpr int t = decltype(t_c)::value;
        if constexpr (t < NT) {
          const float f = mx_scale_of<t>(scale[kPieces == 2 ? kb / 2 : 0]);
          s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(eight_up<kBits>(&kw[t][kb * kBits / 4], f), qop[kb], s[t], 0, 0, 0);
        }
      };
      tile(std::integral_constant<int, 0>{});
      tile(std::integral_constant<int, 1>{});
      tile(std::integral_constant<int, 2>{});
      tile(std::integral_constant<int, 3>{});
    }
    if constexpr (kTail) {                          // keys past the end: by a select, so stray bits never leak
#pragma unroll
      for (int j = 0; j < TG; ++j) s[j / 4][j % 4] = j < lim ? s[j / 4][j % 4] : -INFINITY;
    }
    float p[TG];
    auto weights = [&](float m) {
      float a = 0.f, b = 0.f;
#pragma unroll
      for (int j = 0; j < TG; ++j) {
        p[j] = fexp2(__builtin_fmaf(s[j / 4][j % 4], c, -m));
        if (j & 1) b += p[j]; else a += p[j];
      }
      return a + b;
    };
    constexpr float kMaxSum = 256.0f;               // bounds every weight by 2^8
    float sum = weights(m_run);
    if (__ballot(!(sum <= kMaxSum))) {              // the first unit (m = -inf), or scores far above m
      float mx = s[0][0];
#pragma unroll
      for (int j = 1; j < TG; ++j) mx = fmaxf(mx, s[j / 4][j % 4]);
      mx = fmaxf(mx, __shfl_xor(mx, 16));
      mx = xor32_max(mx);
      const bool grow = mx * c > m_run;
      const float m_new = grow ? mx * c : m_run;
      const float alpha = grow ? fexp2(m_run - m_new) : 1.0f;
      sum = weights(m_new == -INFINITY ? 0.f : m_new);   // (every score so far is minus infinity: weights of 0)
      l_run *= alpha;
#pragma unroll
      for (int q = 0; q < U::TP; ++q) oacc[q] *= alpha;
      m_run = m_new;
    }
    l_run += sum;
    uint32_t pop[TG], rest[TG];                     // the weight's parts at this column's half of each index pair
#pragma unroll
    for (int j = 0; j < TG; ++j) {
      const uint32_t both = twice_bf16(p[j]);
      pop[j] = both & half;
      rest[j] = twice_bf16(p[j] - __builtin_bit_cast(float, both & 0xffff0000u)) & half;
    }
    auto end_v = [&]() {                            // codes and scales past the end become zeros (0 times NaN is NaN)
#pragma unroll
      for (int x = 0; x < TG / 4; ++x) {
        const int left = min(max(lim - 4 * x, 0), 4);
        const uint32_t mask = bytes(left);
#pragma unroll
        for (int q = 0; q < U::TP; ++q) {
          vsc[q][x] &= mask;
          if constexpr (kBits == 4) {
            vw[q][x] &= mask;
          } else {
            vw[q][2 * x] &= left >= 2 ? 0xffffffffu : left == 1 ? 0xffffu : 0u;
            vw[q][2 * x + 1] &= left == 4 ? 0xffffffffu : left == 3 ? 0xffffu : 0u;
          }
        }
      }
    };
    if constexpr (kTail) {
      end_v();
      large &= bytes(lim - vs_tok);
    }
    uint32_t odd = mx_large_scale<kBits>(large);
    if constexpr (kBits == 8) {
      uint32_t nan = 0u;
#pragma unroll
      for (int q = 0; q < U::TP; ++q)
#pragma unroll
        for (int x = 0; x < VW; ++x) nan |= mx_nan_code(vw[q][x]);
      odd |= nan & kMxNanBits;
    }
    if (__builtin_expect(__ballot(odd != 0u) != 0, 0)) {
      take_odd(buf, oacc, lim, half);
      read_v();
      if constexpr (kTail) end_v();
    }
#pragma unroll
    for (int u = 0; u < TG / 4; ++u) {
      bf16x8 x[U::TP];
#pragma unroll
      for (int q = 0; q < U::TP; ++q) {
        const uint32_t w = vsc[q][u];
        const float f0 = mx_scale_of<0>(w), f1 = mx_scale_of<1>(w), f2 = mx_scale_of<2>(w), f3 = mx_scale_of<3>(w);
        if constexpr (kBits == 4) {
          const uint32_t y = vw[q][u];
          x[q] = as_bf16x8(u32x4{mx_up<4, 0>(y, f0), mx_up<4, 1>(y, f1), mx_up<4, 2>(y, f2), mx_up<4, 3>(y, f3)});
        } else {
          const uint32_t y = vw[q][2 * u], z = vw[q][2 * u + 1];
          x[q] = as_bf16x8(u32x4{mx_up<8, 0>(y, f0), mx_up<8, 1>(y, f1), mx_up<8, 0>(z, f2), mx_up<8, 1>(z, f3)});
        }
        oacc[q] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            x[q], as_bf16x8(u32x4{pop[4 * u], pop[4 * u + 1], pop[4 * u + 2], pop[4 * u + 3]}), oacc[q], 0, 0, 0);
      }
#pragma unroll
      for (int q = 0; q < U::TP; ++q)
        oacc[q] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            x[q], as_bf16x8(u32x4{rest[4 * u], rest[4 * u + 1], rest[4 * u + 2], rest[4 * u + 3]}), oacc[q], 0, 0, 0);
    }
  }
};

}  // namespace

template <int D, int kBits>
__global__ __launch_bounds__(kThreads, D * kBits == 256 ? 4 : 2) void decode_mx_kernel(AttnArgs a, DecPlanArgs d) {
  using MX = MxBlock<D, kBits>;
  using U = Unit<D, kBits>;
  constexpr int KB = U::KB, TP = U::TP, kPages = U::kPages;
  // a wave's two buffers, and at its share's end its partials
  constexpr int kStage = 2 * U::kBytes > (int)sizeof(ShareEnd<D>) ? 2 * U::kBytes : (int)sizeof(ShareEnd<D>);
  static_assert(kStage % 16 == 0, "stages stay aligned");
  __shared__ __attribute__((aligned(16))) char stage[kWaves * kStage];
  __shared__ DecPlanLds P;
  __shared__ FinishLds F;
  __shared__ int to_go[kWaves];
  const int lane = threadIdx.x & 63, w = uni(threadIdx.x >> 6);
  const int group = lane >> 4, col = lane & 15, hh = col & 7, odd = col >> 3;
  const int G = a.group, H = a.num_kv_heads, H_q = a.num_q_heads, B = d.batch;

  int most;
  const int total_pages = uni(decode_plan(a, d, P, most));
  if (total_pages < 0) {                            // the prologue cleared the error flag
    if (blockIdx.x == 0 && threadIdx.x == 0) a.ws_hdr[kHdrError] = 1;
    return;
  }
  DecShares<MxCut<D, kBits, kPages>> sh(P, total_pages, most, d);
  DecRun r;
  if (!decode_run(a, d, P, most, total_pages, sh, r)) return;
  const int g = r.g0 + r.j_w;
  const bool head_ok = hh < G && r.j_w >= r.dup;
  const int pages_seen = r.j_w < r.dup ? 1 : a.num_pages;
  const uint32_t half = odd ? 0xffff0000u : 0x0000ffffu;

  f32x4 oacc[TP];
  float m_run = -INFINITY, l_run = 0.f;
  int first_b = -1;                                 // the pair whose end this share holds without its start
  float m_first = 0.f, l_first = 0.f;
  f32x4 o_first[TP];
  bool whole = false;                               // the current pair started inside this share
  PageCursor cur{-1, 0, 1, 1};
#pragma unroll
  for (int p = 0; p < TP; ++p) oacc[p] = o_first[p] = f32x4{0.f, 0.f, 0.f, 0.f};
  char* const st = stage + w * kStage;

  if (r.n > 0) {
    const ConstI32Ptr bt = (ConstI32Ptr)a.block_table;
    const Attend<D, kBits> at(lane);
    const size_t page_bytes = (size_t)H * MX::kBytes;
    const uint8_t* const heads = a.cache + (size_t)g * MX::kBytes;
    struct Ids { int x[kPages]; };
    // a unit: up to kPages pages of the cursor's sequence; `left` pages of the share from its first page on
    auto pages_of = [&](const PageCursor& c, int left) { return min(min(kPages, c.np - c.p), left); };
    auto ids_of = [&](const PageCursor& c, int np) {   // pages past the unit's last one repeat it
      Ids id;
#pragma unroll
      for (int i = 0; i < kPages; ++i)
        id.x[i] = clamp_page(bt[(size_t)c.b * a.bt_stride + c.p + min(i, np - 1)], pages_seen);
      return id;
    };
    const int lane16 = lane * 16;
    constexpr int SC = U::kScaleBytes / 16;         // lanes of a page's scales
    // np pages' copies, np * kCopies + 1 instructions; what a buffer holds in place of the others is masked
    auto send = [&](int buf, Ids id, int np) {
      const unsigned lds = (unsigned)(uintptr_t)((LDS_AS const char*)st) + buf;
      auto page = [&](auto i_c) {
        constexpr int i = decltype(i_c)::value;
        if constexpr (i < kPages) {
          if (i < np) copy_codes<U::kCopies>(heads + (size_t)id.x[i] * page_bytes, lane16, uni(lds + i * U::kPageBytes));
        }
      };
      page(std::integral_constant<int, 0>{});
      page(std::integral_constant<int, 1>{});
      page(std::integral_constant<int, 2>{});
      page(std::integral_constant<int, 3>{});
      int mine = id.x[0];
      if (lane >= SC) mine = id.x[1];
      if constexpr (kPages == 4) {
        if (lane >= 2 * SC) mine = id.x[2];
        if (lane >= 3 * SC) mine = id.x[3];
      }
      if (lane < np * SC)
        copy_scales(heads + (size_t)mine * page_bytes + 2 * MX::kCodes + lane % SC * 16, uni(lds + U::kScales));
    };
    auto send_q = [&](u32x4* q, const PageCursor& c) {
      const uint16_t* row = a.q + ((size_t)c.b * H_q + g * G + min(hh, G - 1)) * D;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) q[kb] = ld16(row + k_channel<D, kBits>(group, kb));
    };
    auto step_past = [&](PageCursor& c, int np) {   // to the unit after (the last of the share goes nowhere)
      c.p += np;
      if (c.p < c.np || c.b + 1 >= B) return;
      c.p = 0;
      ++c.b;
      c.np = uni(P.pre[c.b + 1]) - uni(P.pre[c.b]);
      c.kv = (c.np - 1) * kPage + uni(P.tail[c.b]) + 1;
    };
    u32x4 q_next[KB];
    bf16x8 qop[KB];
    cur = locate(P, r.t0, B);
    int left = r.n, np_cur = pages_of(cur, left);
    Ids id = ids_of(cur, np_cur);
    send_q(q_next, cur);
    send(0, id, np_cur);
    bool fresh = true;                              // the unit is the first of its pair in this share
    PageCursor nxt = cur;
    step_past(nxt, np_cur);
    int np_nxt = pages_of(nxt, left - np_cur);
    if (left > np_cur) id = ids_of(nxt, np_nxt);
    int buf = 0;
    for (;;) {
      // A SIMD's two waves (w and w ^ 4) keep pace: the one with more left issues first (without it 64 sequences of
      // 2K-16K tokens took 124 us in 4 bits, so 120).
      if (lane == 0) *(volatile int*)&to_go[w] = left;
      if (uni(*(volatile int*)&to_go[w ^ 4]) < left) __builtin_amdgcn_s_setprio(1);
      else __builtin_amdgcn_s_setprio(0);
      if (fresh) {
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) qop[kb] = hh < G ? as_bf16x8(q_next[kb]) : zero_bf16x8();
#pragma unroll
        for (int p = 0; p < TP; ++p) oacc[p] = f32x4{0.f, 0.f, 0.f, 0.f};
        m_run = -INFINITY;
        l_run = 0.f;
        whole = cur.p == 0;
      }
      // the next unit's copies go out (its buffer's last reads are complete), then this one's are waited for
      const bool more = left > np_cur;
      PageCursor nn = nxt;
      int np_nn = 0;
      if (more) {
        if (nxt.p == 0) send_q(q_next, nxt);
        __builtin_amdgcn_s_waitcnt(PEARL_LGKMCNT0);
        send(buf ^ U::kBytes, id, np_nxt);
        step_past(nn, np_nxt);
        np_nn = pages_of(nn, left - np_cur - np_nxt);
        if (left > np_cur + np_nxt) id = ids_of(nn, np_nn);
        constexpr int C = U::kCopies;
        if (np_nxt == kPages) __asm__ volatile("s_waitcnt vmcnt(%0)" ::"n"(kPages * C + 1) : "memory");
        else if (np_nxt == 1) __asm__ volatile("s_waitcnt vmcnt(%0)" ::"n"(C + 1) : "memory");
        else if (np_nxt == 2) __asm__ volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * C + 1) : "memory");
        else __asm__ volatile("s_waitcnt vmcnt(%0)" ::"n"(3 * C + 1) : "memory");
      } else {
        __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory");
      }
      if (np_cur == kPages && (cur.p + kPages) * kPage <= cur.kv)
        at.template unit<false>(st + buf, qop, oacc, m_run, l_run, a.scale_log2, U::TG, half);
      else
        at.template unit<true>(st + buf, qop, oacc, m_run, l_run, a.scale_log2,
                               min(cur.kv - cur.p * kPage, np_cur * kPage) - group * U::TG, half);
      const bool ends_here = cur.p + np_cur == cur.np;
      if (ends_here) {
        l_run += __shfl_xor(l_run, 16);
        l_run += __shfl_xor(l_run, 32);
        if (whole) {
          const size_t row = (size_t)cur.b * H_q + g * G + hh;
          const float inv = 1.0f / l_run;
#pragma unroll
          for (int p = 0; p < TP; ++p) {
            u32x4 x;
#pragma unroll
            for (int i = 0; i < 4; ++i) {           // the odd channels from the lane 8 columns on
              const float mine = oacc[p][i] * inv;  // (a bit cast of the element itself takes element 0)
              const int other = __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, mine), 0x128, 0xf, 0xf, false);   // row_ror:8
              x[i] = (uint32_t)bf16_bits(mine) | ((uint32_t)bf16_bits(__builtin_bit_cast(float, other)) << 16);
            }
            if (head_ok && !odd) *reinterpret_cast<u32x4*>(a.out + row * D + 32 * p + 8 * group) = x;
          }
          if (head_ok && lane < 8 && a.lse) a.lse[row] = (m_run + flog2(l_run)) * kLn2;
        } else {                                    // only the first pair can have started earlier
#pragma unroll
          for (int p = 0; p < TP; ++p) o_first[p] = oacc[p];
          m_first = m_run;
          l_first = l_run;
          first_b = cur.b;
        }
      }
      fresh = ends_here;
      left -= np_cur;
      if (!more) {
        if (ends_here) cur.b = -1;                  // the share ends with the pair's end
        break;
      }
      cur = nxt;
      np_cur = np_nxt;
      nxt = nn;
      np_nxt = np_nn;
      buf ^= U::kBytes;
    }
    if (cur.b >= 0) {
      l_run += __shfl_xor(l_run, 16);
      l_run += __shfl_xor(l_run, 32);
    }
  }

  // A kv-head of its own for every wave: its share is the run, so it finishes by itself.  Its partials go to the workspace
  // from the registers, it counts itself in on their pairs and merges those whose last it is; no wave waits for another one.
  // (8 kv-heads and 4 bits, through LDS and together as below and so: 64 sequences of 2K-16K tokens 115.7 and 112.8 us, at
  // d = 64 256 of 200-3000 58.9 and 57.9.  Where waves share a kv-head, below wins, as it joins them first: 4 bits, 2
  // kv-heads, 256 sequences of 1K-8K tokens 64.9 us, with every share a run of its own 69.0; 8 bits, 4 kv-heads, 200 of
  // 300-3000 71.0 and 76.2.)
  if (sh.heads == kWaves) {
    if (r.n <= 0 || r.j_w < r.dup) return;
    CutPair cut[2];
    auto store = [&](int b, const f32x4* o, float m, float l) {
      const int second = uni(P.pre[b]) > r.t0;
      const int own = second ? (r.per_pair ? sh.n_runs + b : 2 * r.x + 1) : r.slot_stride * r.x;
      float* to = a.part_o + (((size_t)g * d.max_dec + own) * G + hh) * D + 8 * group + 4 * odd;
#pragma unroll
      for (int p = 0; p < TP; ++p) {                // four channels from either column half: a group's 8 are 32 bytes
        float mine[2], other[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float give = odd ? o[p][i] : o[p][2 + i];
          mine[i] = odd ? o[p][2 + i] : o[p][i];
          other[i] = __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, give), 0x128, 0xf, 0xf, false));   // row_ror:8
        }
        const f32x4 x = odd ? f32x4{other[0], mine[0], other[1], mine[1]} : f32x4{mine[0], other[0], mine[1], other[1]};
        if (hh < G) st_dev4(to + 32 * p, x);
      }
      if (hh < G && lane < 8) st_dev2(&a.part_ml[2 * (((size_t)g * d.max_dec + own) * G + hh)], m, l);
      return sh.cut_of(P, r, b);
    };
    cut[0].b = cut[1].b = -1;
    if (first_b >= 0) cut[0] = store(first_b, o_first, m_first, l_first);
    if (cur.b >= 0) cut[1] = store(cur.b, oacc, m_run, l_run);
    __builtin_amdgcn_s_waitcnt(PEARL_VMCNT(0));     // the stores are acknowledged before the wave counts itself in
    int seen = -1;
    const int b_mine = lane == 0 ? cut[0].b : cut[1].b, x_mine = lane == 0 ? cut[0].x0 : cut[1].x0;
    if (lane < 2 && b_mine >= 0)
      seen = __hip_atomic_fetch_add(&a.split_cnt[r.per_pair ? g * B + b_mine : g * sh.n_runs + x_mine], 1, __ATOMIC_RELAXED,
                                    __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll 1
    for (int which = 0; which < 2; ++which) {
      const CutPair c = which == 0 ? cut[0] : cut[1];
      if (c.b < 0 || __builtin_amdgcn_readlane(seen, which) != c.n - 1) continue;
      for (int pass = 0; pass < (G + 3) / 4; ++pass) merge_pair<D>(a, c, g, r.slot_stride, d.max_dec, pass);
    }
    return;
  }

  // the waves' partials, merged per pair through LDS
  ShareEnd<D>& E = *reinterpret_cast<ShareEnd<D>*>(st);
  auto leave = [&](int which, const f32x4* o, float m, float l) {
#pragma unroll
    for (int p = 0; p < TP; ++p)
#pragma unroll
      for (int i = 0; i < 4; ++i) E.o[which][hh][32 * p + 8 * group + 2 * i + odd] = o[p][i];
    if (lane < 8) { E.ml[which][hh][0] = m; E.ml[which][hh][1] = l; }
  };
  if (head_ok) {
    if (first_b >= 0) leave(0, o_first, m_first, l_first);
    if (cur.b >= 0) leave(1, oacc, m_run, l_run);
  }
  finish_shares<D>(a, d, P, sh, r, stage, kStage, SharePairs{first_b, cur.b, !whole, r.n > 0}, F);
}

// ------------------------------------------------------------------------------------------------
// host launchers
// ------------------------------------------------------------------------------------------------
namespace {
typedef void (*DecodeMx)(AttnArgs, DecPlanArgs);
DecodeMx decode_mx_of(int head_dim, int bits) {
  return head_dim == 64 ? (bits == 4 ? decode_mx_kernel<64, 4> : decode_mx_kernel<64, 8>)
                        : (bits == 4 ? decode_mx_kernel<128, 4> : decode_mx_kernel<128, 8>);
}
}  // namespace

int decode_mx_grid(int head_dim, int bits) {
  // workgroups a compute unit holds, per kernel: the same on every device that runs gfx950 code
  static std::atomic<int> held[2][2];
  std::atomic<int>& h = held[head_dim == 128][bits == 8];
  int occ = h.load(std::memory_order_relaxed);
  if (occ == 0) {
    if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&occ, decode_mx_of(head_dim, bits), kThreads, 0) != hipSuccess || occ < 1) occ = 1;
    h.store(occ, std::memory_order_relaxed);
  }
  return device_num_cu() * occ;
}

hipError_t launch_decode_mx(const AttnArgs& a, const DecPlanArgs& d, int head_dim, int bits, hipStream_t stream) {
  hipLaunchKernelGGL(decode_mx_of(head_dim, bits), dim3((unsigned)d.grid), dim3(kThreads), 0, stream, a, d);
  return hipGetLastError();
}

}  // namespace pearl
