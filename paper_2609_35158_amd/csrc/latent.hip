// gfx950 kernels of attention over a paged cache of latent vectors (absorbed form; paper, section 4.3, Eq. 1: decode
// is bound by its cache reads, which one short row a token for all heads makes few).
//
// A cached row is (c, r), DC + DR channels; a query row (token, head) is (q_c, q_r).  s_j = scale q . (c_j, r_j), over
// keys j up to the token's position, o = sum softmax(s)_j c_j: the row is the key of every head and its latent part the
// value.  So the rows of a tile are any (token, head) pairs of a sequence, in the order of q: row rho is token rho / H, head
// rho % H.  The softmax is online, in base 2, with state in 32 bits; weights enter the second product in bf16.
//
// A workgroup of 4 waves takes M rows and stages of 64 keys (4 pages):
//   S^T (keys x rows) = K . Q^T: Q stays in registers.  M = 16 or 32: wave w takes the keys of page w for all rows; M = 64: 32 keys
//                       for 32 rows, so that K is read from LDS twice, with half the registers for Q;
//   O^T (channels x rows) += V^T . P^T: wave w takes a quarter of the channels, V^T by transposing reads of the same LDS
//                       rows, once; P goes through LDS, 2 bytes a weight.
// MFMA layouts (lane l): 16x16x32 (M = 16, 32): A row l%16, k 8(l/16)+e; B column l%16, k 8(l/16)+e; D column l%16, row
// 4(l/16)+r.  32x32x16 (M = 64): A row l%32, k 8(l/32)+e; B column l%32, k 8(l/32)+e; D column l%32, row r%4 + 8(r/4) + 4(l/32).
// At M = 64 a wave has its SIMD to itself, in order, and what bounds it is the number of its instructions: hence the larger
// products, two copies a group, and operand addresses that differ in constants.
// A row's maximum is common to the waves.  It may lag the true one by kLag (log2 units), so most stages go on with the old one; where
// some score is further above, a wave weighs with a maximum of its own, and the waves join theirs behind the barrier that they meet at for
// the weights anyway.
//
// Work is cut into equal shares of keys, in the order (sequence, tile, key), on the device from the lengths: each
// workgroup finds its share by itself.  A tile cut by shares leaves (o~, m, l) in the workspace, joined by
// latent_merge_kernel.  `group` workgroups next to one another on an XCD take neighbouring tiles of the same share, so that
// they read the same keys at the same time, from L2.

#include "attn_device.h"

#include <float.h>

#include <type_traits>

namespace pearl {
namespace {

constexpr int kLatWaves = 4;
constexpr int kLatThreads = 64 * kLatWaves;
constexpr int kLatKeys = kLatWaves * kPage;         // of a stage
constexpr float kLag = 8.f;

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ void barrier_lds() { __asm__ volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
__device__ __forceinline__ void wait_copies() { __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

__device__ __forceinline__ float xor16_max(float x) {
  const unsigned u = __builtin_bit_cast(unsigned, x);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return fmaxf(__builtin_bit_cast(float, (unsigned)r[0]), __builtin_bit_cast(float, (unsigned)r[1]));
}
__device__ __forceinline__ float xor16_add(float x) {
  const unsigned u = __builtin_bit_cast(unsigned, x);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
}

// Keep a value in vector or in accumulation registers at this place.  The outputs stay in vector registers, which the rare stages that
// scale them need, and the queries in accumulation registers, from which the products read them; left to itself the compiler moves
// the outputs between the two in every stage.
template <typename T> __device__ __forceinline__ void in_vector(T& x) { __asm__ volatile("" : "+v"(x)); }
__device__ __forceinline__ void in_acc(bf16x8& x) { __asm__ volatile("" : "+a"(x)); }

// The kernel's arguments, read anew where they are used outside the stages: kept over them, they would be spilled.
typedef const __attribute__((address_space(4))) LatentArgs* LatArgsPtr;
__device__ __forceinline__ LatArgsPtr args_anew() {
  LatArgsPtr p = (LatArgsPtr)__builtin_amdgcn_kernarg_segment_ptr();
  __asm__ volatile("" : "+s"(p));
  return p;
}

__device__ __forceinline__ unsigned lds_address(const char* p) { return (unsigned)(uintptr_t)((LDS_AS const char*)p); }

__device__ __forceinline__ long long uni64(long long x) {
  const unsigned lo = uni((int)x), hi = uni((int)(x >> 32));
  return (long long)((unsigned long long)hi << 32 | lo);
}

// A page in LDS: 16 rows of DC channels, then 16 rows of DR.  Chunk (16 bytes) c of latent row r is in slot c ^ f(r) of
// its 16, f a permutation of the rows, so that the row reads of 16 lanes fall into 16 slots.  The transposing reads of 32 lanes take two
// chunks of each of 8 consecutive rows at M = 16 (kWide false), four chunks of 4 consecutive rows at M = 64: f keeps these apart likewise.
// Chunks of the rotated part are in slot c ^ (r / 2) (DR = 64; 32: r / 4), where 2 (4) rows share the banks.
template <int DC, int DR, bool kWide> struct LatPage {
  static constexpr int kWidth = (DC + DR) * 2;      // bytes of a cached row
  static constexpr int kRowBytes = DC * 2, kRotBytes = DR * 2;
  static constexpr int kRot = kPage * kRowBytes;    // offset of the rotated parts
  static constexpr int kBytes = kPage * kWidth;
  static_assert(kBytes % 256 == 0 && kRowBytes % 256 == 0, "the swizzle takes address bits 4 .. 7");
  __device__ static __forceinline__ constexpr int f(int r) {
    return kWide ? ((r & 3) << 2) | ((r >> 2) & 3) : ((r & 7) << 1) | (r >> 3);
  }
  __device__ static __forceinline__ constexpr int rot_f(int r) { return DR == 64 ? (r >> 1) & 7 : (r >> 2) & 3; }
};

// The copies of a page by a wave, 1 KiB an instruction, kRows rows' latent parts each, and then the rotated parts.
// kWide: as LatPage's; without it, where a key is read by one workgroup, the copies go past the caches (nt).
template <int DC, int DR, bool kWide> struct LatCopies {
  using Page = LatPage<DC, DR, kWide>;
  static constexpr int kRows = 1024 / Page::kRowBytes;
  static constexpr int kLatent = kPage / kRows, kCopies = kLatent + kPage * Page::kRotBytes / 1024;
  static_assert(kLatent % 2 == 0 && Page::kWidth % 32 == 0 && (DR == 32 || Page::kWidth % 128 == 0), "copies in pairs; the swizzle's bits");

  // The lane's source offset in the page, of copy i.
  __device__ static __forceinline__ int offset(int i) {
    const int l = threadIdx.x & 63;
    if (i < kLatent) {
      const int r = kRows * i + (kRows == 2 ? l >> 5 : 0), slot = kRows == 2 ? l & 31 : l;
      return r * Page::kWidth + 16 * (slot ^ Page::f(r));
    }
    constexpr int kChunks = Page::kRotBytes / 16;
    const int r = (64 * (i - kLatent) + l) / kChunks;
    return r * Page::kWidth + Page::kRowBytes + 16 * ((l % kChunks) ^ Page::rot_f(r));
  }

  // Copies i and (if there is one) i + 1 of the page at src to the page at the LDS address lds, if `go`.  The branch is the
  // instructions' own: one that the compiler sees splits the products' code in two, with moves of all outputs between them.  An
  // instruction's immediate offset advances both addresses.  (i is a constant where this is inlined.)
  __device__ static __forceinline__ void copy2(int i, const char* src, unsigned lds, int go) {
    const unsigned to = uni((int)lds + 1024 * i);
#define PEARL_LATENT_COPY(SECOND, NT)                                                                                          \
  __asm__ volatile("s_cmp_eq_u32 %4, 0\n\t"                                                                                    \
                   "s_cbranch_scc1 .Lno_copy%=\n\t"                                                                            \
                   "s_mov_b32 m0, %3\n\t"                                                                                      \
                   "s_nop 0\n\t"                                                                                               \
                   "global_load_lds_dwordx4 %0, %2" NT "\n\t" SECOND ".Lno_copy%=:"                                           \
                   :                                                                                                           \
                   : "v"(offset(i)), "v"(offset(i + 1) - 1024), "s"(src), "s"(to), "s"(uni(go))                                \
                   : "memory", "scc", "m0")
    if (kWide) {
      if (i + 1 < kCopies) PEARL_LATENT_COPY("global_load_lds_dwordx4 %1, %2 offset:1024\n", "");
      else PEARL_LATENT_COPY("", "");
    } else {
      if (i + 1 < kCopies) PEARL_LATENT_COPY("global_load_lds_dwordx4 %1, %2 offset:1024 nt\n", " nt");
      else PEARL_LATENT_COPY("", " nt");
    }
#undef PEARL_LATENT_COPY
  }

  __device__ static __forceinline__ void page(const char* src, unsigned lds) {
#pragma unroll
    for (int i = 0; i < kCopies; i += 2) copy2(i, src, lds, 1);
  }

  // Zeros in place of the rows from `valid` on.
  __device__ static __forceinline__ void clear(char* page, int valid) {
    const int l = threadIdx.x & 63;
    for (int i = valid * Page::kRowBytes + 16 * l; i < Page::kRot; i += 1024) *reinterpret_cast<u32x4*>(page + i) = u32x4{0u, 0u, 0u, 0u};
    for (int i = Page::kRot + valid * Page::kRotBytes + 16 * l; i < Page::kBytes; i += 1024)
      *reinterpret_cast<u32x4*>(page + i) = u32x4{0u, 0u, 0u, 0u};
  }
};

// What finding a workgroup's share takes.
struct LatFind {
  long long sum[kLatWaves], before;
  int found, bad;
};

// Both kernels' notes on a tile.
template <int DC, int M> struct LatNotes {
  int odd[DC];                                      // of each channel: the first key with a value that is not finite and ..
  int any_odd;                                      // .. whether there is one, among those that only some of the tile's rows see
  int limit[M];                                     // the last key that a row sees
};

template <int DC, int DR> struct LatLds16 {
  char page[kLatWaves][2][LatPage<DC, DR, false>::kBytes];   // at the end of a tile: the waves' outputs
  LatNotes<DC, 16> notes;
  float max[kLatWaves][16], sum[kLatWaves][16];
  LatFind find;
};

template <int DC, int DR> struct LatLds64 {
  static constexpr int kStage = kLatWaves * LatPage<DC, DR, true>::kBytes;
  char stage[2][kStage];
  char p[64 * kLatKeys * 2];                        // weights: rows of 128 bytes, chunk c of row r in slot c ^ (r / 2)
  LatNotes<DC, 64> notes;
  float max[2][64];                                 // a row's maximum in each half of the keys; at the end its sums
  int flag[2];                                      // some score is far above its row's maximum; one a stage in turn
  LatFind find;
};

// M = 16: what a wave holds of a tile, of which it has all rows and every fourth page.
template <int DC, int DR> struct LatRows16 {
  static constexpr int M = 16;
  using Page = LatPage<DC, DR, false>;
  using Copies = LatCopies<DC, DR, false>;
  static constexpr int kSteps = DC / 32, kAll = kSteps + DR / 32;
  static constexpr int kBlocks = DC / 16;           // of 16 channels
  static constexpr int kAhead = 4;                  // LDS reads of the products' operands, ahead of them
  bf16x8 q[kAll];
  f32x4 o[kBlocks], s;
  float m, l;
  int g16, l16;

  __device__ __forceinline__ void start(const uint16_t* rows, int n_rows) {
    g16 = (threadIdx.x & 63) >> 4;
    l16 = threadIdx.x & 15;
    const uint16_t* const src = rows + min(l16, n_rows - 1) * (size_t)(DC + DR) + 8 * g16;
#pragma unroll
    for (int k = 0; k < kAll; ++k) q[k] = as_bf16x8(ld16(src + 32 * k));
    m = -FLT_MAX;
    l = 0.f;
#pragma unroll
    for (int d = 0; d < kBlocks; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  __device__ __forceinline__ void pin_queries() {
#pragma unroll
    for (int k = 0; k < kAll; ++k) in_acc(q[k]);
  }
  __device__ __forceinline__ void scores(const char* page) {
    // of the lane's first chunk; those of the steps after it differ in address bits 6 and 7, and by whole 256 bytes
    const int at = l16 * Page::kRowBytes + 16 * (g16 ^ Page::f(l16)), rot = Page::kRot + l16 * Page::kRotBytes + 16 * (g16 ^ Page::rot_f(l16));
    auto key_of = [&](int k) {
      return as_bf16x8(*reinterpret_cast<const u32x4*>(page + (k < kSteps ? (at ^ (64 * (k & 3))) + 256 * (k >> 2) : rot ^ (64 * (k - kSteps)))));
    };
    bf16x8 key[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) key[k] = key_of(k);
    s = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < kAll; ++k) {
      s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(key[k % kAhead], q[k], s, 0, 0, 0);
      if (k + kAhead < kAll) key[k % kAhead] = key_of(k + kAhead);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  __device__ __forceinline__ void mask(const int* limits, int key0) {
    const int limit = limits[l16];
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (key0 + 4 * g16 + r > limit) s[r] = -__builtin_inff();
  }
  __device__ __forceinline__ float largest() const { return fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])); }
  // Whether some score is far above its row's maximum so far; the new maximum.
  __device__ __forceinline__ bool above(float scale) const { return __ballot(fmaf(largest(), scale, -m) > kLag) != 0; }
  __device__ __forceinline__ void raise(float scale) {
    const float x = fmaxf(m, xor32_max(xor16_max(largest() * scale)));
    scale_to(x);
  }
  __device__ __forceinline__ void scale_to(float x) {
    const float alpha = fexp2(m - x);
    m = x;
    l *= alpha;
#pragma unroll
    for (int d = 0; d < kBlocks; ++d) o[d] *= alpha;
  }
  __device__ __forceinline__ void add_values(const char* page, float scale) {
    // The weights of the lane's row and keys 4 g16 .. + 3 are where the product (16x16x16: A row l%16, k 4(l/16)+e; B column l%16, k
    // 4(l/16)+e) takes them.  Of the values the lane addresses row 4 g16 + l16 / 4, four channels of block 0.
    const int r = 4 * g16 + (l16 >> 2), at = r * Page::kRowBytes + 16 * (((l16 >> 1) & 1) ^ Page::f(r)) + 8 * (l16 & 1);
    auto value_of = [&](int d) { return lds_read_tr(page, (at ^ (32 * (d & 7))) + 256 * (d >> 3)); };
    i16x4 value[kAhead];
#pragma unroll
    for (int d = 0; d < kAhead; ++d) value[d] = value_of(d);
    float x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = fexp2(fmaf(s[i], scale, -m));
    l += (x[0] + x[1]) + (x[2] + x[3]);
    const i16x4 p = __builtin_bit_cast(i16x4, bf16x4{(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]});
#pragma unroll
    for (int d = 0; d < kBlocks; ++d) {
      o[d] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(value[d % kAhead], p, o[d], 0, 0, 0);
      if (d + kAhead < kBlocks) value[d % kAhead] = value_of(d + kAhead);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
};

// M = 64: what a wave holds of a tile, and its parts of a stage.
template <int DC, int DR> struct LatRows64 {
  static constexpr int M = 64;
  using Page = LatPage<DC, DR, true>;
  using Copies = LatCopies<DC, DR, true>;
  using Lds = LatLds64<DC, DR>;
  static constexpr int kSteps = DC / 16, kAll = kSteps + DR / 16;
  static constexpr int kTiles = DC / kLatWaves / 32;    // of 32 channels
  static constexpr int kAhead = 4;
  bf16x8 q[kAll];                                   // of the wave's 32 rows
  f32x16 o[kTiles][2], s;                           // outputs of all rows
  float m[2], l, sum, ref, factor[2][2];            // m: of the lane's row in both halves
  int w, half, l32;                                 // wave w has the scores of keys 32 (w / 2) .. and rows 32 (w % 2) ..

  __device__ __forceinline__ int own() const { return 32 * (w & 1) + l32; }
  __device__ __forceinline__ float own_max() const { return w & 1 ? m[1] : m[0]; }
  __device__ __forceinline__ void start(int wave, const uint16_t* rows, int n_rows) {
    w = wave;
    half = (threadIdx.x & 63) >> 5;
    l32 = threadIdx.x & 31;
    const uint16_t* const src = rows + min(own(), n_rows - 1) * (size_t)(DC + DR) + 8 * half;
#pragma unroll
    for (int k = 0; k < kAll; ++k) q[k] = as_bf16x8(ld16(src + 16 * k));
    m[0] = m[1] = -FLT_MAX;
    l = 0.f;
#pragma unroll
    for (int d = 0; d < kTiles; ++d)
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][t][r] = 0.f;
  }
  __device__ __forceinline__ void pin_queries() {
#pragma unroll
    for (int k = 0; k < kAll; ++k) in_acc(q[k]);
  }
  __device__ __forceinline__ void pin_outputs() {
#pragma unroll
    for (int d = 0; d < kTiles; ++d) {
      in_vector(o[d][0]);
      in_vector(o[d][1]);
    }
  }
  template <typename Next> __device__ __forceinline__ void scores(const char* stage, Next&& next_copies) {
    const char* const pages = stage + 2 * (w >> 1) * Page::kBytes;
    // of the lane's first chunk; those of the steps after it differ in address bits 5 .. 7, and by whole 256 bytes
    const int r = l32 & 15, page = (l32 >> 4) * Page::kBytes;
    const int at = page + r * Page::kRowBytes + 16 * (half ^ Page::f(r)), rot = page + Page::kRot + r * Page::kRotBytes + 16 * (half ^ Page::rot_f(r));
    auto key_of = [&](int k) {
      return as_bf16x8(*reinterpret_cast<const u32x4*>(pages + (k < kSteps ? (at ^ (32 * (k & 7))) + 256 * (k >> 3) : rot ^ (32 * (k - kSteps)))));
    };
    bf16x8 key[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) key[k] = key_of(k);
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
    for (int k = 0; k < kAll; ++k) {
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(key[k % kAhead], q[k], s, 0, 0, 0);
      if (k + kAhead < kAll) key[k % kAhead] = key_of(k + kAhead);
      if (k % 4 == 1) next_copies(k / 2);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  __device__ __forceinline__ void mask(const Lds& lds, int key0) {
    const int key = key0 + 32 * (w >> 1) + 4 * half, limit = lds.notes.limit[own()];
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (key + (i & 3) + 8 * (i >> 2) > limit) s[i] = -__builtin_inff();
  }
  __device__ __forceinline__ float largest() const {
    float x = fmaxf(s[0], s[1]);
#pragma unroll
    for (int i = 2; i < 16; i += 2) x = fmaxf(x, fmaxf(s[i], s[i + 1]));
    return x;
  }
  __device__ __forceinline__ void weigh(Lds& lds, int stage, float scale) {
    ref = own_max();
    const float top = largest();
    if (__ballot(fmaf(top, scale, -ref) > kLag)) {
      ref = fmaxf(ref, ceilf(xor32_max(top * scale)));
      lds.flag[stage & 1] = 1;
    }
    char* const to = lds.p + own() * 128 + 8 * half;
    sum = 0.f;
#pragma unroll
    for (int a = 0; a < 4; ++a) {
      float p[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) p[r] = fexp2(fmaf(s[4 * a + r], scale, -ref));
      sum += (p[0] + p[1]) + (p[2] + p[3]);
      *reinterpret_cast<bf16x4*>(to + 16 * ((4 * (w >> 1) + a) ^ ((l32 >> 1) & 7))) = bf16x4{(__bf16)p[0], (__bf16)p[1], (__bf16)p[2], (__bf16)p[3]};
    }
    if (half == 0) lds.max[w >> 1][own()] = ref;
  }
  __device__ __forceinline__ void join(const Lds& lds) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const float a = lds.max[0][32 * t + l32], b = lds.max[1][32 * t + l32], x = fmaxf(a, b), alpha = fexp2(m[t] - x);
      m[t] = x;
      if (t == (w & 1)) {
        l *= alpha;
        sum *= fexp2(ref - x);
      }
      factor[0][t] = fexp2(a - x);
      factor[1][t] = fexp2(b - x);
#pragma unroll
      for (int d = 0; d < kTiles; ++d) o[d][t] *= alpha;
    }
  }
  template <bool kScaled> __device__ __forceinline__ void add_values(const Lds& lds, const char* stage) {
    l += sum;
    // The lane's row of 8 (l / 32) + 0 .. 3 of the values, channels of tile 0; four rows further the swizzle differs in chunk bit 0.
    const int j = l32 & 15, r = 8 * half + (j >> 2), c = DC / 32 * w + 2 * (l32 >> 4) + ((j >> 1) & 1);
    const int at = r * Page::kRowBytes + 16 * ((c & ~15) | ((c & 15) ^ Page::f(r))) + 8 * (j & 1), at4 = (at ^ 16) + 4 * Page::kRowBytes;
    const int from = l32 * 128 + 16 * (half ^ ((l32 >> 1) & 7));
    constexpr int kParts = kLatWaves * kTiles;      // (page, tile), tiles of a page in turn
    auto value_of = [&](int i) {
      const char* const page = stage + i / kTiles * Page::kBytes;
      return concat_tr(lds_read_tr(page, at ^ (64 * (i % kTiles))), lds_read_tr(page, at4 ^ (64 * (i % kTiles))));
    };
    auto weights_of = [&](int page, int t) {
      bf16x8 p = as_bf16x8(*reinterpret_cast<const u32x4*>(lds.p + 4096 * t + (from ^ (32 * page))));
      if constexpr (kScaled)
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = (__bf16)((float)p[e] * factor[page >> 1][t]);
      return p;
    };
    bf16x8 p[2][2], value[kAhead];                  // p: of this page and the next one
    p[0][0] = weights_of(0, 0);
    p[0][1] = weights_of(0, 1);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) value[i] = value_of(i);
#pragma unroll
    for (int i = 0; i < kParts; ++i) {
      const int page = i / kTiles, d = i % kTiles;
      if (d == 0 && page + 1 < kLatWaves) {
        p[(page + 1) & 1][0] = weights_of(page + 1, 0);
        p[(page + 1) & 1][1] = weights_of(page + 1, 1);
      }
      const bf16x8 x = value[i % kAhead];
      o[d][0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, p[page & 1][0], o[d][0], 0, 0, 0);
      o[d][1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, p[page & 1][1], o[d][1], 0, 0, 0);
      if (i + kAhead < kParts) value[i % kAhead] = value_of(i + kAhead);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  __device__ __forceinline__ void set_odd(const Lds& lds) {
#pragma unroll
    for (int d = 0; d < kTiles; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int first = lds.notes.odd[DC / kLatWaves * w + 32 * d + (i & 3) + 8 * (i >> 2) + 4 * half];
#pragma unroll
        for (int t = 0; t < 2; ++t)
          if (first <= lds.notes.limit[32 * t + l32]) o[d][t][i] = __builtin_nanf("");
      }
  }
  __device__ __forceinline__ void sums(Lds& lds) {
    const float x = xor32_add(l);
    if (half == 0) lds.max[w >> 1][own()] = x;
  }
  template <typename F> __device__ __forceinline__ void each(const Lds& lds, F&& f) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int r = 32 * t + l32;
      f(r, m[t], lds.max[0][r] + lds.max[1][r], w == 0 && half == 0, [&](auto&& put) {
#pragma unroll
        for (int d = 0; d < kTiles; ++d)
#pragma unroll
          for (int a = 0; a < 4; ++a)
            put(DC / kLatWaves * w + 32 * d + 8 * a + 4 * half, f32x4{o[d][t][4 * a], o[d][t][4 * a + 1], o[d][t][4 * a + 2], o[d][t][4 * a + 3]});
      });
    }
  }
};

// ---- the plan --------------------------------------------------------------------------------------------------------
// A sequence's rows are cut into tiles of `tile_rows` (group * M).  Work is measured in keys: tile u costs its keys, kTileCost and
// what its rows add, such that the cost of tiles 0 .. u - 1 is u (ctx + kTileCost) + (u (u + 1) slope >> 8), slope
// being 256 times half the tokens of a tile.
constexpr int kTileCost = 64;

struct LatSeq {
  int q_start, q_len, ctx;
};

struct LatPlan {
  int tile_rows, slope, heads;
  __device__ __forceinline__ long long before(const LatSeq& s, long long u) const {
    return u * (s.ctx + kTileCost) + ((u * (u + 1) * slope) >> 8);
  }
  __device__ __forceinline__ int tiles(const LatSeq& s) const {
    return (int)(((long long)s.q_len * heads + tile_rows - 1) / tile_rows);
  }
  // stages of the keys that rows up to `row` see
  __device__ __forceinline__ int stages(const LatSeq& s, int row) const {
    return (s.ctx + row / heads + 1 + kLatKeys - 1) / kLatKeys;
  }
  // the stage at which cost `at` of a tile that starts at 0 is cut
  __device__ __forceinline__ static int stage_at(long long at, int stages) {
    const long long j = (at - kTileCost) / kLatKeys;
    return j < 0 ? 0 : j > stages ? stages : (int)j;
  }
  // the tile that cost `at` of a sequence falls into
  __device__ __forceinline__ int tile_at(const LatSeq& s, long long at) const {
    int lo = 0, hi = tiles(s);                      // before(lo) <= at < before(hi)
    while (hi - lo > 1) {
      const int mid = lo + (hi - lo) / 2;
      if (before(s, mid) <= at) lo = mid;
      else hi = mid;
    }
    return lo;
  }
};

// `total` cut into `shares`, which differ by 1 at most.
struct LatShares {
  long long each;
  int more, shares;                                 // the first `more` are one longer
  LatShares() = default;
  __device__ __forceinline__ LatShares(long long total, int n) : each(total / n), more((int)(total - each * n)), shares(n) {}
  __device__ __forceinline__ long long start(int s) const { return each * s + min(s, more); }
  // the share that position `at` is in
  __device__ __forceinline__ int of(long long at) const {
    int s = min((int)((float)at / (float)each), shares - 1);   // off by 1 at most
    while (s > 0 && start(s) > at) --s;
    while (s + 1 < shares && start(s + 1) <= at) ++s;
    return s;
  }
};

__device__ __forceinline__ LatSeq lat_seq(const LatentArgs& a, int b) {
  if (!a.cu) return LatSeq{b, 1, a.ctx_lens[b]};
  const int start = a.cu[b];
  return LatSeq{start, a.cu[b + 1] - start, a.ctx_lens[b]};
}

// The same of one sequence for the whole wave, in scalar registers.
__device__ __forceinline__ LatSeq lat_seq_uni(const LatentArgs& a, int b) {
  const LatSeq s = lat_seq(a, b);
  return LatSeq{uni(s.q_start), uni(s.q_len), uni(s.ctx)};
}

__device__ __forceinline__ bool lat_bad(const LatentArgs& a, const LatSeq& s) {
  const long long kv = (long long)s.ctx + s.q_len;
  return s.q_len < 0 || s.ctx < 0 || s.q_start < 0 || s.q_len > a.max_q_len || (long long)s.q_start + s.q_len > a.total_q ||
         kv > a.max_kv_len || (kv + kPage - 1) / kPage > a.bt_stride;
}

__device__ __forceinline__ long long shfl_up64(long long x, int d) {
  const int lo = __shfl_up((int)x, d), hi = __shfl_up((int)(x >> 32), d);
  return (long long)(((unsigned long long)(unsigned)hi << 32) | (unsigned)lo);
}

// A workgroup's work: the tiles of its share, of each the workgroup's member and the stages.
struct LatWork {
  LatPlan plan;
  LatShares cut;
  LatSeq seq;
  long long at, lo, hi;                             // cost before the sequence; of the share
  int index, share, member, b, u;
  int4 job;
  // the tile at hand
  long long t1;
  int r0, n_rows, j0, j1, slot;
  size_t row0;
  bool starts, ends;                                // the share has the tile's first key, its last one

  template <int M> __device__ __forceinline__ void tile() {
    const long long t0 = at + plan.before(seq, u);
    t1 = at + plan.before(seq, u + 1);
    const int rows = seq.q_len * plan.heads;        // below 2^28 (2^21 tokens, 128 heads)
    const int all_stages = plan.stages(seq, min((u + 1) * plan.tile_rows, rows) - 1);
    r0 = u * plan.tile_rows + member * M;
    n_rows = min(M, rows - r0);
    starts = t0 >= lo;
    ends = t1 <= hi;
    slot = 2 * index + (starts ? 1 : 0);
    row0 = (size_t)seq.q_start * plan.heads + r0;
    j0 = j1 = 0;
    if (n_rows <= 0) return;
    const int stages = plan.stages(seq, r0 + n_rows - 1);
    j0 = starts ? 0 : min(LatPlan::stage_at(lo - t0, all_stages), stages);
    j1 = ends ? stages : min(LatPlan::stage_at(hi - t0, all_stages), stages);
    if (starts && !ends) job = int4{(int)row0, n_rows, index, cut.of(t1 - 1) - share + 1};
    // a piece of a cut tile without keys
    if (j0 >= j1 && !(starts && ends) && threadIdx.x < M)
      reinterpret_cast<float2*>(args_anew()->part_ml)[(size_t)slot * M + threadIdx.x] = float2{-FLT_MAX, 0.f};
  }
  // Whether there is a tile after this one.
  __device__ __forceinline__ bool next(const LatentArgs& a) {
    if (t1 >= hi) return false;
    if (++u == plan.tiles(seq)) {
      at = t1;
      u = 0;
      do seq = lat_seq_uni(a, ++b);
      while (seq.q_len == 0);
    }
    return true;
  }
};

// Finds the workgroup's share; false: it has none.  Workgroups with one number modulo `group` take the same member of the tiles, and shares
// of an XCD's workgroups follow one another.
template <int M> __device__ __forceinline__ bool lat_find(const LatentArgs& a, LatFind& lds, LatWork& work) {
  const int tid = threadIdx.x, lane = tid & 63, w = uni(tid >> 6);
  const int group = a.group;
  const int per_xcd = (int)gridDim.x / kNumXcd;
  work.index = (int)(blockIdx.x % kNumXcd) * per_xcd + (int)(blockIdx.x / kNumXcd);
  work.share = work.index / group;
  work.member = work.index - work.share * group;
  work.plan = LatPlan{group * M, a.slope, a.heads};
  work.job = int4{0, 0, 0, 0};
  if (tid == 0) lds.bad = 0;
  __syncthreads();
  const int per = (a.batch + kLatThreads - 1) / kLatThreads;
  long long mine = 0;
  {
    bool bad = false;
    for (int i = 0; i < per; ++i) {
      const int b = tid * per + i;
      if (b >= a.batch) break;
      const LatSeq s = lat_seq(a, b);
      if (lat_bad(a, s)) bad = true;
      else mine += work.plan.before(s, work.plan.tiles(s));
    }
    if (bad) lds.bad = 1;
  }
  long long upto = mine;                            // of this wave's threads up to this one
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const long long y = shfl_up64(upto, d);
    if (lane >= d) upto += y;
  }
  if (lane == 63) lds.sum[w] = upto;
  __syncthreads();
  if (blockIdx.x == 0 && tid == 0) a.ws_hdr[kHdrError] = lds.bad;
  long long total = 0;
#pragma unroll
  for (int v = 0; v < kLatWaves; ++v) {
    if (v == w) upto += total;
    total += uni64(lds.sum[v]);
  }
  int shares = (int)gridDim.x / group;
  if (total < (long long)shares * a.min_share) shares = (int)max(1ll, total / a.min_share);
  if (uni(lds.bad) || total == 0 || work.share >= shares) {
    if (tid == 0) a.jobs[work.index] = work.job;
    return false;
  }
  work.cut = LatShares(total, shares);
  const long long lo = work.cut.start(work.share);
  work.lo = lo;
  work.hi = work.cut.start(work.share + 1);
  if (upto - mine <= lo && lo < upto) {
    lds.found = tid;
    lds.before = upto - mine;
  }
  __syncthreads();
  work.b = uni(lds.found) * per;
  work.at = uni64(lds.before);
  work.seq = lat_seq_uni(a, work.b);
  for (;;) {
    const long long c = work.plan.before(work.seq, work.plan.tiles(work.seq));
    if (lo < work.at + c) break;
    work.at += c;
    work.seq = lat_seq_uni(a, ++work.b);
  }
  work.u = work.plan.tile_at(work.seq, lo - work.at);
  return true;
}

// Keys that only some of the rows see have weight 0 in the others, and 0 times a value that is not finite is NaN.  So such a value becomes 0, in the
// page at hand (key0: its first key), and its channel is noted.  (The value is part of its key too: in rows that see it its score is NaN or infinite, so its
// channel's output is NaN there, if not the whole row, which is what the end of the tile makes of the note.)
template <typename Page, int DC, int M> __device__ __forceinline__ void note_odd(char* page, int key0, LatNotes<DC, M>& notes) {
  for (int i = threadIdx.x & 63; i < kPage * DC / 8; i += 64) {
    const int r = i / (DC / 8), c = i % (DC / 8);
    u32x4 v = *reinterpret_cast<const u32x4*>(page + 16 * i);
    bool bad = false;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t half = e & 1 ? 0x7f800000u : 0x7f80u;
      if ((v[e >> 1] & half) == half) {
        v[e >> 1] &= e & 1 ? 0xffffu : 0xffff0000u;
        atomicMin(&notes.odd[8 * ((c & ~15) | ((c & 15) ^ Page::f(r))) + e], key0 + r);
        bad = true;
      }
    }
    if (bad) {
      *reinterpret_cast<u32x4*>(page + 16 * i) = v;
      notes.any_odd = 1;
    }
  }
}

template <int DC, int M> __device__ __forceinline__ void clear_notes(LatNotes<DC, M>& notes) {
  for (int i = threadIdx.x; i < DC; i += kLatThreads) notes.odd[i] = INT32_MAX;
  if (threadIdx.x == 0) notes.any_odd = 0;
}

}  // namespace

// Up to 16 rows a sequence: every wave takes pages of its own, two in LDS, and no barrier until the tile ends, where the four waves'
// outputs are joined in LDS.  The products are far from their limit here, what counts is that copies never pause.
template <int DC, int DR>
__global__ __launch_bounds__(kLatThreads, 1) void latent16_kernel(LatentArgs a) {
  using Rows = LatRows16<DC, DR>;
  using Page = typename Rows::Page;
  using Copies = typename Rows::Copies;
  constexpr int M = 16;
  __shared__ __attribute__((aligned(256))) LatLds16<DC, DR> lds;
  const int tid = threadIdx.x, lane = tid & 63, w = uni(tid >> 6);
  clear_notes(lds.notes);
  LatWork work;
  if (!lat_find<M>(a, lds.find, work)) return;
  char* const buffers = lds.page[w][0];
  do {
    work.tile<M>();
    if (work.j0 >= work.j1) continue;
    const LatSeq seq = work.seq;
    const int r0 = work.r0, n_rows = work.n_rows, last = seq.ctx + (r0 + n_rows - 1) / a.heads;   // the last key
    const int kv = seq.ctx + seq.q_len, p1 = min(work.j1 * kLatWaves, last / kPage + 1);
    const int first_limit = seq.ctx + r0 / a.heads;        // keys behind it are not all rows'
    const bool in_part = last != first_limit;
    const int32_t* const bt = a.block_table + (size_t)work.b * a.bt_stride;
    // Ids of 64 of the wave's pages at once, lane i's page p + 4 i.  They are waited for here, and the queries before the loop: the compiler,
    // which does not know of the copies, would wait in every page, for these too.
    auto ids_from = [&](int p) {
      int ids = bt[min(p + kLatWaves * lane, p1 - 1)];
      __asm__ volatile("" : "+v"(ids));
      return ids;
    };
    auto page_at = [&](int ids, int i) {
      const int id = __builtin_amdgcn_readlane(ids, i);
      return reinterpret_cast<const char*>(a.cache) + (size_t)clamp_page(id, a.num_pages) * Page::kBytes;
    };
    int p = work.j0 * kLatWaves + w, ids = ids_from(p), i = 0;   // i: the page's number among the ids
    if (p < p1) Copies::page(page_at(ids, 0), lds_address(buffers));
    Rows x;
    x.start(args_anew()->q + work.row0 * (DC + DR), n_rows);
    if (tid < M) lds.notes.limit[tid] = seq.ctx + (r0 + min(tid, n_rows - 1)) / a.heads;
    x.pin_queries();
    barrier_lds();
    int parity = 0;
    for (;;) {                                      // pages whose scores are near the maxima so far; others end behind the inner loop
      bool above = false;
      char* page = nullptr;
#pragma unroll 1
      for (; p < p1; p += kLatWaves, parity ^= 1) {
        x.pin_queries();
        page = buffers + parity * Page::kBytes;
        if (p + kLatWaves < p1) {
          if (++i == 64) {
            ids = ids_from(p + kLatWaves);
            i = 0;
          }
          Copies::page(page_at(ids, i), lds_address(buffers) + (parity ^ 1) * Page::kBytes);
          __asm__ volatile("s_waitcnt vmcnt(%0)" ::"n"(Copies::kCopies) : "memory");
        } else {
          wait_copies();
        }
        const int key0 = p * kPage;
        if (kv - key0 < kPage) Copies::clear(page, kv - key0);   // rows behind the sequence's end
        x.scores(page);
        if (key0 + kPage - 1 > first_limit) {
          x.mask(lds.notes.limit, key0);
          if (in_part) note_odd<Page>(page, key0, lds.notes);
        }
        if (x.above(a.scale_log2)) {
          above = true;
          break;
        }
        x.add_values(page, a.scale_log2);
      }
      if (!above) break;
      x.raise(a.scale_log2);
      x.add_values(page, a.scale_log2);
      p += kLatWaves;
      parity ^= 1;
    }
    // ---- the waves' maxima and sums, then their outputs scaled alike
    x.l = xor32_add(xor16_add(x.l));
    if (x.g16 == 0) {
      lds.max[w][x.l16] = x.m;
      lds.sum[w][x.l16] = x.l;
    }
    barrier_lds();
    const bool odd = uni(lds.notes.any_odd) != 0;
    const float top = fmaxf(fmaxf(lds.max[0][x.l16], lds.max[1][x.l16]), fmaxf(lds.max[2][x.l16], lds.max[3][x.l16]));
    x.scale_to(top);
    // outputs of a wave: rows of DC channels in 32 bits, chunk c of row r in slot c ^ r of its 16
    constexpr int kWaveBytes = M * DC * 4;
    static_assert(kWaveBytes <= 2 * Page::kBytes, "in the wave's own buffers");
#pragma unroll
    for (int d = 0; d < Rows::kBlocks; ++d)
      *reinterpret_cast<f32x4*>(buffers + x.l16 * DC * 4 + 16 * ((4 * d + x.g16) ^ x.l16)) = x.o[d];
    barrier_lds();
    const LatArgsPtr args = args_anew();
    for (int r = w; r < n_rows || (r < M && !(work.starts && work.ends)); r += kLatWaves) {
      const float t = fmaxf(fmaxf(lds.max[0][r], lds.max[1][r]), fmaxf(lds.max[2][r], lds.max[3][r]));
      float l = 0.f;
#pragma unroll
      for (int v = 0; v < kLatWaves; ++v) l = fmaf(lds.sum[v][r], fexp2(lds.max[v][r] - t), l);
      const float inv = 1.f / l;
#pragma unroll
      for (int c = 0; c < DC; c += 256) {
        const int channel = c + 4 * lane;
        f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int v = 0; v < kLatWaves; ++v)
          y += *reinterpret_cast<const f32x4*>(lds.page[v][0] + r * DC * 4 + 16 * ((channel / 4) ^ r));
        if (odd)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (lds.notes.odd[channel + e] <= lds.notes.limit[r]) y[e] = __builtin_nanf("");
        if (work.starts && work.ends) {
          y *= inv;
          *reinterpret_cast<bf16x4*>(args->out + (work.row0 + r) * DC + channel) = bf16x4{(__bf16)y[0], (__bf16)y[1], (__bf16)y[2], (__bf16)y[3]};
        } else {
          *reinterpret_cast<f32x4*>(args->part_o + ((size_t)work.slot * M + r) * DC + channel) = y;
        }
      }
      if (lane == 0) {
        if (!(work.starts && work.ends)) reinterpret_cast<float2*>(args->part_ml)[(size_t)work.slot * M + r] = float2{t, l};
        else if (args->lse) args->lse[work.row0 + r] = (t + flog2(l)) * kLn2;
      }
    }
    barrier_lds();                                  // the next tile writes all of it
    if (odd) {
      clear_notes(lds.notes);
      barrier_lds();
    }
  } while (work.next(a));
  if (tid == 0) args_anew()->jobs[work.index] = work.job;
}

// More rows: tiles of 64.
template <int DC, int DR>
__global__ __launch_bounds__(kLatThreads, 1) void latent64_kernel(LatentArgs a) {
  using Rows = LatRows64<DC, DR>;
  using Page = typename Rows::Page;
  using Copies = typename Rows::Copies;
  using Lds = LatLds64<DC, DR>;
  constexpr int M = 64;
  __shared__ __attribute__((aligned(256))) Lds lds;
  const int tid = threadIdx.x, w = uni(tid >> 6);
  clear_notes(lds.notes);
  if (tid == 0) lds.flag[0] = lds.flag[1] = 0;
  LatWork work;
  if (!lat_find<M>(a, lds.find, work)) return;
  const unsigned my_page = lds_address(lds.stage[0]) + w * Page::kBytes;   // page w of a stage is this wave's to bring
  do {
    work.tile<M>();
    const int j0 = work.j0, j1 = work.j1;
    if (j0 >= j1) continue;
    const LatSeq seq = work.seq;
    const int r0 = work.r0, n_rows = work.n_rows;
    const int kv = seq.ctx + seq.q_len, pages = (kv + kPage - 1) / kPage;
    const int32_t* const bt = a.block_table + (size_t)work.b * a.bt_stride;
    const char* const cache = reinterpret_cast<const char*>(a.cache);
    // Page w of stage j (the last one where there is none; zeros take its place) goes to buffer j & 1.  Its id is read a stage
    // ahead, as a vector: a scalar load in flight would hold up the LDS reads, whose counter it shares.
    auto page_id = [&](int j) { return bt[min(j * kLatWaves + w, pages - 1)]; };
    auto page_at = [&](int id) { return cache + (size_t)clamp_page(uni(id), a.num_pages) * Page::kBytes; };
    Copies::page(page_at(page_id(j0)), my_page + (j0 & 1) * Lds::kStage);
    int id = page_id(j0 + 1);
    Rows x;
    x.start(w, args_anew()->q + work.row0 * (DC + DR), n_rows);
    if (tid < M) lds.notes.limit[tid] = seq.ctx + (r0 + min(tid, n_rows - 1)) / a.heads;
    const int first_limit = seq.ctx + r0 / a.heads;        // keys behind it are not all rows'
    const bool in_part = (r0 + n_rows - 1) / a.heads != r0 / a.heads;
    int j = j0;
    // Stages whose scores are near the maxima so far run in the inner loop; the others, the first one among them, end behind it (inside
    // it, their scaling would have the compiler move all outputs in every stage).
    for (;;) {
      bool above = false;
#pragma unroll 1
      for (; j < j1; ++j) {
        x.pin_queries();
        char* const stage = lds.stage[j & 1];
        char* const page = stage + w * Page::kBytes;
        const int key0 = j * kLatKeys, valid = kv - key0 - kPage * w;
        wait_copies();
        if (valid < kPage) Copies::clear(page, max(valid, 0));   // rows behind the sequence's end
        barrier_lds();                              // the stage is there; the other buffer and P are free
        const char* const src = page_at(id);
        const unsigned dst = my_page + (~j & 1) * Lds::kStage;
        const int more = j + 1 < j1;
        id = page_id(j + 2);
        if (w == 0) lds.flag[(j + 1) & 1] = 0;
        // the next stage's copies go out among the products: issued together, they would hold the wave
        x.scores(stage, [&](int i) {
          if (i < Copies::kCopies) Copies::copy2(i, src, dst, more);
        });
        if (key0 + kLatKeys - 1 > first_limit) {
          x.mask(lds, key0);
          if (in_part) {
            barrier_lds();                          // another wave has the page's scores for the other rows
            note_odd<Page>(page, key0 + kPage * w, lds.notes);
          }
        }
        x.weigh(lds, j, a.scale_log2);
        barrier_lds();
        if (uni(lds.flag[j & 1])) {
          above = true;
          break;
        }
        x.pin_outputs();
        x.template add_values<false>(lds, stage);
      }
      if (!above) break;
      x.join(lds);
      x.template add_values<true>(lds, lds.stage[j & 1]);
      ++j;
    }
    // ---- the rows' sums over lanes and waves, then the output or the partial
    const LatArgsPtr args = args_anew();
    barrier_lds();
    const bool odd = uni(lds.notes.any_odd) != 0;
    if (odd) x.set_odd(lds);
    if (tid == 0) lds.flag[0] = lds.flag[1] = 0;
    x.sums(lds);
    barrier_lds();
    x.each(lds, [&](int r, float m, float l, bool first, auto&& channels) {
      if (work.starts && work.ends) {
        const float inv = 1.f / l;
        if (r >= n_rows) return;
        uint16_t* const dst = args->out + (work.row0 + r) * DC;
        channels([&](int c, const f32x4& o) {
          const f32x4 y = o * inv;
          *reinterpret_cast<bf16x4*>(dst + c) = bf16x4{(__bf16)y[0], (__bf16)y[1], (__bf16)y[2], (__bf16)y[3]};
        });
        if (args->lse && first) args->lse[work.row0 + r] = (m + flog2(l)) * kLn2;
      } else {
        float* const dst = args->part_o + ((size_t)work.slot * M + r) * DC;
        channels([&](int c, const f32x4& o) { *reinterpret_cast<f32x4*>(dst + c) = o; });
        if (first) reinterpret_cast<float2*>(args->part_ml)[(size_t)work.slot * M + r] = float2{m, l};
      }
    });
    if (odd) clear_notes(lds.notes);
    barrier_lds();                                  // the next tile writes the limits
  } while (work.next(a));
  if (tid == 0) args_anew()->jobs[work.index] = work.job;
}

// Joins the partials of a cut tile: job (first row, rows, index of the first piece's workgroup, shares).  Its first piece is in slot
// 1 of that workgroup, the others in slot 0 of the shares that follow, in order (kLatentGrid pieces at most).  A lane takes DC / 64 channels of a
// row.  Few pieces: a wave a row.  Many: the waves take a fourth of them each, row by row.  Workgroups run on the XCD that wrote the first piece.
template <int DC, int M>
__global__ __launch_bounds__(kLatThreads) void latent_merge_kernel(LatentArgs a) {
  static_assert(kLatentGrid <= 64 * kLatWaves, "a lane a piece");
  constexpr int kRows = M / 16, kC = DC / 64;       // rows of a workgroup
  const int4 job = a.jobs[blockIdx.x % kNumXcd * (kLatentGrid / kNumXcd) + blockIdx.x / kNumXcd];
  const int r0 = blockIdx.y * kRows;
  if (r0 >= job.y) return;
  __shared__ float s_top[kLatWaves], s_sum[kLatWaves];
  __shared__ __attribute__((aligned(16))) float s_o[kLatWaves][DC];
  const int lane = threadIdx.x & 63, w = uni(threadIdx.x >> 6), n = job.w, end = min(r0 + kRows, job.y);
  const bool few = n <= 16;
  const int first = few ? 0 : w, step = few ? 1 : kLatWaves, mine = n > first ? (n - first + step - 1) / step : 0;   // this wave's pieces
  auto slot = [&](int i) { return (size_t)(i == 0 ? 2 * job.z + 1 : 2 * (job.z + i * a.group)) * M; };
  for (int r = few ? r0 + w : r0; r < end; r += few ? kLatWaves : 1) {
    // lane k holds the maximum and sum of the wave's piece k; a piece that saw nothing counts nothing, its outputs may be unwritten
    const float2 ml = lane < mine ? reinterpret_cast<const float2*>(a.part_ml)[slot(step * lane + first) + r] : float2{-FLT_MAX, 0.f};
    const bool seen = ml.y != 0.f;
    float top = seen ? ml.x : -FLT_MAX;
    top = xor32_max(xor16_max(top));
#pragma unroll
    for (int d = 8; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    if (!few) {
      if (lane == 0) s_top[w] = top;
      __syncthreads();
      top = fmaxf(fmaxf(s_top[0], s_top[1]), fmaxf(s_top[2], s_top[3]));
    }
    const float weight = seen ? fexp2(ml.x - top) : 0.f;
    float l = seen ? weight * ml.y : 0.f;
    l = xor32_add(xor16_add(l));
#pragma unroll
    for (int d = 8; d > 0; d >>= 1) l += __shfl_xor(l, d);
    const unsigned long long all_seen = __ballot(seen);
    float o[kC];
#pragma unroll
    for (int c = 0; c < kC; ++c) o[c] = 0.f;
#pragma unroll 4
    for (int k = 0; k < mine; ++k) {
      const bool use = all_seen >> k & 1;
      const float f = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, weight), k));
      const float* const src = a.part_o + (slot(step * k + first) + r) * DC + 4 * lane;
#pragma unroll
      for (int c = 0; c < kC; c += 4) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(src + 64 * c);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[c + e] = use ? fmaf(f, x[e], o[c + e]) : o[c + e];
      }
    }
    if (!few) {
      if (lane == 0) s_sum[w] = l;
#pragma unroll
      for (int c = 0; c < kC; c += 4) *reinterpret_cast<f32x4*>(&s_o[w][64 * c + 4 * lane]) = f32x4{o[c], o[c + 1], o[c + 2], o[c + 3]};
      __syncthreads();
      if (w == 0) {
        l = (s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]);
#pragma unroll
        for (int c = 0; c < kC; ++c) {
          const int at = 64 * (c & ~3) + 4 * lane + (c & 3);
          o[c] = (s_o[0][at] + s_o[1][at]) + (s_o[2][at] + s_o[3][at]);
        }
      }
    }
    if (few || w == 0) {
      const size_t row = (size_t)job.x + r;
      const float inv = 1.f / l;
#pragma unroll
      for (int c = 0; c < kC; c += 4)
        *reinterpret_cast<bf16x4*>(a.out + row * DC + 64 * c + 4 * lane) =
            bf16x4{(__bf16)(o[c] * inv), (__bf16)(o[c + 1] * inv), (__bf16)(o[c + 2] * inv), (__bf16)(o[c + 3] * inv)};
      if (a.lse && lane == 0) a.lse[row] = (top + flog2(l)) * kLn2;
    }
    if (!few) __syncthreads();                      // the next row's sums
  }
}

namespace {
template <int DC, int DR> hipError_t launch_dims(const LatentArgs& a, int tile, bool merge, hipStream_t stream) {
  const dim3 grid(kLatentGrid), threads(kLatThreads), merge_grid(kLatentGrid, 16);
  if (merge && tile == 16) hipLaunchKernelGGL((latent_merge_kernel<DC, 16>), merge_grid, threads, 0, stream, a);
  else if (merge) hipLaunchKernelGGL((latent_merge_kernel<DC, 64>), merge_grid, threads, 0, stream, a);
  else if (tile == 16) hipLaunchKernelGGL((latent16_kernel<DC, DR>), grid, threads, 0, stream, a);
  else hipLaunchKernelGGL((latent64_kernel<DC, DR>), grid, threads, 0, stream, a);
  return hipGetLastError();
}
}  // namespace

hipError_t launch_latent(const LatentArgs& a, int latent_dim, int tile, bool merge, hipStream_t stream) {
  return latent_dim == 512 ? launch_dims<512, 64>(a, tile, merge, stream) : launch_dims<256, 32>(a, tile, merge, stream);
}

}  // namespace pearl
