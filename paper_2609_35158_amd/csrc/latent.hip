// gfx950 kernels of attention over a paged cache of latent vectors (absorbed form; paper, section 4.3, Eq. 1: decode
// is bound by its cache reads, which one short row a token for all heads makes few).
//
// A cached row is (c, r), DC + DR channels; a query row (token, head) is (q_c, q_r).  s_j = scale q . (c_j, r_j), over
// keys j up to the token's position, o = sum softmax(s)_j c_j: the row is the key of every head and its latent part the
// value.  So the rows of a tile are any (token, head) pairs of a sequence, in the order of q: row rho is token rho / H, head
// rho % H.  The softmax is online, in base 2, with state in 32 bits; weights enter the second product in bf16.
//
// A workgroup of 4 waves takes M rows and stages of 64 keys (4 pages):
//   S^T (keys x rows) = K . Q^T: wave w takes the keys of page w of the stage for all rows; Q stays in registers, so K is
//                       read from LDS once;
//   O^T (channels x rows) += V^T . P^T: wave w takes a quarter of the channels, V^T by transposing reads of the same LDS
//                       rows, once; P goes through LDS, 2 bytes a weight.
// (16x16x32 MFMA: A row l%16, k 8(l/16)+e; B column l%16, k 8(l/16)+e; D column l%16, row 4(l/16)+r.)  With rows
// dealt to waves instead, every wave would read every key: at 64 rows 4 times the LDS reads, which then bound both products.
// A row's maximum is common to the waves.  It may lag the true one by kLag (log2 units), so most stages go on with the old one after
// one barrier; where some score is further above, the waves exchange their maxima and weigh the stage again.
//
// Work is cut into equal shares of keys, in the order (sequence, tile, key), on the device from the lengths: each
// workgroup finds its share by itself.  A tile cut by shares leaves (o~, m, l) in the workspace, joined by
// latent_merge_kernel.  `group` workgroups next to one another on an XCD take neighbouring tiles of the same share, so that
// they read the same keys at the same time, from L2.

#include "attn_device.h"

#include <float.h>

namespace pearl {
namespace {

constexpr int kLatThreads = 256;
constexpr int kLatWaves = kLatThreads / 64;
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
__device__ __forceinline__ void in_vector(f32x4& x) { __asm__ volatile("" : "+v"(x)); }
__device__ __forceinline__ void in_acc(bf16x8& x) { __asm__ volatile("" : "+a"(x)); }

__device__ __forceinline__ long long uni64(long long x) {
  const unsigned lo = uni((int)x), hi = uni((int)(x >> 32));
  return (long long)((unsigned long long)hi << 32 | lo);
}

// A staged page: 16 rows of DC channels, then 16 rows of DR.  Chunk (16 bytes) c of latent row r is in slot c ^ f(r) of
// its 16 (the row reads of 16 lanes fall into 16 slots, and the transposing reads of 32 lanes, rows {0-3, 8-11} or {4-7,
// 12-15} and two chunks each, into 16); of the rotated part in slot c ^ (r / 2) (DR = 64; 32: r / 4), where 2 (4)
// rows share the banks.
template <int DC, int DR> struct LatPage {
  static constexpr int kWidth = (DC + DR) * 2;      // bytes of a cached row
  static constexpr int kRowBytes = DC * 2, kRotBytes = DR * 2;
  static constexpr int kRot = kPage * kRowBytes;    // offset of the rotated parts
  static constexpr int kBytes = kPage * kWidth;
  static_assert(kBytes % 256 == 0 && kRowBytes % 256 == 0, "the swizzle takes address bits 4 .. 7");
  __device__ static __forceinline__ int f(int r) { return (r & 8) | ((r & 3) << 1) | ((r >> 2) & 1); }
  __device__ static __forceinline__ int rot_f(int r) { return DR == 64 ? (r >> 1) & 7 : (r >> 2) & 3; }
};

// The lanes' parts of a page's copies, 1 KiB an instruction.
template <int DC, int DR> struct LatCopies {
  using Page = LatPage<DC, DR>;
  static constexpr int kRows = 1024 / Page::kRowBytes;       // of an instruction
  static constexpr int kLatent = kPage / kRows, kRot = kPage * Page::kRotBytes / 1024;
  static_assert(Page::kWidth % 32 == 0 && (DR == 32 || Page::kWidth % 128 == 0), "the swizzle takes bits above the rows' alignment");
  // 16 times the lane's slot, swizzled by its part of the row, and the offset of its row among an instruction's; the same of the
  // rotated parts' first instruction.
  int lane16, row, rot;

  __device__ __forceinline__ LatCopies() {
    const int l = threadIdx.x & 63;
    lane16 = 16 * l;
    row = 0;
    if constexpr (kRows == 2) {
      lane16 = 16 * ((l & 31) ^ Page::f(l >> 5));
      row = (l >> 5) * Page::kWidth;
    }
    constexpr int kChunks = Page::kRotBytes / 16;
    const int r = l / kChunks, slot = l % kChunks;
    rot = r * Page::kWidth + Page::kRowBytes + 16 * (slot ^ Page::rot_f(r));
  }

  // The page at src to LDS.  An instruction's immediate offset advances both addresses, 1 KiB each.
  __device__ __forceinline__ void copy(const char* src, const char* lds) const {
    int lane_off = lane16, rot_off = rot;
    __asm__ volatile("" : "+v"(lane_off), "+v"(rot_off));   // formed here each time: kept over the stages, the offsets would be spilled
#pragma unroll
    for (int i = 0; i < kLatent; i += 4) {
      int off[4];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        off[k] = (lane_off ^ (Page::f(kRows * (i + k)) << 4)) + row + k * (kRows * Page::kWidth - 1024);
      copy4(src + i * kRows * Page::kWidth, off, lds + 1024 * i);
    }
    // 8 rows further (DR = 64) the swizzle differs in chunk bit 2
#pragma unroll
    for (int i = 0; i < kRot; ++i) copy1(src + i * 8 * Page::kWidth, rot_off ^ (64 * i), lds + Page::kRot + 1024 * i);
  }

  __device__ static __forceinline__ unsigned lds_address(const char* p) {
    return __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)((LDS_AS const char*)p));
  }
  __device__ static __forceinline__ void copy4(const char* base, const int* off, const char* lds) {
    unsigned saved;
    __asm__ volatile(
        "s_mov_b32 %0, m0\n\t"
        "s_mov_b32 m0, %6\n\t"
        "s_nop 0\n\t"
        "global_load_lds_dwordx4 %1, %5\n\t"
        "global_load_lds_dwordx4 %2, %5 offset:1024\n\t"
        "global_load_lds_dwordx4 %3, %5 offset:2048\n\t"
        "global_load_lds_dwordx4 %4, %5 offset:3072\n\t"
        "s_mov_b32 m0, %0"
        : "=&s"(saved)
        : "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]), "s"(base), "s"(lds_address(lds))
        : "memory");
  }
  __device__ static __forceinline__ void copy1(const char* base, int off, const char* lds) {
    unsigned saved;
    __asm__ volatile(
        "s_mov_b32 %0, m0\n\t"
        "s_mov_b32 m0, %3\n\t"
        "s_nop 0\n\t"
        "global_load_lds_dwordx4 %1, %2\n\t"
        "s_mov_b32 m0, %0"
        : "=&s"(saved)
        : "v"(off), "s"(base), "s"(lds_address(lds))
        : "memory");
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

__device__ __forceinline__ bool lat_bad(const LatentArgs& a, const LatSeq& s) {
  const long long kv = (long long)s.ctx + s.q_len;
  return s.q_len < 0 || s.ctx < 0 || s.q_start < 0 || s.q_len > a.max_q_len || (long long)s.q_start + s.q_len > a.total_q ||
         kv > a.max_kv_len || (kv + kPage - 1) / kPage > a.bt_stride;
}

__device__ __forceinline__ long long shfl_up64(long long x, int d) {
  const int lo = __shfl_up((int)x, d), hi = __shfl_up((int)(x >> 32), d);
  return (long long)(((unsigned long long)(unsigned)hi << 32) | (unsigned)lo);
}

}  // namespace

// Work with `group` g = index % group; shares of an XCD's workgroups follow one another.
template <int DC, int DR, int M>
__global__ __launch_bounds__(kLatThreads, 1) void latent_kernel(LatentArgs a) {
  using Page = LatPage<DC, DR>;
  constexpr int RG = M / 16;                        // row groups
  constexpr int kSteps = DC / 32, kRotSteps = DR / 32;
  constexpr int kBlocks = DC / kLatWaves / 16;      // blocks of 16 channels of a wave
  constexpr int kStage = kLatWaves * Page::kBytes;
  constexpr int kAhead = 3;                         // LDS reads of the products' operands, ahead of them
  constexpr int kKeepQ = M == 64 ? (DC == 512 ? 16 : kSteps + kRotSteps) : M == 32 ? kSteps + kRotSteps : 0;   // steps whose queries are in accumulation registers
  __shared__ __attribute__((aligned(256))) char s_stage[2 * kStage];
  __shared__ __attribute__((aligned(256))) char s_p[M * kLatKeys * 2];
  __shared__ float s_max[kLatWaves][M];
  __shared__ int s_limit[M];
  __shared__ int s_flag[2];                         // some score is far above its row's maximum; one a stage in turn
  __shared__ int s_odd[DC];                         // of each channel: the first key with a value that is not finite and ..
  __shared__ int s_any_odd;                         // .. whether there is one, among those that only some of the tile's rows see
  __shared__ long long s_sum[kLatWaves];
  __shared__ int s_found, s_bad;
  __shared__ long long s_before;
  const int tid = threadIdx.x, lane = tid & 63, w = uni(tid >> 6);
  const int g16 = lane >> 4, l16 = lane & 15;

  // ---- this workgroup's share
  const int group = a.group;
  const int per_xcd = (int)gridDim.x / kNumXcd;
  const int index = (int)(blockIdx.x % kNumXcd) * per_xcd + (int)(blockIdx.x / kNumXcd);
  int share = index / group;
  const int member = index - share * group;
  const LatPlan plan{a.group * M, a.slope, a.heads};
  if (tid == 0) { s_bad = 0; s_flag[0] = s_flag[1] = s_any_odd = 0; }
  for (int i = tid; i < DC; i += kLatThreads) s_odd[i] = INT32_MAX;
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
      else mine += plan.before(s, plan.tiles(s));
    }
    if (bad) s_bad = 1;
  }
  long long upto = mine;                            // of this wave's threads up to this one
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const long long y = shfl_up64(upto, d);
    if (lane >= d) upto += y;
  }
  if (lane == 63) s_sum[w] = upto;
  __syncthreads();
  int4* const job = a.jobs + index;
  if (blockIdx.x == 0 && tid == 0) a.ws_hdr[kHdrError] = s_bad;
  long long total = 0;
#pragma unroll
  for (int v = 0; v < kLatWaves; ++v) {
    if (v == w) upto += total;
    total += uni64(s_sum[v]);
  }
  int shares = (int)gridDim.x / group;
  if (total < (long long)shares * a.min_share) shares = (int)max(1ll, total / a.min_share);
  if (uni(s_bad) || total == 0 || share >= shares) {
    if (tid == 0) *job = int4{0, 0, 0, 0};
    return;
  }
  const LatShares cut(total, shares);
  const long long lo = cut.start(share), hi = cut.start(share + 1);
  if (upto - mine <= lo && lo < upto) {
    s_found = tid;
    s_before = upto - mine;
  }
  __syncthreads();
  int b = uni(s_found) * per;
  long long at = uni64(s_before);                   // cost before sequence b
  LatSeq seq = lat_seq(a, b);
  for (;;) {
    const long long c = plan.before(seq, plan.tiles(seq));
    if (lo < at + c) break;
    at += c;
    seq = lat_seq(a, ++b);
  }
  int u = plan.tile_at(seq, lo - at);
  int4 my_job = {0, 0, 0, 0};

  // ---- lanes' addresses
  const LatCopies<DC, DR> copies;
  // of a key's chunk g16; those of the steps after it differ in address bits 6 and 7, and by whole 256 bytes
  const int k_off = l16 * Page::kRowBytes + 16 * (g16 ^ Page::f(l16));
  const int rot_off = Page::kRot + l16 * Page::kRotBytes + 16 * (g16 ^ Page::rot_f(l16));
  int v_off[2];                                     // of block 0: the wave's channels start at chunk (DC / 32) w
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = 8 * (g16 & 1) + 4 * i + (l16 >> 2), c = DC / 32 * w + ((l16 >> 1) & 1);
    v_off[i] = (g16 >> 1) * Page::kBytes + r * Page::kRowBytes + 16 * ((c & ~15) | ((c & 15) ^ Page::f(r))) + 8 * (l16 & 1);
  }
  const int h16 = (l16 >> 1) & 7;                   // swizzle of P's 128-byte rows
  const int p_write = l16 * 128 + 16 * ((2 * w + (g16 >> 1)) ^ h16) + 8 * (g16 & 1);
  const int p_read = l16 * 128 + 16 * (g16 ^ h16);  // of keys 0 .. 31; ^ 64 of the others

  // ---- tiles
  for (;;) {
    const long long t0 = at + plan.before(seq, u), t1 = at + plan.before(seq, u + 1);
    const int rows = seq.q_len * a.heads;           // below 2^28 (2^21 tokens, 128 heads)
    const int all_stages = plan.stages(seq, min((u + 1) * plan.tile_rows, rows) - 1);
    const int r0 = u * plan.tile_rows + member * M, n_rows = min(M, rows - r0);
    const bool starts = t0 >= lo, ends = t1 <= hi;
    if (n_rows > 0) {
      const int stages = plan.stages(seq, r0 + n_rows - 1);
      const int j0 = starts ? 0 : min(LatPlan::stage_at(lo - t0, all_stages), stages);
      const int j1 = ends ? stages : min(LatPlan::stage_at(hi - t0, all_stages), stages);
      const int slot = 2 * index + (starts ? 1 : 0);
      const size_t row0 = (size_t)seq.q_start * a.heads + r0;
      if (starts && !ends) my_job = int4{(int)row0, n_rows, index, cut.of(t1 - 1) - share + 1};
      if (j0 >= j1) {
        if (!(starts && ends) && tid < M) reinterpret_cast<float2*>(a.part_ml)[(size_t)slot * M + tid] = float2{-FLT_MAX, 0.f};
      } else {
        const int kv = seq.ctx + seq.q_len, pages = (kv + kPage - 1) / kPage;
        const ConstI32Ptr bt = (ConstI32Ptr)(a.block_table + (size_t)b * a.bt_stride);
        const char* const cache = reinterpret_cast<const char*>(a.cache);
        // page w of stage j, to its buffer: the page id is read a stage ahead
        auto page_id = [&](int j) { return clamp_page(bt[min(j * kLatWaves + w, pages - 1)], a.num_pages); };
        auto issue = [&](int j, int id) {
          if (j * kLatWaves + w < pages)
            copies.copy(cache + (size_t)id * Page::kBytes, s_stage + (j & 1) * kStage + w * Page::kBytes);
        };
        issue(j0, page_id(j0));
        int id = page_id(j0 + 1);
        // queries: 16 bytes of row l16 of each group, channels 32 step + 8 g16
        bf16x8 q[RG][kSteps + kRotSteps];
        // the last key that a row sees
        barrier_lds();
        if (tid < M) s_limit[tid] = seq.ctx + (r0 + min(tid, n_rows - 1)) / a.heads;
#pragma unroll
        for (int rg = 0; rg < RG; ++rg) {
          const int r = 16 * rg + l16;
          const uint16_t* const src = a.q + (row0 + min(r, n_rows - 1)) * (size_t)(DC + DR) + 8 * g16;
#pragma unroll
          for (int k = 0; k < kSteps + kRotSteps; ++k) q[rg][k] = as_bf16x8(ld16(src + 32 * k));
        }
        const int first_limit = seq.ctx + r0 / a.heads;    // keys behind it are not all rows'
        const bool in_part = (r0 + n_rows - 1) / a.heads != r0 / a.heads;
        f32x4 o[kBlocks][RG];
        float m[RG], l[RG];
#pragma unroll
        for (int rg = 0; rg < RG; ++rg) {
          m[rg] = -FLT_MAX;
          l[rg] = 0.f;
#pragma unroll
          for (int d = 0; d < kBlocks; ++d) o[d][rg] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        f32x4 s[RG];                                // scores of the wave's 16 keys
        float sum[RG];
        // Weights with the rows' maxima so far, to P; the largest exponent.
        auto weigh = [&]() {
          float top = -FLT_MAX;
#pragma unroll
          for (int rg = 0; rg < RG; ++rg) {
            float x[4], p[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              x[r] = fmaf(s[rg][r], a.scale_log2, -m[rg]);
              p[r] = fexp2(x[r]);
            }
            top = fmaxf(top, fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])));
            sum[rg] = (p[0] + p[1]) + (p[2] + p[3]);
            *reinterpret_cast<bf16x4*>(s_p + 2048 * rg + p_write) = bf16x4{(__bf16)p[0], (__bf16)p[1], (__bf16)p[2], (__bf16)p[3]};
          }
          return top;
        };
        auto add_values = [&](const char* stage) {
#pragma unroll
          for (int rg = 0; rg < RG; ++rg) l[rg] += sum[rg];
          // value operands are read kAhead blocks ahead of their products
          int off0 = v_off[0], off1 = v_off[1];
          __asm__ volatile("" : "+v"(off0), "+v"(off1));
          auto value_of = [&](int i) {
            const char* const at = stage + i / kBlocks * 2 * Page::kBytes;
            return concat_tr(lds_read_tr(at, off0 ^ (32 * (i % kBlocks))), lds_read_tr(at, off1 ^ (32 * (i % kBlocks))));
          };
          bf16x8 p[RG], value[kAhead];
#pragma unroll
          for (int i = 0; i < kAhead; ++i) value[i] = value_of(i);
#pragma unroll
          for (int i = 0; i < kLatKeys / 32 * kBlocks; ++i) {
            if (i % kBlocks == 0) {
#pragma unroll
              for (int rg = 0; rg < RG; ++rg)
                p[rg] = as_bf16x8(*reinterpret_cast<const u32x4*>(s_p + 2048 * rg + (p_read ^ (64 * (i / kBlocks)))));
            }
            const bf16x8 x = value[i % kAhead];
#pragma unroll
            for (int rg = 0; rg < RG; ++rg)
              o[i % kBlocks][rg] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, p[rg], o[i % kBlocks][rg], 0, 0, 0);
            if (i + kAhead < kLatKeys / 32 * kBlocks) value[i % kAhead] = value_of(i + kAhead);
            __builtin_amdgcn_sched_barrier(0);
          }
        };
        int j = j0;
        // Stages whose scores are near the maxima so far run in the inner loop; the others, the first one among them, behind it (inside it,
        // their scaling would have the compiler copy all outputs in every stage).
        for (;;) {
          bool above = false;
#pragma unroll 1
          for (; j < j1; ++j) {
            if constexpr (kKeepQ > 0) {
#pragma unroll
              for (int rg = 0; rg < RG; ++rg)
#pragma unroll
                for (int k = 0; k < kKeepQ; ++k) in_acc(q[rg][k]);
            }
            char* const page = s_stage + (j & 1) * kStage + w * Page::kBytes;
            const int key0 = j * kLatKeys;
            wait_copies();
            const int valid = kv - key0 - kPage * w;  // rows of this wave's page
            if (valid < kPage) {                    // the others become zeros
              const int from = max(valid, 0);
              for (int i = from * Page::kRowBytes + 16 * lane; i < Page::kRot; i += 1024) *reinterpret_cast<u32x4*>(page + i) = u32x4{0u, 0u, 0u, 0u};
              for (int i = Page::kRot + from * Page::kRotBytes + 16 * lane; i < Page::kBytes; i += 1024)
                *reinterpret_cast<u32x4*>(page + i) = u32x4{0u, 0u, 0u, 0u};
            }
            barrier_lds();                          // the other buffer and P are free
            if (j + 1 < j1) {
              issue(j + 1, id);
              if (j + 2 < j1) id = page_id(j + 2);
            }
            if (tid == 0) s_flag[(j + 1) & 1] = 0;
#pragma unroll
            for (int rg = 0; rg < RG; ++rg) s[rg] = f32x4{0.f, 0.f, 0.f, 0.f};
            // key operands are read kAhead steps ahead of their products
            int at = k_off, at_rot = rot_off;
            __asm__ volatile("" : "+v"(at), "+v"(at_rot));
            auto key_of = [&](int k) {
              const int off = k < kSteps ? (at ^ (64 * (k & 3))) + 256 * (k >> 2) : at_rot ^ (64 * (k - kSteps));
              return as_bf16x8(*reinterpret_cast<const u32x4*>(page + off));
            };
            bf16x8 key[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) key[k] = key_of(k);
#pragma unroll
            for (int k = 0; k < kSteps + kRotSteps; ++k) {
              const bf16x8 x = key[k % kAhead];
#pragma unroll
              for (int rg = 0; rg < RG; ++rg) s[rg] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, q[rg][k], s[rg], 0, 0, 0);
              if (k + kAhead < kSteps + kRotSteps) key[k % kAhead] = key_of(k + kAhead);
              __builtin_amdgcn_sched_barrier(0);
            }
            if (key0 + kLatKeys - 1 > first_limit) {
              const int key = key0 + kPage * w + 4 * g16;
#pragma unroll
              for (int rg = 0; rg < RG; ++rg) {
                const int limit = s_limit[16 * rg + l16];
#pragma unroll
                for (int r = 0; r < 4; ++r)
                  if (key + r > limit) s[rg][r] = -__builtin_inff();
              }
              // Keys that only some of the rows see have weight 0 in the others, and 0 times a value that is not finite is NaN: it becomes 0 and
              // its channel is noted.  (The value is part of its key too: in rows that see it its score is NaN or infinite, so its
              // channel's output is NaN there, if not the whole row, which is what the end of the tile makes of the note.)
              if (in_part) {
                for (int i = lane; i < kPage * DC / 8; i += 64) {
                  const int r = i / (DC / 8), c = i % (DC / 8);
                  u32x4 x = *reinterpret_cast<const u32x4*>(page + 16 * i);
                  bool bad = false;
#pragma unroll
                  for (int e = 0; e < 8; ++e) {
                    const uint32_t half = e & 1 ? 0x7f800000u : 0x7f80u;
                    if ((x[e >> 1] & half) == half) {
                      x[e >> 1] &= e & 1 ? 0xffffu : 0xffff0000u;
                      atomicMin(&s_odd[8 * ((c & ~15) | ((c & 15) ^ Page::f(r))) + e], key0 + kPage * w + r);
                      bad = true;
                    }
                  }
                  if (bad) {
                    *reinterpret_cast<u32x4*>(page + 16 * i) = x;
                    s_any_odd = 1;
                  }
                }
              }
            }
            const float top = weigh();
            if (__ballot(top > kLag) && lane == 0) s_flag[j & 1] = 1;
            barrier_lds();
            if (uni(s_flag[j & 1])) {
              above = true;
              break;
            }
#pragma unroll
            for (int rg = 0; rg < RG; ++rg)
#pragma unroll
              for (int d = 0; d < kBlocks; ++d) in_vector(o[d][rg]);
            add_values(s_stage + (j & 1) * kStage);
          }
          if (!above) break;
          // the waves agree on new maxima and weigh the stage again
#pragma unroll
          for (int rg = 0; rg < RG; ++rg) {
            float x = fmaxf(fmaxf(s[rg][0], s[rg][1]), fmaxf(s[rg][2], s[rg][3])) * a.scale_log2;
            x = xor32_max(xor16_max(x));
            if (g16 == 0) s_max[w][16 * rg + l16] = x;
          }
          barrier_lds();
#pragma unroll
          for (int rg = 0; rg < RG; ++rg) {
            float x = m[rg];
#pragma unroll
            for (int v = 0; v < kLatWaves; ++v) x = fmaxf(x, s_max[v][16 * rg + l16]);
            const float alpha = fexp2(m[rg] - x);
            m[rg] = x;
            l[rg] *= alpha;
#pragma unroll
            for (int d = 0; d < kBlocks; ++d) o[d][rg] *= alpha;
          }
          weigh();
          barrier_lds();
          add_values(s_stage + (j & 1) * kStage);
          ++j;
        }
        // ---- the rows' sums over lanes and waves, then the output or the partial
        barrier_lds();
        const bool odd = uni(s_any_odd) != 0;
        if (odd) {
#pragma unroll
          for (int d = 0; d < kBlocks; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int first = s_odd[DC / kLatWaves * w + 16 * d + 4 * g16 + e];
#pragma unroll
              for (int rg = 0; rg < RG; ++rg)
                if (first <= s_limit[16 * rg + l16]) o[d][rg][e] = __builtin_nanf("");
            }
        }
        if (tid == 0) s_flag[0] = s_flag[1] = 0;
#pragma unroll
        for (int rg = 0; rg < RG; ++rg) {
          const float x = xor32_add(xor16_add(l[rg]));
          if (g16 == 0) s_max[w][16 * rg + l16] = x;
        }
        barrier_lds();
        if (odd) {                                  // all have read it; the next tile's stages are behind another barrier
          for (int i = tid; i < DC; i += kLatThreads) s_odd[i] = INT32_MAX;
          if (tid == 0) s_any_odd = 0;
        }
#pragma unroll
        for (int rg = 0; rg < RG; ++rg) {
          const int r = 16 * rg + l16;
          float x = 0.f;
#pragma unroll
          for (int v = 0; v < kLatWaves; ++v) x += s_max[v][r];
          const int channel = DC / kLatWaves * w + 4 * g16;
          if (starts && ends) {
            const float inv = 1.f / x;
            if (r < n_rows) {
              uint16_t* const dst = a.out + (row0 + r) * DC + channel;
#pragma unroll
              for (int d = 0; d < kBlocks; ++d) {
                const f32x4 y = o[d][rg] * inv;
                *reinterpret_cast<bf16x4*>(dst + 16 * d) = bf16x4{(__bf16)y[0], (__bf16)y[1], (__bf16)y[2], (__bf16)y[3]};
              }
              if (a.lse && w == 0 && g16 == 0) a.lse[row0 + r] = (m[rg] + flog2(x)) * kLn2;
            }
          } else {
            float* const dst = a.part_o + ((size_t)slot * M + r) * DC + channel;
#pragma unroll
            for (int d = 0; d < kBlocks; ++d) *reinterpret_cast<f32x4*>(dst + 16 * d) = o[d][rg];
            if (w == 0 && g16 == 0) reinterpret_cast<float2*>(a.part_ml)[(size_t)slot * M + r] = float2{m[rg], x};
          }
        }
      }
    }
    if (t1 >= hi) break;
    if (++u == plan.tiles(seq)) {
      at = t1;
      u = 0;
      do seq = lat_seq(a, ++b);
      while (seq.q_len == 0);
    }
  }
  if (tid == 0) *job = my_job;
}

// Joins the partials of a cut tile: job (first row, rows, index of the first piece's workgroup, shares).  Its first piece is in slot
// 1 of that workgroup, the others in slot 0 of the shares that follow, in order.
template <int DC, int M>
__global__ __launch_bounds__(DC / 4) void latent_merge_kernel(LatentArgs a) {
  const int4 job = a.jobs[blockIdx.x];
  const int r = blockIdx.y;
  if (r >= job.y) return;
  const int n = job.w, c = threadIdx.x * 4;
  auto slot = [&](int i) { return (size_t)(i == 0 ? 2 * job.z + 1 : 2 * (job.z + i * a.group)) * M + r; };
  const float2* const ml = reinterpret_cast<const float2*>(a.part_ml);
  float top = -FLT_MAX;
  for (int i = 0; i < n; ++i) {
    const float2 x = ml[slot(i)];
    if (x.y != 0.f) top = fmaxf(top, x.x);
  }
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  float l = 0.f;
  for (int i = 0; i < n; ++i) {
    const float2 x = ml[slot(i)];
    if (x.y == 0.f) continue;                       // nothing seen; its o~ may be unwritten
    const float weight = fexp2(x.x - top);
    l = fmaf(weight, x.y, l);
    o += weight * *reinterpret_cast<const f32x4*>(a.part_o + slot(i) * DC + c);
  }
  const size_t row = (size_t)job.x + r;
  const f32x4 y = o * (1.f / l);
  *reinterpret_cast<bf16x4*>(a.out + row * DC + c) = bf16x4{(__bf16)y[0], (__bf16)y[1], (__bf16)y[2], (__bf16)y[3]};
  if (a.lse && threadIdx.x == 0) a.lse[row] = (top + flog2(l)) * kLn2;
}

namespace {
template <int DC, int DR, int M> hipError_t launch_m(const LatentArgs& a, bool merge, hipStream_t stream) {
  if (!merge) hipLaunchKernelGGL((latent_kernel<DC, DR, M>), dim3(kLatentGrid), dim3(kLatThreads), 0, stream, a);
  else hipLaunchKernelGGL((latent_merge_kernel<DC, M>), dim3(kLatentGrid, M), dim3(DC / 4), 0, stream, a);
  return hipGetLastError();
}
template <int DC, int DR> hipError_t launch_dims(const LatentArgs& a, int tile, bool merge, hipStream_t stream) {
  return tile == 16 ? launch_m<DC, DR, 16>(a, merge, stream) : tile == 32 ? launch_m<DC, DR, 32>(a, merge, stream)
                                                                          : launch_m<DC, DR, 64>(a, merge, stream);
}
}  // namespace

hipError_t launch_latent(const LatentArgs& a, int latent_dim, int tile, bool merge, hipStream_t stream) {
  return latent_dim == 512 ? launch_dims<512, 64>(a, tile, merge, stream) : launch_dims<256, 32>(a, tile, merge, stream);
}

}  // namespace pearl
