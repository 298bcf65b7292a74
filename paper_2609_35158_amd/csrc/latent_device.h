// What the gfx950 kernels of attention over latent rows (latent16.hip, latent64.hip) share: a page's place in LDS, the cut of the
// work, and values that are not finite.
#pragma once

#include "attn_device.h"
#include "rope_latent.h"

#include <float.h>

namespace pearl {
namespace {

constexpr int kLatWaves = 4;
constexpr int kLatThreads = 64 * kLatWaves;
constexpr int kLatKeysShift = 6, kLatKeys = 1 << kLatKeysShift;   // of a stage: where work is cut
// A row's maximum may lag the true one by so much (log2 units): weights are below 2^8, sums of 2^25 keys below 2^33.
constexpr float kLag = 8.f;

// In place of a row's sum in a piece of a cut tile that has no keys.  (The sum of a piece whose scores are all minus infinity is 0, its outputs are 0 or, in
// channels with values that are not finite, NaN.)
constexpr float kNoKeys = -1.f;

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
// its 16, f a permutation of the rows.  A 16 byte read of a row a lane is served 16 lanes at a time, rows 0-3 and 12-15 of one lane group with
// rows 4-11 of its neighbour: f puts these into 16 slots, given that the
// groups' chunks differ in bits 2 and 3: in step k of the scores' product, of 32 channels, group g takes channels 128 (k / 4) + 32 g + 8 (k % 4) .., of
// keys and queries alike (with neighbouring chunks in the groups such reads take twice as long: a third of all LDS cycles at 64 rows).  The transposing reads of 32 lanes take two
// chunks of each of 8 consecutive rows at M = 16 (kWide false), four chunks of 4 consecutive rows at M = 64: f keeps these apart likewise.
// Chunk c of the rotated part is in slot c ^ (r / 2) (DR = 64; at 32, where 4 rows share the banks, c ^ (0, 2, 3, 1)[r / 4]).
template <int DC, int DR, bool kWide> struct LatPage {
  static constexpr int kWidth = (DC + DR) * 2;      // bytes of a cached row
  static constexpr int kRowBytes = DC * 2, kRotBytes = DR * 2;
  static constexpr int kRot = kPage * kRowBytes;    // offset of the rotated parts
  static constexpr int kBytes = kPage * kWidth;
  static_assert(kBytes % 256 == 0 && kRowBytes % 256 == 0, "the swizzle takes address bits 4 .. 7");
  __device__ static __forceinline__ constexpr int f(int r) {
    return kWide ? ((r & 3) << 2) | ((r >> 2) & 3) : ((r & 7) << 1) | (r >> 3);
  }
  __device__ static __forceinline__ constexpr int rot_f(int r) { return DR == 64 ? (r >> 1) & 7 : 0x78 >> (2 * (r >> 2)) & 3; }
};

// Copies into LDS take their address from m0, which nothing else in these kernels uses (the compiler does not keep it across an asm).
//
// Queries: 16 rows of a cached row's width to a page in LDS, by a wave.  The last of `valid` rows stands for those behind it.
template <typename Page> __device__ __forceinline__ void lat_queries(const uint16_t* rows, int valid, const char* page) {
  const int l = threadIdx.x & 63;
  auto copy = [&](int off, int at) {
    __asm__ volatile("s_mov_b32 m0, %2\n\t"
                     "s_nop 0\n\t"
                     "global_load_lds_dwordx4 %0, %1"
                     :
                     : "v"(off), "s"(rows), "s"(uni((int)lds_address(page) + at))
                     : "memory", "m0");
  };
  constexpr int kSlots = Page::kRowBytes / 16, kChunks = Page::kRotBytes / 16;
#pragma unroll
  for (int i = 0; i < kPage * kSlots; i += 64) {
    const int r = (i + l) / kSlots;
    copy(min(r, valid - 1) * Page::kWidth + 16 * ((l % kSlots) ^ Page::f(r)), 16 * i);
  }
#pragma unroll
  for (int i = 0; i < kPage * kChunks; i += 64) {
    const int r = (i + l) / kChunks;
    copy(min(r, valid - 1) * Page::kWidth + Page::kRowBytes + 16 * ((l % kChunks) ^ Page::rot_f(r)), Page::kRot + 16 * i);
  }
}

// Where the scores' product finds a lane's operand of step k, in row l16 of a page.
template <typename Page> struct LatOperand {
  static constexpr int kSteps = Page::kRowBytes / 64;
  int at, rot;
  __device__ __forceinline__ void start(int l16, int g16) {
    at = l16 * Page::kRowBytes + 16 * ((4 * g16) ^ Page::f(l16));
    rot = Page::kRot + l16 * Page::kRotBytes + 16 * (g16 ^ Page::rot_f(l16));
  }
  __device__ __forceinline__ bf16x8 get(const char* page, int k) const {
    return as_bf16x8(*reinterpret_cast<const u32x4*>(page + (k < kSteps ? (at ^ (16 * (k & 3))) + 256 * (k >> 2) : rot ^ (64 * (k - kSteps)))));
  }
};

// What finding a workgroup's share takes.
struct LatFind {
  long long sum[8], before;                         // a wave each
  int found, bad;
};

// Both kernels' notes on a tile.
template <int DC, int M> struct LatNotes {
  int odd[DC];                                      // of each channel: the first key with a value that is not finite and ..
  int any_odd;                                      // .. whether there is one, among those that only some of the tile's rows see
  int limit[M];                                     // the last key that a row sees
};

// ---- the plan --------------------------------------------------------------------------------------------------------
// A sequence's rows are cut into tiles of `tile_rows` (group * M).  Work is measured in keys: tile u costs its keys, tile_cost (its
// start, join and stores, in the time of so many keys) and what its rows add, such that the cost of tiles 0 .. u - 1 is u (ctx + tile_cost) +
// (u (u + 1) slope >> 8), slope being 256 times half the tokens of a tile.

struct LatSeq {
  int q_start, q_len, ctx;
};

struct LatPlan {
  int tile_rows, tile_shift, slope, heads;          // tile_rows = 1 << tile_shift
  int tile_cost;
  unsigned long long per_head;                      // 2^35 / heads, rounded up
  // row / heads: exact, as rows are below 2^28 and heads 128 at most
  __device__ __forceinline__ int token(int row) const { return (int)(((unsigned long long)(unsigned)row * per_head) >> 35); }
  __device__ __forceinline__ long long before(const LatSeq& s, long long u) const {
    return u * (s.ctx + tile_cost) + ((u * (u + 1) * slope) >> 8);
  }
  __device__ __forceinline__ int tiles(const LatSeq& s) const {
    return (s.q_len * heads + tile_rows - 1) >> tile_shift;   // at most 2^21 tokens of 128 heads
  }
  // stages of the keys that rows up to `row` see
  __device__ __forceinline__ int stages(const LatSeq& s, int row) const {
    return (s.ctx + token(row) + kLatKeys) >> kLatKeysShift;
  }
  // the stage at which cost `at` of a tile that starts at 0 is cut
  __device__ __forceinline__ int stage_at(long long at, int stages) const {
    const long long j = (at - tile_cost) >> kLatKeysShift;
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
  __device__ __forceinline__ LatShares(long long total, int n) : shares(n) {
    each = uni64((long long)((double)total / (double)n));       // exact, below 2^53, or off by 1
    while (each * n > total) --each;
    while (total - each * n >= n) ++each;
    more = (int)(total - each * n);
  }
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

__device__ __forceinline__ long long lane64(long long x, int l) {
  const unsigned lo = __builtin_amdgcn_readlane((int)x, l), hi = __builtin_amdgcn_readlane((int)(x >> 32), l);
  return (long long)((unsigned long long)hi << 32 | lo);
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
    j0 = starts ? 0 : min(plan.stage_at(lo - t0, all_stages), stages);
    j1 = ends ? stages : min(plan.stage_at(hi - t0, all_stages), stages);
    if (starts && !ends) job = int4{(int)row0, n_rows, index, cut.of(t1 - 1) - share + 1};
    // a piece of a cut tile without keys, whose outputs stay unwritten
    if (j0 >= j1 && !(starts && ends) && threadIdx.x < M)
      reinterpret_cast<float2*>(args_anew()->part_ml)[(size_t)slot * M + threadIdx.x] = float2{-FLT_MAX, kNoKeys};
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

// Finds the workgroup's share; false: it has none.  Workgroups with one number modulo `group` (a power of two) take the same member of the
// tiles, and shares of an XCD's workgroups follow one another.
template <int M, int kWaves, int kTileCost> __device__ __forceinline__ bool lat_find(const LatentArgs& a, LatFind& lds, LatWork& work) {
  constexpr int kThreads = 64 * kWaves;
  const int tid = threadIdx.x, lane = tid & 63, w = uni(tid >> 6);
  const int group = a.group;
  work.plan = LatPlan{group * M, __builtin_ctz(group * M), a.slope, a.heads, kTileCost, a.per_head};
  work.job = int4{0, 0, 0, 0};
  // Up to 64 sequences: a lane each, in every wave; nothing goes through LDS, and no length is read twice (one sequence of 2731 tokens 17.1 ->
  // 16.6 us).
  const bool few = a.batch <= 64;
  const int per = few ? 1 : (a.batch + kThreads - 1) / kThreads, first = few ? lane : tid * per;
  LatSeq seq = {0, 0, 0};
  long long mine = 0;
  bool bad = false;
  if (!few) {
    if (tid == 0) lds.bad = 0;
    __syncthreads();
  }
  for (int i = 0; i < per; ++i) {
    const int b = first + i;
    if (b >= a.batch) break;
    seq = lat_seq(a, b);
    if (lat_bad(a, seq)) bad = true;
    else mine += work.plan.before(seq, work.plan.tiles(seq));
  }
  long long upto = mine;                            // of this wave's lanes up to this one
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const long long y = shfl_up64(upto, d);
    if (lane >= d) upto += y;
  }
  long long total = 0;
  if (few) {
    bad = __ballot(bad) != 0;
    total = lane64(upto, 63);
  } else {
    if (bad) lds.bad = 1;
    if (lane == 63) lds.sum[w] = upto;
    __syncthreads();
    bad = uni(lds.bad) != 0;
#pragma unroll
    for (int v = 0; v < kWaves; ++v) {
      if (v == w) upto += total;
      total += uni64(lds.sum[v]);
    }
  }
  if (blockIdx.x == 0 && tid == 0) a.ws_hdr[kHdrError] = bad;
  int shares = (int)gridDim.x / group;
  if (total < (long long)shares << a.min_share_shift) shares = (int)max(1ll, total >> a.min_share_shift);
  // the workgroups that have a share are spread over the XCDs; the others have the numbers behind theirs
  const int x = (int)(blockIdx.x % kNumXcd), i = (int)(blockIdx.x / kNumXcd), n = (shares + kNumXcd - 1) / kNumXcd * group;
  work.index = i < n ? x * n + i : kNumXcd * n + x * ((int)gridDim.x / kNumXcd - n) + i - n;
  work.share = work.index >> __builtin_ctz(group);
  work.member = work.index & (group - 1);
  if (bad || total == 0 || work.share >= shares) {
    if (tid == 0) a.jobs[work.index] = work.job;
    return false;
  }
  work.cut = LatShares(total, shares);
  const long long lo = work.cut.start(work.share);
  work.lo = lo;
  work.hi = work.cut.start(work.share + 1);
  if (few) {
    work.b = __builtin_ctzll(__ballot(upto > lo));  // lo is below the total, that of the last lane
    work.at = lane64(upto - mine, work.b);
    work.seq = LatSeq{__builtin_amdgcn_readlane(seq.q_start, work.b), __builtin_amdgcn_readlane(seq.q_len, work.b),
                      __builtin_amdgcn_readlane(seq.ctx, work.b)};
  } else {
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
  }
  work.u = work.plan.tile_at(work.seq, lo - work.at);
  return true;
}

// Keys that only some of the rows see have weight 0 in the others, and 0 times a value that is not finite is NaN.  So such a value becomes 0, in the
// page at hand (key0: its first key), and its channel is noted.  (The value is part of its key too: in rows that see it its score is NaN or infinite, so its
// channel's output is NaN there, if not the whole row, which is what the end of the tile makes of the note.)
// Rows r0 .. r1 - 1 of the page.
template <typename Page, int DC, int M> __device__ __forceinline__ void note_odd(char* page, int key0, LatNotes<DC, M>& notes, int r0 = 0, int r1 = kPage) {
  for (int i = r0 * (DC / 8) + (threadIdx.x & 63); i < r1 * (DC / 8); i += 64) {
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

// By the first 256 of the threads that call it.
template <int DC, int M> __device__ __forceinline__ void clear_notes(LatNotes<DC, M>& notes, int thread) {
  if (thread >= 256) return;
  for (int i = thread; i < DC; i += 256) notes.odd[i] = INT32_MAX;
  if (thread == 0) notes.any_odd = 0;
}

}  // namespace
}  // namespace pearl
