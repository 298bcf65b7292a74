// gfx950 kernels of attention over a paged cache of latent vectors (absorbed form; paper, section 4.3, Eq. 1: decode
// is bound by its cache reads, which one short row a token for all heads makes few), for up to 16 rows a sequence, and the join of what is
// cut.
//
// A cached row is (c, r), DC + DR channels; a query row (token, head) is (q_c, q_r).  s_j = scale q . (c_j, r_j), over
// keys j up to the token's position, o = sum softmax(s)_j c_j: the row is the key of every head and its latent part the
// value.  So the rows of a tile are any (token, head) pairs of a sequence, in the order of q: row rho is token rho / H, head
// rho % H.  The softmax is online, in base 2, with state in 32 bits; weights enter the second product in bf16,
// as the values do: they are rounded one by one, the sums that divide them are not.  That takes the outputs' distance from 64 bits from 0.0017 (the rounding to
// bf16 alone) to 0.0021 at most at 512 channels and 0.0023 at 256; a second part of each weight would double the second product, near half of all.
//   S^T (keys x rows) = K . Q^T    16x16x32 MFMA: A row l%16, k 8(l/16)+e; B column l%16, k 8(l/16)+e; D column l%16, row 4(l/16)+r
//   O^T (channels x rows) += V^T . P^T   16x16x16 MFMA: A row l%16, k 4(l/16)+e; B column l%16, k 4(l/16)+e: P^T is where S^T was
//
// Work is cut into equal shares of keys, in the order (sequence, tile, key), on the device from the lengths: each
// workgroup finds its share by itself.  A tile cut by shares leaves (o~, m, l) in the workspace, joined by
// latent_merge_kernel.  With tiles of 64 rows `group` workgroups next to one another on an XCD take neighbouring tiles of the same share, so that
// they read the same keys at the same time, from L2 (no sequence has two tiles of 16 rows).

#include "latent_device.h"

namespace pearl {
namespace {

// The copies of a page by a wave, 1 KiB an instruction, kRows rows' latent parts each, and then the rotated parts.
// A key is read by one workgroup here: the copies go past the caches (nt).
template <int DC, int DR> struct LatCopies {
  using Page = LatPage<DC, DR, false>;
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

  // The page at src to the one at the LDS address lds, two copies an asm.  An instruction's immediate offset advances both addresses.
  __device__ static __forceinline__ void page(const char* src, unsigned lds) {
#pragma unroll
    for (int i = 0; i < kCopies; i += 2) {
      const unsigned to = uni((int)lds + 1024 * i);
      if (i + 1 < kCopies)
        __asm__ volatile("s_mov_b32 m0, %3\n\t"
                         "s_nop 0\n\t"
                         "global_load_lds_dwordx4 %0, %2 nt\n\t"
                         "global_load_lds_dwordx4 %1, %2 offset:1024 nt"
                         :
                         : "v"(offset(i)), "v"(offset(i + 1) - 1024), "s"(src), "s"(to)
                         : "memory", "m0");
      else
        __asm__ volatile("s_mov_b32 m0, %2\n\t"
                         "s_nop 0\n\t"
                         "global_load_lds_dwordx4 %0, %1 nt"
                         :
                         : "v"(offset(i)), "s"(src), "s"(to)
                         : "memory", "m0");
    }
  }

  // Zeros in place of the rows from `valid` on.
  __device__ static __forceinline__ void clear(char* page, int valid) {
    const int l = threadIdx.x & 63;
    for (int i = valid * Page::kRowBytes + 16 * l; i < Page::kRot; i += 1024) *reinterpret_cast<u32x4*>(page + i) = u32x4{0u, 0u, 0u, 0u};
    for (int i = Page::kRot + valid * Page::kRotBytes + 16 * l; i < Page::kBytes; i += 1024)
      *reinterpret_cast<u32x4*>(page + i) = u32x4{0u, 0u, 0u, 0u};
  }
};

template <int DC, int DR> struct LatLds16 {
  char page[kLatWaves][2][LatPage<DC, DR, false>::kBytes];   // at the end of a tile: the waves' outputs
  LatNotes<DC, 16> notes;
  float max[kLatWaves][16], sum[kLatWaves][16];
  LatFind find;
};

// M = 16: what a wave holds of a tile, of which it has all rows and every fourth page.
template <int DC, int DR> struct LatRows16 {
  static constexpr int M = 16;
  using Page = LatPage<DC, DR, false>;
  using Copies = LatCopies<DC, DR>;
  static constexpr int kSteps = DC / 32, kAll = kSteps + DR / 32;
  static constexpr int kBlocks = DC / 16;           // of 16 channels
  static constexpr int kAhead = 4;                  // LDS reads of the products' operands, ahead of them
  bf16x8 q[kAll];
  f32x4 o[kBlocks], s;
  float m, l;
  int g16, l16;
  LatOperand<Page> operand;

  __device__ __forceinline__ void start(const char* queries) {
    g16 = (threadIdx.x & 63) >> 4;
    l16 = threadIdx.x & 15;
    operand.start(l16, g16);
#pragma unroll
    for (int k = 0; k < kAll; ++k) q[k] = operand.get(queries, k);
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
    auto key_of = [&](int k) { return operand.get(page, k); };
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
  __device__ __forceinline__ void raise(float to_log2) {
    const float x = fmaxf(m, xor32_max(xor16_max(largest() * to_log2)));
    const float alpha = fexp2(m - x);
    m = x;
    l *= alpha;
    scale(alpha);
  }
  __device__ __forceinline__ void scale(float f) {
#pragma unroll
    for (int d = 0; d < kBlocks; ++d) o[d] *= f;
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

}  // namespace

// Up to 16 rows a sequence: every wave takes pages of its own, two in LDS, and no barrier until the tile ends, where the four waves'
// outputs are joined in LDS.  The products are far from their limit here, what counts is that copies never pause.
// 64 sequences of 2K to 16K tokens and 16 heads, 666 MB: 110 us (6.0 TB/s; read past the caches the same bytes take 94), of which 98 in the pages;
// 5 us until the first page is asked for (lengths, cut, page ids) and 6 for the join.  One sequence of 2731 tokens: 11 us, and 5
// for the join of its 42 pieces.  Four waves that share stages of 64 keys: 143 and 31 us for both cases with their joins.
template <int DC, int DR>
__global__ __launch_bounds__(kLatThreads, 1) void latent16_kernel(LatentArgs a) {
  using Rows = LatRows16<DC, DR>;
  using Page = typename Rows::Page;
  using Copies = typename Rows::Copies;
  // of 64, 128, 192 and 256: a step of 64 sequences 121.1, 120.4, 118.9, 118.9 us, one of 400 short ones of 4 heads 57.9, 55.2, 55.1, 55.4 us
  constexpr int M = 16, kTileCost = 192;
  __shared__ __attribute__((aligned(256))) LatLds16<DC, DR> lds;
  const int tid = threadIdx.x, lane = tid & 63, w = uni(tid >> 6);
  clear_notes(lds.notes, tid);
  LatWork work;
  if (!lat_find<M, kLatWaves, kTileCost>(a, lds.find, work)) return;
  char* const buffers = lds.page[w][0];
  do {
    work.tile<M>();
    if (work.j0 >= work.j1) continue;
    const LatSeq seq = work.seq;
    const int r0 = work.r0, n_rows = work.n_rows, last = seq.ctx + work.plan.token(r0 + n_rows - 1);   // the last key
    const int p1 = min(work.j1 * kLatWaves, last / kPage + 1);
    const int first_limit = seq.ctx + work.plan.token(r0);   // keys behind it are not all rows'
    const bool in_part = last != first_limit;
    const int32_t* const bt = a.block_table + (size_t)work.b * a.bt_stride;
    lat_queries<Page>(args_anew()->q + work.row0 * (DC + DR), n_rows, buffers + Page::kBytes);
    // Ids of 64 of the wave's pages at once, lane i's page p + 4 i.  They are waited for here: the compiler, which does not know of the copies,
    // would wait in every page, for these too.
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
    if (p < p1) __asm__ volatile("s_waitcnt vmcnt(%0)" ::"n"(Copies::kCopies) : "memory");   // the queries
    else wait_copies();
    x.start(buffers + Page::kBytes);
    if (tid < M) lds.notes.limit[tid] = seq.ctx + work.plan.token(r0 + min(tid, n_rows - 1));
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
        if (last + 1 - key0 < kPage) Copies::clear(page, last + 1 - key0);   // keys that no row sees are none of the products'
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
    const bool whole = work.starts && work.ends;
    const LatArgsPtr args = args_anew();
    const float top = fmaxf(fmaxf(lds.max[0][x.l16], lds.max[1][x.l16]), fmaxf(lds.max[2][x.l16], lds.max[3][x.l16]));
    float l = 0.f;
#pragma unroll
    for (int v = 0; v < kLatWaves; ++v) l = fmaf(lds.sum[v][x.l16], fexp2(lds.max[v][x.l16] - top), l);
    if (tid < M) {
      if (!whole) reinterpret_cast<float2*>(args->part_ml)[(size_t)work.slot * M + tid] = float2{top, l};
      else if (args->lse && tid < n_rows) args->lse[work.row0 + tid] = (top + flog2(l)) * kLn2;
    }
    x.scale(fexp2(x.m - top) * (whole ? 1.f / l : 1.f));
    // outputs of a wave: rows of DC channels in 32 bits, chunk c of row r in slot c ^ r of its 16
    constexpr int kWaveBytes = M * DC * 4;
    static_assert(kWaveBytes <= 2 * Page::kBytes, "in the wave's own buffers");
#pragma unroll
    for (int d = 0; d < Rows::kBlocks; ++d)
      *reinterpret_cast<f32x4*>(buffers + x.l16 * DC * 4 + 16 * ((4 * d + x.g16) ^ x.l16)) = x.o[d];
    barrier_lds();
    // a wave every fourth row
    const int rows = whole ? n_rows : M;
#pragma unroll 2
    for (int r = w; r < rows; r += kLatWaves) {
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
        if (whole) *reinterpret_cast<bf16x4*>(args->out + (work.row0 + r) * DC + channel) = bf16x4{(__bf16)y[0], (__bf16)y[1], (__bf16)y[2], (__bf16)y[3]};
        else *reinterpret_cast<f32x4*>(args->part_o + ((size_t)work.slot * M + r) * DC + channel) = y;
      }
    }
    barrier_lds();                                  // the next tile writes all of it
    if (odd) {
      clear_notes(lds.notes, tid);
      barrier_lds();
    }
  } while (work.next(a));
  if (tid == 0) args_anew()->jobs[work.index] = work.job;
}

// Joins the partials of cut tiles: job (first row, rows, index of the first piece's workgroup, shares).  A tile's first piece is in slot
// 1 of that workgroup, the others in slot 0 of the shares that follow, in order (kLatentGrid pieces at most).  A lane takes DC / 64 channels of a
// row.  Bound by the latency of job, maxima and partials (5 to 6 us), where all workgroups cut 64-row tiles by the partials' 67 MB (15 us, 4.5 TB/s).
// Work is counted in turns of a workgroup: four rows of few pieces, a wave each, or one row of many, of which each wave takes a fourth
// (one wave with 62 pieces in a row waited for 16 times its first loads).
template <int DC, int M>
__global__ __launch_bounds__(kLatThreads) void latent_merge_kernel(LatentArgs a) {
  static_assert(kLatentGrid == kLatThreads, "a thread a job; a lane a piece");
  // at most 0, 3, 8 and 64 pieces are few: one sequence of 42 pieces 16.2, 16.4, 16.3, 21.2 us with its attention, of 8000 tokens and 128 heads 25.1,
  // 25.0, 25.0, 31.3, two prompts of 300 tokens and 128 heads 100.8, 81.9, 81.4, 81.7
  constexpr int kC = DC / 64, kFew = 8, kChunk = 4;   // kChunk: pieces asked for at once (8: the same or 1 to 4% slower)
  __shared__ float s_top[kLatWaves], s_sum[kLatWaves];
  __shared__ int s_turns[kLatWaves];
  __shared__ __attribute__((aligned(16))) int s_end[kLatentGrid];    // turns of the jobs up to each one
  __shared__ __attribute__((aligned(16))) int4 s_job[kLatentGrid];
  __shared__ __attribute__((aligned(16))) float s_o[kLatWaves][DC];
  const int tid = threadIdx.x, lane = tid & 63, w = uni(tid >> 6);
  int total = 0;
  {
    const int4 job = a.jobs[tid];
    int end = job.w <= kFew ? (job.y + kLatWaves - 1) / kLatWaves : job.y;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int y = __shfl_up(end, d);
      if (lane >= d) end += y;
    }
    if (lane == 63) s_turns[w] = end;
    __syncthreads();
#pragma unroll
    for (int v = 0; v < kLatWaves; ++v) {
      if (v == w) end += total;
      total += s_turns[v];
    }
    s_end[tid] = end;
    s_job[tid] = job;
    __syncthreads();
  }
  for (int turn = blockIdx.x; turn < total; turn += gridDim.x) {
    const int4 ends = *reinterpret_cast<const int4*>(&s_end[4 * lane]);
    const int j = __popcll(__ballot(ends.x <= turn)) + __popcll(__ballot(ends.y <= turn)) + __popcll(__ballot(ends.z <= turn)) +
                  __popcll(__ballot(ends.w <= turn));
    const int4 job = s_job[j];
    const int n = uni(job.w), rows = uni(job.y), at = turn - (j ? uni(s_end[j - 1]) : 0);
    const bool few = n <= kFew;
    const int first = few ? 0 : w, step = few ? 1 : kLatWaves, mine = (n - first + step - 1) / step;   // this wave's pieces
    const int r = few ? kLatWaves * at + w : at;
    if (r >= rows) continue;                        // only where no other wave waits for this one
    auto slot = [&](int i) { return (size_t)(i == 0 ? 2 * job.z + 1 : 2 * (job.z + i * a.group)) * M; };
    // The first pieces are asked for before their weights are known (one sequence of 42 pieces 19.1 -> 16.2 us with its attention).  Lane k holds the maximum and sum of the wave's piece k; a piece without
    // keys counts nothing, its outputs are unwritten.
    const float2 ml = lane < mine ? reinterpret_cast<const float2*>(a.part_ml)[slot(step * lane + first) + r] : float2{-FLT_MAX, kNoKeys};
    f32x4 x[kChunk][kC / 4];
    auto load = [&](int k0) {
#pragma unroll
      for (int j = 0; j < kChunk; ++j) {
        const float* const src = a.part_o + (slot(step * min(k0 + j, mine - 1) + first) + r) * DC + 4 * lane;
#pragma unroll
        for (int c = 0; c < kC; c += 4) x[j][c / 4] = *reinterpret_cast<const f32x4*>(src + 64 * c);
      }
    };
    if (mine > 0) load(0);
    const bool seen = ml.y != kNoKeys;
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
    for (int k0 = 0; k0 < mine; k0 += kChunk) {
      if (k0 > 0) load(k0);
#pragma unroll
      for (int j = 0; j < kChunk; ++j) {
        const int k = min(k0 + j, mine - 1);
        const bool use = k0 + j < mine && (all_seen >> k & 1);
        const float f = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, weight), k));
#pragma unroll
        for (int c = 0; c < kC; ++c) o[c] = use ? fmaf(f, x[j][c / 4][c % 4], o[c]) : o[c];
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
    if (!few) __syncthreads();                      // the next turn's sums
  }
}

namespace {
template <int DC, int DR> hipError_t launch_dims(const LatentArgs& a, int tile, bool merge, hipStream_t stream) {
  const dim3 grid(kLatentGrid), threads(kLatThreads), merge_grid(8 * kLatentGrid);   // as many as the card holds at once
  if (merge && tile == 16) hipLaunchKernelGGL((latent_merge_kernel<DC, 16>), merge_grid, threads, 0, stream, a);
  else if (merge) hipLaunchKernelGGL((latent_merge_kernel<DC, 64>), merge_grid, threads, 0, stream, a);
  else hipLaunchKernelGGL((latent16_kernel<DC, DR>), grid, threads, 0, stream, a);
  return hipGetLastError();
}
}  // namespace

hipError_t launch_latent(const LatentArgs& a, int latent_dim, int tile, bool merge, hipStream_t stream) {
  if (!merge && tile == 64) return launch_latent64(a, latent_dim, stream);
  return latent_dim == 512 ? launch_dims<512, 64>(a, tile, merge, stream) : launch_dims<256, 32>(a, tile, merge, stream);
}

}  // namespace pearl
