// gfx950 kernel of attention over a paged cache of latent vectors (what it computes: latent16.hip) for sequences of more than 16 rows:
// tiles of 64 rows.
//
// A workgroup has 8 waves, two on each SIMD: four take the scores and their weights, four the values, a stage (32 keys, 2 pages; at 256 channels
// 64 keys, 4 pages) behind, so that the one's products run while the other weighs, waits or copies.
//   S^T (keys x rows) = K . Q^T: score wave w has the keys of every second page from w % 2 on and rows 32 (w / 2) .., Q in registers (16x16x32 MFMA: A row l%16,
//                       k 8(l/16)+e; B column l%16, k 8(l/16)+e; D column l%16, row 4(l/16)+r);
//   O^T (channels x rows) += V^T . P^T: value wave w has a quarter of the channels and all rows, V^T by transposing reads of the same LDS
//                       rows (32x32x16 MFMA: A row l%32, k 8(l/32)+e; B column l%32, k 8(l/32)+e; D column l%32, row r%4 + 8(r/4) + 4(l/32)).
// Step t between two barriers: scores of stage t, values of stage t - 1, and the copies of stage t + 2 go out (four stages in LDS: t - 1 and t in
// use, t + 1 on its way or there; at 256 channels three, of twice the keys, and the copies of stage t + 1).
// A row's maximum is common to all.  It may lag the true one by kLag (log2 units), so most stages go on with the old one.  Where some score
// is further above, a score wave weighs with a maximum of its own, rounded up to a whole number, and behind the next barrier all waves take up the
// largest; what was weighed with another is scaled by a power of two.

// Bound by the score and value waves' chains: a step of 32 keys takes about 1950 cycles, of which the matrix units are busy 1088 (54%).  A value
// wave's: 150 for weights and flag, 600 to 780 for seven to nine copies (36 KiB a step pass at 20 cycles a KiB), 620 for its products, 350 for operands,
// arrival and barrier; a score wave's: 870 for scores beside the others' products, 430 for weights, 140 for sums, the rest waits; at 512 channels it makes
// two of the copies behind its scores (2.56 -> 2.51 ms for the long turns below; four 2.57, or behind the weights 2.54).
// Measured at 512 channels: turns of 500 to 2000 tokens on contexts of 4K to 16K, 16 heads, 2.90 TFLOP, 2.51 ms (1155 TF/s; the library's product of
// two 8192 x 8192 matrices 1350); of 64 to 400 tokens 0.83 ms (1115 TF/s).  A step of 32 sequences with 128 heads, 282 MB and 66 GFLOP, 84 us: bytes on
// their way, two stages a compute unit.  At 256 channels six prompts of 300 to 2000 tokens, 115 GFLOP, 182 us.
// Tried: four waves that do both in turn, stages of 64 keys, two in LDS (2.69 ms); eight in lockstep or in two alternating sets (3.4 to 3.5 ms); copies
// spread among the products (2.78 for 2.66 ms on one card: the copies go out while the score waves have the matrix units); touching the lines of later stages so that they
// are in L2 (2.90 for 2.50 ms).

#include "latent_device.h"

namespace pearl {
namespace {

constexpr int kWaves64 = 8;

template <int DC> struct LatStage {
  static constexpr int kPages = DC == 512 ? 2 : 4, kKeys = kPage * kPages, kShift = DC == 512 ? 5 : 6;
  static constexpr int kStages = DC == 512 ? 4 : 3, kLead = kStages - 2;   // kLead: stages on their way
  static constexpr int kRowBytes = 2 * kKeys;       // of a row's weights; chunk c of row r is in slot c ^ f(r)
  __device__ static __forceinline__ constexpr int f(int r) { return DC == 512 ? (r >> 2) & 3 : (r >> 1) & 7; }
};

template <int DC, int DR> struct LatLds64 {
  using Page = LatPage<DC, DR, true>;
  using Stage = LatStage<DC>;
  char page[Stage::kStages][Stage::kPages][Page::kBytes];
  char p[2][64 * Stage::kRowBytes];                 // weights of a stage
  LatNotes<DC, 64> notes;
  int limit2[64];                                   // notes.limit of every other tile
  float max[2][2][64];                              // of a stage, of every second page: the rows' maxima that their weights were taken with
  float sum[2][64];                                 // at the end of a tile: the rows' sums, in parts
  int flag[2];                                      // the last step with some score far above its row's maximum, of even and odd ones
  LatFind find;
};

// The copies of a stage, 1 KiB an instruction: half a page (8 rows) a value wave or (256 channels) a page, of which a score wave makes kPairs pairs.
template <int DC, int DR> struct LatMyCopies {
  using Page = LatPage<DC, DR, true>;
  static constexpr int kMine = DC == 512 ? 8 : 16;  // rows
  static constexpr int kRows = 1024 / Page::kRowBytes, kLatent = kMine / kRows, kCopies = kLatent + 1;
  static constexpr int kPairs = DC == 512 ? 1 : 0;  // that a score wave makes, the last ones of the latent parts
  static constexpr int kGiven = kLatent - 2 * kPairs, kGivenRow = kRows * kGiven;
  static_assert(kMine * Page::kRotBytes == 1024, "one instruction takes the rotated parts");
  int off[kCopies];                                 // the lane's source offsets in the page
  __device__ __forceinline__ void start(int half) {
    const int l = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < kLatent; ++i) {
      const int r = 8 * half + kRows * i + (kRows == 2 ? l >> 5 : 0), slot = kRows == 2 ? l & 31 : l;
      off[i] = r * Page::kWidth + 16 * (slot ^ Page::f(r)) - 1024 * (i & 1);   // the second of a pair has 1 KiB as its immediate
    }
    constexpr int kChunks = Page::kRotBytes / 16;
    const int r = l / kChunks + 8 * half;
    off[kLatent] = r * Page::kWidth + Page::kRowBytes + 16 * ((l % kChunks) ^ Page::rot_f(r));
  }
  // Copies i and i + 1 (the last one, of the rotated parts, by itself) to the page at the LDS address lds, if `go` (the branches are the
  // instructions' own: ones that the compiler sees split the products' code, with moves of all outputs between the parts); past the caches (nt) if it is 2,
  // where no other workgroup reads the keys (64 sequences of 64 heads: 140 instead of 160 us; with two workgroups to the keys of 128 heads
  // 216 instead of 209, with eight 3190 instead of 2590).
  __device__ __forceinline__ void copy2(int i, int half, const char* src, unsigned lds, int go) const {
    if (i < kLatent) {
      const unsigned to = uni((int)lds + half * 8 * Page::kRowBytes + 1024 * i);
      __asm__ volatile(
          "s_cmp_eq_u32 %4, 0\n\t"
          "s_cbranch_scc1 .Lno_copy%=\n\t"
          "s_mov_b32 m0, %3\n\t"
          "s_cmp_eq_u32 %4, 2\n\t"
          "s_cbranch_scc1 .Lpast%=\n\t"
          "global_load_lds_dwordx4 %0, %2\n\t"
          "global_load_lds_dwordx4 %1, %2 offset:1024\n\t"
          "s_branch .Lno_copy%=\n"
          ".Lpast%=:\n\t"
          "global_load_lds_dwordx4 %0, %2 nt\n\t"
          "global_load_lds_dwordx4 %1, %2 offset:1024 nt\n"
          ".Lno_copy%=:"
          :
          : "v"(off[i]), "v"(off[i + 1]), "s"(src), "s"(to), "s"(uni(go))
          : "memory", "scc", "m0");
    } else {
      const unsigned to = uni((int)lds + Page::kRot + 1024 * half);
      __asm__ volatile(
          "s_cmp_eq_u32 %3, 0\n\t"
          "s_cbranch_scc1 .Lno_copy%=\n\t"
          "s_mov_b32 m0, %2\n\t"
          "s_cmp_eq_u32 %3, 2\n\t"
          "s_cbranch_scc1 .Lpast%=\n\t"
          "global_load_lds_dwordx4 %0, %1\n\t"
          "s_branch .Lno_copy%=\n"
          ".Lpast%=:\n\t"
          "global_load_lds_dwordx4 %0, %1 nt\n"
          ".Lno_copy%=:"
          :
          : "v"(off[kLatent]), "s"(src), "s"(to), "s"(uni(go))
          : "memory", "scc", "m0");
    }
  }
  // Zeros in place of the latent parts of rows r0 .. r1 - 1 from row `valid` of the page on (of rotated parts scores alone are made, which are masked).
  __device__ static __forceinline__ void clear(char* page, int r0, int r1, int valid) {
    for (int i = max(valid, r0) * Page::kRowBytes + 16 * (threadIdx.x & 63); i < r1 * Page::kRowBytes; i += 1024)
      *reinterpret_cast<u32x4*>(page + i) = u32x4{0u, 0u, 0u, 0u};
  }
};

// A score wave: pages `page`, page + 2, .. of a stage, rows row0 ..
template <int DC, int DR> struct LatScores {
  using Page = LatPage<DC, DR, true>;
  using Lds = LatLds64<DC, DR>;
  using Stage = LatStage<DC>;
  static constexpr int kAll = (DC + DR) / 32, kMine = Stage::kPages / 2;
  static constexpr int kAhead = 4;                  // LDS reads of the product's operands, ahead of it
  bf16x8 q[2][kAll];
  f32x4 s[kMine][2];
  float m[2], l[2], sum[2], ref[2];
  LatOperand<Page> operand;
  int page, row0, g16, l16, place;                  // place: of the lane's weights among a stage's (the next page's: ^ 64)

  // The queries come as pages through the stages that are not on their way yet; wave 2 h + p brings rows 32 h + 16 p ..
  __device__ static __forceinline__ const char* queries(const Lds& lds, int i) {
    return lds.page[Stage::kLead + i / Stage::kPages][i % Stage::kPages];
  }
  __device__ __forceinline__ void start(Lds& lds, int wave, const uint16_t* rows, int n_rows) {
    page = wave & 1;
    const int h = wave >> 1;
    row0 = 32 * h;
    const int first = min(row0 + 16 * page, n_rows - 1);
    lat_queries<Page>(rows + first * (DC + DR), min(n_rows - first, kPage), queries(lds, 2 * h + page));
    g16 = (threadIdx.x & 63) >> 4;
    l16 = threadIdx.x & 15;
    operand.start(l16, g16);
    place = (row0 + l16) * Stage::kRowBytes + 16 * ((2 * page + (g16 >> 1)) ^ Stage::f(l16)) + 8 * (g16 & 1);
    wait_copies();
    barrier_lds();
#pragma unroll
    for (int rg = 0; rg < 2; ++rg) {
#pragma unroll
      for (int k = 0; k < kAll; ++k) q[rg][k] = operand.get(queries(lds, 2 * h + rg), k);
      m[rg] = -FLT_MAX;
      l[rg] = sum[rg] = 0.f;
      ref[rg] = -FLT_MAX;
      if (g16 < 2) lds.max[g16][page][row0 + 16 * rg + l16] = -FLT_MAX;
    }
  }
  // The products; flag: of the step before, asked for among the operands' reads.
  __device__ __forceinline__ int scores(const Lds& lds, const char* stage, int step) {
    const int flag = lds.flag[(step - 1) & 1];
    const char* const at_page = stage + page * Page::kBytes;
    auto key_of = [&](int i) { return operand.get(at_page + i / kAll * 2 * Page::kBytes, i % kAll); };
    bf16x8 key[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) key[i] = key_of(i);
#pragma unroll
    for (int i = 0; i < kMine * kAll; ++i) {
      const int h = i / kAll, k = i % kAll;
      const bf16x8 x = key[i % kAhead];
      if (k == 0) s[h][0] = s[h][1] = f32x4{0.f, 0.f, 0.f, 0.f};
      s[h][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, q[0][k], s[h][0], 0, 0, 0);
      s[h][1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, q[1][k], s[h][1], 0, 0, 0);
      if (i + kAhead < kMine * kAll) key[i % kAhead] = key_of(i + kAhead);
      __builtin_amdgcn_sched_barrier(0);
    }
    return uni(flag);
  }
  __device__ __forceinline__ void mask(const int* limits, int key0) {
#pragma unroll
    for (int rg = 0; rg < 2; ++rg) {
      const int limit = limits[row0 + 16 * rg + l16] - key0 - kPage * page - 4 * g16;
#pragma unroll
      for (int h = 0; h < kMine; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (2 * kPage * h + r > limit) s[h][rg][r] = -__builtin_inff();
    }
  }
  __device__ __forceinline__ float largest(int rg) const {
    float x = fmaxf(fmaxf(s[0][rg][0], s[0][rg][1]), fmaxf(s[0][rg][2], s[0][rg][3]));
#pragma unroll
    for (int h = 1; h < kMine; ++h) x = fmaxf(x, fmaxf(fmaxf(s[h][rg][0], s[h][rg][1]), fmaxf(s[h][rg][2], s[h][rg][3])));
    return x;
  }
  __device__ __forceinline__ void weigh(Lds& lds, int step, float scale) {
    float p[kMine][2][4], top = -FLT_MAX;
    auto weights = [&](int rg) {
#pragma unroll
      for (int h = 0; h < kMine; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r) p[h][rg][r] = fexp2(fmaf(s[h][rg][r], scale, -ref[rg]));
    };
#pragma unroll
    for (int rg = 0; rg < 2; ++rg) {
      ref[rg] = m[rg];
      weights(rg);
      top = fmaxf(top, fmaf(largest(rg), scale, -m[rg]));
    }
    if (__ballot(top > kLag)) {
#pragma unroll
      for (int rg = 0; rg < 2; ++rg) {
        ref[rg] = fmaxf(m[rg], ceilf(xor32_max(xor16_max(largest(rg) * scale))));
        weights(rg);
        if (g16 == 0) lds.max[step & 1][page][row0 + 16 * rg + l16] = ref[rg];
      }
      lds.flag[step & 1] = step;
    }
    char* const to = lds.p[step & 1];
#pragma unroll
    for (int rg = 0; rg < 2; ++rg) {
      sum[rg] = 0.f;
#pragma unroll
      for (int h = 0; h < kMine; ++h) {
        const float* const x = p[h][rg];
        sum[rg] += (x[0] + x[1]) + (x[2] + x[3]);
        *reinterpret_cast<bf16x4*>(to + (place ^ (64 * h)) + kPage * Stage::kRowBytes * rg) = bf16x4{(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]};
      }
    }
  }
  // Behind the barrier after weigh(step): the stage's sums, and new maxima if there are any (flag == step), with the weights in LDS scaled to
  // them.  A wave's maxima in LDS are older ones, no larger, where its own scores are near them.
  __device__ __forceinline__ void take_up(Lds& lds, int step, int flag) {
    if (flag == step) {
#pragma unroll
      for (int rg = 0; rg < 2; ++rg) {
        const int r = row0 + 16 * rg + l16;
        const float x = fmaxf(m[rg], fmaxf(lds.max[step & 1][0][r], lds.max[step & 1][1][r])), f = fexp2(ref[rg] - x);
        l[rg] *= fexp2(m[rg] - x);
        sum[rg] *= f;
        m[rg] = x;
#pragma unroll
        for (int h = 0; h < kMine; ++h) {
          bf16x4& p = *reinterpret_cast<bf16x4*>(lds.p[step & 1] + (place ^ (64 * h)) + kPage * Stage::kRowBytes * rg);
          p = bf16x4{(__bf16)((float)p[0] * f), (__bf16)((float)p[1] * f), (__bf16)((float)p[2] * f), (__bf16)((float)p[3] * f)};
        }
      }
      barrier_lds();
    }
    l[0] += sum[0];
    l[1] += sum[1];
  }
  __device__ __forceinline__ void sums(Lds& lds) {
#pragma unroll
    for (int rg = 0; rg < 2; ++rg) {
      const float x = xor32_add(xor16_add(l[rg]));
      if (g16 == 0) lds.sum[page][row0 + 16 * rg + l16] = x;
    }
  }
};

// A value wave: a quarter of the channels of all rows.
template <int DC, int DR> struct LatValues {
  using Page = LatPage<DC, DR, true>;
  using Lds = LatLds64<DC, DR>;
  using Stage = LatStage<DC>;
  static constexpr int kTiles = DC / 4 / 32, kAll = Stage::kPages * kTiles;   // of 32 channels
  static constexpr int kAhead = 4;
  f32x16 o[kTiles][2];
  float m[2];                                       // of rows l32 and 32 + l32
  bf16x8 p[Stage::kPages][2], value[kAhead];
  int channel0, half, l32, at;

  __device__ __forceinline__ void start(int wave) {
    channel0 = DC / 4 * wave;
    half = (threadIdx.x & 63) >> 5;
    l32 = threadIdx.x & 31;
    const int j = l32 & 15, r = 8 * half + (j >> 2), c = channel0 / 8 + 2 * (l32 >> 4) + ((j >> 1) & 1);
    at = r * Page::kRowBytes + 16 * ((c & ~15) | ((c & 15) ^ Page::f(r))) + 8 * (j & 1);
    m[0] = m[1] = -FLT_MAX;
#pragma unroll
    for (int d = 0; d < kTiles; ++d)
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][t][r] = 0.f;
  }
  // New maxima.  In asm, in place: the compiler would copy all outputs to and from other registers, in every step.  It does not know there
  // that products still write them, so they are waited for (16 passes, 19 wait states at most).
  __device__ __forceinline__ void take_up(const Lds& lds, int step) {
    float alpha[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const float x = fmaxf(m[t], fmaxf(lds.max[step & 1][0][32 * t + l32], lds.max[step & 1][1][32 * t + l32]));
      alpha[t] = fexp2(m[t] - x);
      m[t] = x;
    }
#pragma unroll
    for (int d = 0; d < kTiles; ++d)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        f32x16& y = o[d][t];
        __asm__ volatile(
            "s_nop 15\n\t"
            "s_nop 7\n\t"
            "v_mul_f32 %0, %0, %16\n\t"
            "v_mul_f32 %1, %1, %16\n\t"
            "v_mul_f32 %2, %2, %16\n\t"
            "v_mul_f32 %3, %3, %16\n\t"
            "v_mul_f32 %4, %4, %16\n\t"
            "v_mul_f32 %5, %5, %16\n\t"
            "v_mul_f32 %6, %6, %16\n\t"
            "v_mul_f32 %7, %7, %16\n\t"
            "v_mul_f32 %8, %8, %16\n\t"
            "v_mul_f32 %9, %9, %16\n\t"
            "v_mul_f32 %10, %10, %16\n\t"
            "v_mul_f32 %11, %11, %16\n\t"
            "v_mul_f32 %12, %12, %16\n\t"
            "v_mul_f32 %13, %13, %16\n\t"
            "v_mul_f32 %14, %14, %16\n\t"
            "v_mul_f32 %15, %15, %16\n\t"
            "s_nop 3"
            : "+v"(y[0]), "+v"(y[1]), "+v"(y[2]), "+v"(y[3]), "+v"(y[4]), "+v"(y[5]), "+v"(y[6]), "+v"(y[7]), "+v"(y[8]), "+v"(y[9]),
              "+v"(y[10]), "+v"(y[11]), "+v"(y[12]), "+v"(y[13]), "+v"(y[14]), "+v"(y[15])
            : "v"(alpha[t]));
      }
  }
  // Operand i of a stage's products: page i / kTiles, channels 32 (i % kTiles) .. of the wave's.
  __device__ __forceinline__ bf16x8 value_of(const char* stage, int i) const {
    // at: the lane's row of 8 (l / 32) + 0 .. 3 of the values, channels of tile 0; four rows further the swizzle differs in chunk bit 0
    const int at4 = (at ^ 16) + 4 * Page::kRowBytes;
    const char* const page = stage + i / kTiles * Page::kBytes;
    return concat_tr(lds_read_tr(page, at ^ (64 * (i % kTiles))), lds_read_tr(page, at4 ^ (64 * (i % kTiles))));
  }
  __device__ __forceinline__ void first(const char* stage) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) value[i] = value_of(stage, i);
  }
  __device__ __forceinline__ void weights(const Lds& lds, int step) {
    const char* const from = lds.p[step & 1] + l32 * Stage::kRowBytes;
#pragma unroll
    for (int page = 0; page < Stage::kPages; ++page)
#pragma unroll
      for (int t = 0; t < 2; ++t)
        p[page][t] = as_bf16x8(*reinterpret_cast<const u32x4*>(from + 32 * Stage::kRowBytes * t + 16 * ((2 * page + half) ^ Stage::f(l32))));
  }
  // The stage's products, behind first() and weights().
  __device__ __forceinline__ void add(const char* stage) {
#pragma unroll
    for (int i = 0; i < kAll; ++i) {
      const int page = i / kTiles, d = i % kTiles;
      const bf16x8 x = value[i % kAhead];
      o[d][0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, p[page][0], o[d][0], 0, 0, 0);
      o[d][1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, p[page][1], o[d][1], 0, 0, 0);
      if (i + kAhead < kAll) value[i % kAhead] = value_of(stage, i + kAhead);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
};

}  // namespace

template <int DC, int DR>
__global__ __launch_bounds__(64 * kWaves64, 2) void latent64_kernel(LatentArgs a) {
  using Page = LatPage<DC, DR, true>;
  using Copies = LatMyCopies<DC, DR>;
  using Stage = LatStage<DC>;
  using Lds = LatLds64<DC, DR>;
  // 512 channels, of 64, 128, 192 and 256: two prompts of 300 tokens and 128 heads 102, 88, 84, 80 us; 256 channels, of 64, 256, 512 and 768: six
  // prompts of up to 2000 tokens 288, 218, 182, 186 us
  constexpr int kTileCost = DC == 512 ? 256 : 512;
  constexpr int M = 64, kStages = Stage::kStages, kLead = Stage::kLead, kStageShift = Stage::kShift, kStageKeys = Stage::kKeys;
  __shared__ __attribute__((aligned(256))) Lds lds;
  const int tid = threadIdx.x, w = uni(tid >> 6);
  clear_notes(lds.notes, tid);
  if (tid == 0) lds.flag[0] = lds.flag[1] = -1;
  LatWork work;
  if (!lat_find<M, kWaves64, kTileCost>(a, lds.find, work)) return;
  int step = 0;                                     // of the workgroup, over all tiles
  bool odd_before = false;                          // the value waves': the tile before left notes
  int* limits = lds.notes.limit;                    // in turn with limit2: the value waves may still read the tile's before
  do {
    work.tile<M>();
    if (work.j0 >= work.j1) continue;
    const LatSeq seq = work.seq;
    const int r0 = work.r0, n_rows = work.n_rows, last = seq.ctx + work.plan.token(r0 + n_rows - 1);   // the last key
    const int first_limit = seq.ctx + work.plan.token(r0);   // keys behind it are not all rows'
    constexpr int kCut = kLatKeys / kStageKeys;
    const int i0 = kCut * work.j0, n = min(kCut * work.j1, (last >> kStageShift) + 1) - i0;   // stages
    const bool in_part = last != first_limit;
    auto look = [&](int i) { return in_part && ((i0 + i) << kStageShift) + kStageKeys - 1 > first_limit; };   // keys that rows see in part
    if (tid < M) limits[tid] = seq.ctx + work.plan.token(r0 + min(tid, n_rows - 1));
    const int part = DC == 512 ? w & 1 : 0, page = DC == 512 ? (w >> 1) & 1 : w & 3;   // this wave brings rows from 8 part on of a stage's page `page`
    const int pages = last / kPage + 1;
    const int32_t* const bt = a.block_table + (size_t)work.b * a.bt_stride;
    // Ids of 64 stages' pages at once (the last one where there is none; zeros take its place).  They are waited for here: the
    // compiler, which does not know of the copies, would wait in every step, for these too.
    auto ids_from = [&](int i) {
      int ids = bt[min(Stage::kPages * (i0 + i + (tid & 63)) + page, pages - 1)];
      __asm__ volatile("" : "+v"(ids));
      return ids;
    };
    auto source = [&](int ids, int i) {             // of stage i
      const int id = __builtin_amdgcn_readlane(ids, i & 63);
      return reinterpret_cast<const char*>(a.cache) + (size_t)clamp_page(id, a.num_pages) * Page::kBytes;
    };
    const unsigned pages_at = lds_address(lds.page[0][page]);
    constexpr int kStageBytes = Stage::kPages * Page::kBytes;
    const int how = a.group == 1 ? 2 : 1;
    if (w < 4) {
      LatScores<DC, DR> x;
      __builtin_amdgcn_s_setprio(3);
      x.start(lds, w, args_anew()->q + work.row0 * (DC + DR), n_rows);
      Copies copies;
      copies.start(part);
      int ids = ids_from(0);
#pragma unroll 1
      for (int i = 0; i <= n; ++i, ++step) {
        const char* src = nullptr;
        if constexpr (Copies::kPairs > 0) {
          if (((i + kLead) & 63) == 0) ids = ids_from(i + kLead);
          src = source(ids, i + kLead);
          if (i + 1 < n) __asm__ volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * Copies::kPairs) : "memory");
          else wait_copies();
          const int valid = last + 1 - ((i0 + i) << kStageShift) - kPage * page;
          if (i > kLead && i < n && valid < kPage)
            Copies::clear(lds.page[i % kStages][page], 8 * part + Copies::kGivenRow, 8 * part + Copies::kMine, max(valid, 0));
        }
        barrier_lds();
        const int key0 = (i0 + i) << kStageShift;
        const int flag = i < n ? x.scores(lds, lds.page[i % kStages][0], step) : uni(lds.flag[(step - 1) & 1]);
        if (i > 0) {
#pragma unroll
          for (int c = Copies::kGiven; c < Copies::kLatent; c += 2)
            copies.copy2(c, part, src, pages_at + (i + kLead) % kStages * kStageBytes, i + kLead < n ? how : 0);
          x.take_up(lds, step - 1, flag);
          if (look(i - 1)) barrier_lds();           // while the value waves see to values that are not finite
        }
        if (i == n) continue;
        if (key0 + kStageKeys - 1 > first_limit) x.mask(limits, key0);
        x.weigh(lds, step, a.scale_log2);
      }
      x.sums(lds);
      barrier_lds();
    } else {
      Copies copies;
      copies.start(part);
      int ids = ids_from(0);
      LatValues<DC, DR> x;
      auto bring = [&](int i) {
        const char* const src = source(ids, i);
#pragma unroll
        for (int c = 0; c < Copies::kCopies; c += 2) copies.copy2(c, part, src, pages_at + i % kStages * kStageBytes, how);
      };
      bring(0);
      if (kLead > 1 && n > 1) bring(1);
      x.start(w - 4);
      barrier_lds();                                // the queries are there
      if (odd_before) clear_notes(lds.notes, tid - 256);   // all have left the tile before
      odd_before = false;
      // Behind it a stage of this wave's is there for all, and the one after it on its way.
      auto arrive = [&](int i) {
        if (kLead > 1 && i + 1 < n) {
          if (i == 0) __asm__ volatile("s_waitcnt vmcnt(%0)" ::"n"(Copies::kCopies) : "memory");
          else __asm__ volatile("s_waitcnt vmcnt(%0)" ::"n"(Copies::kCopies - 2 * Copies::kPairs) : "memory");
        } else {
          wait_copies();
        }
        const int valid = last + 1 - ((i0 + i) << kStageShift) - kPage * page;   // keys that no row sees are none of the products'
        if (i < n && valid < kPage) Copies::clear(lds.page[i % kStages][page], 8 * part, 8 * part + (i > kLead ? Copies::kGivenRow : Copies::kMine), max(valid, 0));
        barrier_lds();
      };
      arrive(0);
      if (n > kLead) bring(kLead);
      ++step;
#pragma unroll 1
      for (int i = 1; i <= n; ++i, ++step) {
        const char* const stage = lds.page[(i - 1) % kStages][0];
        x.first(stage);                             // before the weights are there
        if (((i + kLead) & 63) == 0) ids = ids_from(i + kLead);
        const char* const src = source(ids, i + kLead);
        arrive(i);
        if (look(i - 1)) {
          note_odd<Page>(lds.page[(i - 1) % kStages][page], ((i0 + i - 1) << kStageShift) + kPage * page, lds.notes, 8 * part, 8 * part + Copies::kMine);
          barrier_lds();
          x.first(stage);
        }
        const int flag = lds.flag[(step - 1) & 1];
        x.weights(lds, step - 1);
        if (uni(flag) == step - 1) {
          x.take_up(lds, step - 1);
          barrier_lds();
          x.weights(lds, step - 1);
        }
        // All copies at once, while the score waves have the matrix units; these waves' products are made while the others weigh.
        const int more = i + kLead < n ? how : 0;
#pragma unroll
        for (int c = 0; c < Copies::kCopies; c += 2)
          if (c < Copies::kGiven || c == Copies::kLatent) copies.copy2(c, part, src, pages_at + (i + kLead) % kStages * kStageBytes, more);
        x.add(stage);
      }
      // ---- the output or the partial
      barrier_lds();
      const LatArgsPtr args = args_anew();
      const bool odd = uni(lds.notes.any_odd) != 0;
      odd_before = odd;
      const bool whole = work.starts && work.ends;
      // Through LDS, so that rows are stored in whole lines (half a row's share by the lane that has it: 10 times as long): 32 rows at once, in
      // places that this wave brings (the first stages', the others may take the next tile's queries), chunk c of row r in slot c ^ r.
      constexpr int kShare = DC / 4, kChunks = kShare / 4;    // of a row: the wave's channels, in chunks of 4
      static_assert(kPage * kShare * 4 == 8 * Page::kRowBytes, "16 rows are half a page's");
      auto place = [&](int r, int c) {
        return lds.page[DC == 512 ? r >> 4 : 0][page] + (DC == 512 ? part : r >> 4) * 8 * Page::kRowBytes + (r & 15) * kShare * 4 + 16 * (c ^ (r & 15));
      };
      int lane = tid & 63;
      __asm__ volatile("" : "+v"(lane));            // else the addresses are made before the first tile, and kept in scratch memory
      const int l32 = lane & 31, half = lane >> 5;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int r = 32 * t + l32;
        const float l = lds.sum[0][r] + lds.sum[1][r], f = whole ? 1.f / l : 1.f;
        if (x.channel0 == 0 && half == 0) {
          if (!whole) reinterpret_cast<float2*>(args->part_ml)[(size_t)work.slot * M + r] = float2{x.m[t], l};
          else if (args->lse && r < n_rows) args->lse[work.row0 + r] = (x.m[t] + flog2(l)) * kLn2;
        }
#pragma unroll
        for (int d = 0; d < LatValues<DC, DR>::kTiles; ++d)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            *reinterpret_cast<f32x4*>(place(l32, 8 * d + 2 * e + half)) =
                f32x4{x.o[d][t][4 * e], x.o[d][t][4 * e + 1], x.o[d][t][4 * e + 2], x.o[d][t][4 * e + 3]} * f;
        const int c = lane % kChunks, r0 = lane / kChunks, channel = x.channel0 + 4 * c;
        constexpr int kAtOnce = 64 / kChunks;       // rows of an instruction
        if (odd)
#pragma unroll 1
          for (int r = r0; r < 32; r += kAtOnce)
#pragma unroll 1
            for (int k = 0; k < 4; ++k)
              if (lds.notes.odd[channel + k] <= limits[32 * t + r]) *reinterpret_cast<float*>(place(r, c) + 4 * k) = __builtin_nanf("");
        if (!whole) {
          float* const to = args->part_o + ((size_t)work.slot * M + 32 * t + r0) * DC + channel;
#pragma unroll 4
          for (int r = 0; r < 32; r += kAtOnce) *reinterpret_cast<f32x4*>(to + r * DC) = *reinterpret_cast<const f32x4*>(place(r + r0, c));
        } else {
          uint16_t* const to = args->out + (work.row0 + 32 * t + r0) * DC + channel;
#pragma unroll 4
          for (int r = 0; r < 32; r += kAtOnce) {
            const f32x4 y = *reinterpret_cast<const f32x4*>(place(r + r0, c));
            if (32 * t + r + r0 < n_rows) *reinterpret_cast<bf16x4*>(to + r * DC) = bf16x4{(__bf16)y[0], (__bf16)y[1], (__bf16)y[2], (__bf16)y[3]};
          }
        }
      }
    }
    limits = limits == lds.limit2 ? lds.notes.limit : lds.limit2;
  } while (work.next(a));
  if (tid == 0) args_anew()->jobs[work.index] = work.job;
}

hipError_t launch_latent64(const LatentArgs& a, int latent_dim, hipStream_t stream) {
  const dim3 grid(kLatentGrid), threads(64 * kWaves64);
  if (latent_dim == 512) hipLaunchKernelGGL((latent64_kernel<512, 64>), grid, threads, 0, stream, a);
  else hipLaunchKernelGGL((latent64_kernel<256, 32>), grid, threads, 0, stream, a);
  return hipGetLastError();
}

}  // namespace pearl
