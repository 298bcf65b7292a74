// gfx950 decode attention over a cache of MX blocks (mx_format.h): one new token per sequence, each query
// head over the cached keys of its kv-head (paper, section 4.3, Eq. 1: the KV-cache read per
// sequence is what a decode step costs).
//
// The launch is cut as decode_kernel's (decode_shares.h): every wave streams an equal run of the batch's
// pages, whatever the lengths.  A wave takes four pages (64 keys) of a sequence at a time:
//   S^T (keys x heads)   = K . Q^T      16x16x32 MFMA, A = K rows, B = the group's queries
//   O^T (dims x heads)  += V^T . P^T    16x16x32 MFMA, A = V^T, B = the weights
// and holds no tile in LDS: the cache's layout gives each lane its operands in 16-byte loads.
//   * Lane l loads, of K tile t (t = 0..3), the row of page (l % 16) / 4, slot 4 t + l % 4, channels of k group
//     l / 16, and of V the channel pairs 16 p + l % 16 (p = 0 .. D/32 - 1) of page l / 16, all its 16 tokens.
//   * So tile t's S^T holds in lane l, rows 4 (l / 16) + i, the scores of page l / 16, slots 4 t + i: the 16
//     slots of the page whose V that lane holds.  The weights are P.V's B operand as they are.
//   * Elements are turned into bf16 by the conversion instructions, which apply the scale: exact.  K pairs are
//     neighbouring channels under one scale and are operands at once; V pairs are two channels of one
//     token, and one byte permute per two tokens sorts them by channel.
// The products have 16 columns for at most 8 heads.  Columns 0..7 and 8..15 hold the same queries, and the weights
// enter P.V in two bf16 parts, the upper 8 significant bits in one half of the columns and the rest in the
// other; their outputs are added when the pair is done.  Weights to 16 bits cost no product more.
// The running maximum may lag the true one by 8 (log2 units), as in the prefill kernel, so most steps find no maximum.
//
// What bounds it: the loads of four pages are sent before the four pages before them are computed, so
// 8 waves hold about 70 KB (4 bits) in flight per compute unit.

#include "decode_shares.h"
#include "mx_format.h"

#include <algorithm>
#include <atomic>
#include <mutex>

namespace pearl {

namespace {

constexpr int kUnitPages = 4;                       // pages of a step

struct MxCut {                                      // 2176 bytes of K and V a page and kv-head at 4 bits, d = 128
  static constexpr int kMinPages = 32, kPieceCost = 8, kWholePages = 56;
};

// Four pages' codes and scales as a lane holds them.
template <int D, int kBits> struct Unit {
  static constexpr int KW = D * kBits / 128;        // dwords of a K row and lane
  static constexpr int TP = D / 32;                 // groups of 16 channel pairs
  static constexpr int VW = kBits;                  // dwords of a channel pair's 16 tokens
  static constexpr int KS = D == 128 && kBits == 8 ? 2 : 1;   // blocks of a lane's K channels
  uint32_t k[4][KW];
  uint32_t v[TP][VW];
  u32x4 vs[TP];
  uint32_t ks[KS];
};

// The first channel of k-step ks of a lane's k group: 16-byte pieces of a row, in the order they are loaded.
template <int D, int kBits> __device__ __forceinline__ int k_channel(int group, int ks) {
  if constexpr (D == 128 && kBits == 8) return 64 * (ks >> 1) + 16 * group + 8 * (ks & 1);
  else return D / 4 * group + 8 * ks;
}

template <int N> __device__ __forceinline__ void load_words(uint32_t* dst, const uint8_t* src) {
  if constexpr (N == 2) {
    const u32x2 x = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(src));
    dst[0] = x[0];
    dst[1] = x[1];
  } else {
    const u32x4 x = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src));
#pragma unroll
    for (int i = 0; i < 4; ++i) dst[i] = x[i];
  }
}

template <int D, int kBits> struct Lane {           // a lane's offsets in a block
  using MX = MxBlock<D, kBits>;
  using U = Unit<D, kBits>;
  int k, ks, v;
  __device__ __forceinline__ explicit Lane(int lane) {
    const int m = lane & 15, group = lane >> 4;
    k = (m & 3) * MX::kRow + (U::KW >= 4 ? 16 : 8) * group;
    const int blk = D == 128 && kBits == 4 ? group : group >> 1;
    ks = MX::kKScales + ((m & 3) * MX::kBlocks + blk) * 4;
    v = MX::kVCodes + m * 16;
  }
  // kb: the block of this lane's K page, vb: of its V page
  __device__ __forceinline__ void load(U& u, const uint8_t* kb, const uint8_t* vb) const {
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int c = 0; c < (U::KW + 3) / 4; ++c) load_words<U::KW == 2 ? 2 : 4>(&u.k[t][4 * c], kb + k + 4 * t * MX::kRow + 64 * c);
#pragma unroll
    for (int c = 0; c < U::KS; ++c) u.ks[c] = *reinterpret_cast<const uint32_t*>(kb + ks + 8 * c);
#pragma unroll
    for (int p = 0; p < U::TP; ++p) u.vs[p] = *reinterpret_cast<const u32x4*>(vb + MX::kVScales + 16 * p);
#pragma unroll
    for (int p = 0; p < U::TP; ++p)
#pragma unroll
      for (int h = 0; h < U::VW / 4; ++h) load_words<4>(&u.v[p][4 * h], vb + v + (h * (D / 2) + 16 * p) * 16);
  }
};

template <int kBits, int kFirst> __device__ __forceinline__ bf16x8 eight_up(const uint32_t* w, float f) {
  if constexpr (kBits == 4)
    return as_bf16x8(u32x4{mx_up<4, 0>(w[0], f), mx_up<4, 1>(w[0], f), mx_up<4, 2>(w[0], f), mx_up<4, 3>(w[0], f)});
  else
    return as_bf16x8(u32x4{mx_up<8, 0>(w[0], f), mx_up<8, 1>(w[0], f), mx_up<8, 0>(w[1], f), mx_up<8, 1>(w[1], f)});
}

// Channel pairs of token s (0..15) of a lane's unit, as two bf16.
template <int kBits, int s> __device__ __forceinline__ uint32_t v_pair(const uint32_t* w, const u32x4& scales) {
  const float f = mx_scale_of<s % 4>(scales[s / 4]);
  if constexpr (kBits == 4) return mx_up<4, s % 4>(w[s / 4], f);
  else return mx_up<8, s % 2>(w[s / 2], f);
}

// Attends the heads to one unit.  lim: the slots of page l / 16 that this sequence attends to (16 unless kTail).
template <int D, int kBits, bool kTail>
__device__ __forceinline__ void consume(Unit<D, kBits>& u, const bf16x8* qop, f32x4 (*oacc)[2], float& m_run, float& l_run,
                                        float c, int lim, uint32_t part_hi, uint32_t part_lo) {
  using U = Unit<D, kBits>;
  constexpr int KB = D / 32;
  f32x4 s[4];
  auto tile = [&](auto t_c) {
    constexpr int t = decltype(t_c)::value;
    s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      const float f = mx_scale_of<t>(u.ks[U::KS == 2 ? kb / 2 : 0]);
      s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(eight_up<kBits, 0>(&u.k[t][kb * kBits / 4], f), qop[kb], s[t], 0, 0, 0);
    }
  };
  tile(std::integral_constant<int, 0>{});
  tile(std::integral_constant<int, 1>{});
  tile(std::integral_constant<int, 2>{});
  tile(std::integral_constant<int, 3>{});
  if constexpr (kTail) {
    // keys past the end: scores by a select, so stray bits never leak, and V codes and scales to zero
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) s[t][i] = 4 * t + i < lim ? s[t][i] : -INFINITY;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const int left = min(max(lim - 4 * w, 0), 4);                        // tokens 4 w .. that count
      const uint32_t mask = left == 4 ? 0xffffffffu : (1u << (8 * left)) - 1u;
#pragma unroll
      for (int p = 0; p < U::TP; ++p) {
        u.vs[p][w] &= mask;
        if constexpr (kBits == 4) {
          u.v[p][w] &= mask;
        } else {
          u.v[p][2 * w] &= left >= 2 ? 0xffffffffu : left == 1 ? 0xffffu : 0u;
          u.v[p][2 * w + 1] &= left == 4 ? 0xffffffffu : left == 3 ? 0xffffu : 0u;
        }
      }
    }
  }
  float p[16];
  auto weights = [&](float m) {
    float a = 0.f, b = 0.f;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p[4 * t + i] = fexp2(__builtin_fmaf(s[t][i], c, -m));
        if (i & 1) b += p[4 * t + i]; else a += p[4 * t + i];
      }
    return a + b;
  };
  constexpr float kMaxSum = 256.0f;                 // bounds every weight by 2^8
  float sum = weights(m_run);
  if (__ballot(!(sum <= kMaxSum))) {                // the first unit (m = -inf), or scores far above m
    float mx = s[0][0];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) mx = fmaxf(mx, s[t][i]);
    mx = fmaxf(mx, __shfl_xor(mx, 16));
    mx = xor32_max(mx);
    const bool grow = mx * c > m_run;
    const float m_new = grow ? mx * c : m_run;
    const float alpha = grow ? fexp2(m_run - m_new) : 1.0f;
    sum = weights(m_new);
    l_run *= alpha;
#pragma unroll
    for (int q = 0; q < U::TP; ++q) {
      oacc[q][0] *= alpha;
      oacc[q][1] *= alpha;
    }
    m_run = m_new;
  }
  l_run += sum;
  // this column's part of the weights: the upper 16 bits of each, or the rest, which is never 0 unless the
  // weight is, so that an infinite value stays infinite
  bf16x8 pop[2];
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    const uint32_t w = __builtin_bit_cast(uint32_t, p[j]);
    const float y = __builtin_bit_cast(float, w & part_hi) - __builtin_bit_cast(float, w & part_lo);
    pop[j / 8][j % 8] = (__bf16)fmaxf(y, fminf(p[j], 0x1p-100f));
  }
  auto group = [&](auto p_c) {
    constexpr int q = decltype(p_c)::value;
    uint32_t x[16];
    auto token = [&](auto s_c) { x[decltype(s_c)::value] = v_pair<kBits, decltype(s_c)::value>(u.v[q], u.vs[q]); };
    token(std::integral_constant<int, 0>{}); token(std::integral_constant<int, 1>{});
    token(std::integral_constant<int, 2>{}); token(std::integral_constant<int, 3>{});
    token(std::integral_constant<int, 4>{}); token(std::integral_constant<int, 5>{});
    token(std::integral_constant<int, 6>{}); token(std::integral_constant<int, 7>{});
    token(std::integral_constant<int, 8>{}); token(std::integral_constant<int, 9>{});
    token(std::integral_constant<int, 10>{}); token(std::integral_constant<int, 11>{});
    token(std::integral_constant<int, 12>{}); token(std::integral_constant<int, 13>{});
    token(std::integral_constant<int, 14>{}); token(std::integral_constant<int, 15>{});
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      u32x4 even, odd;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        even[j] = __builtin_amdgcn_perm(x[8 * h + 2 * j + 1], x[8 * h + 2 * j], 0x05040100u);
        odd[j] = __builtin_amdgcn_perm(x[8 * h + 2 * j + 1], x[8 * h + 2 * j], 0x07060302u);
      }
      oacc[q][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(even), pop[h], oacc[q][0], 0, 0, 0);
      oacc[q][1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(odd), pop[h], oacc[q][1], 0, 0, 0);
    }
  };
  group(std::integral_constant<int, 0>{});
  group(std::integral_constant<int, 1>{});
  if constexpr (U::TP == 4) {
    group(std::integral_constant<int, 2>{});
    group(std::integral_constant<int, 3>{});
  }
}

}  // namespace

template <int D, int kBits>
__global__ __launch_bounds__(kThreads, 2) void decode_mx_kernel(AttnArgs a, DecPlanArgs d) {
  using MX = MxBlock<D, kBits>;
  using U = Unit<D, kBits>;
  constexpr int KB = D / 32, TP = U::TP;
  __shared__ __attribute__((aligned(16))) ShareEnd<D> stage[kWaves];
  __shared__ DecPlanLds P;
  __shared__ FinishLds F;
  const int lane = threadIdx.x & 63, w = uni(threadIdx.x >> 6);
  const int group = lane >> 4, col = lane & 15, hh = col & 7;
  const int G = a.group, H = a.num_kv_heads, H_q = a.num_q_heads, B = d.batch;

  int most;
  const int total_pages = uni(decode_plan(a, d, P, most));
  if (total_pages < 0) {                            // the prologue cleared the error flag
    if (blockIdx.x == 0 && threadIdx.x == 0) a.ws_hdr[kHdrError] = 1;
    return;
  }
  DecShares<MxCut> sh(P, total_pages, most, d);
  DecRun r;
  if (!decode_run(a, d, P, most, total_pages, sh, r)) return;
  const int g = r.g0 + r.j_w;
  const bool head_ok = col < G && r.j_w >= r.dup;
  const int pages_seen = r.j_w < r.dup ? 1 : a.num_pages;
  const uint32_t part_hi = col < 8 ? 0xffff0000u : 0xffffffffu, part_lo = col < 8 ? 0u : 0xffff0000u;

  f32x4 oacc[TP][2];
  float m_run = -INFINITY, l_run = 0.f;
  int first_b = -1;                                 // the pair whose end this share holds without its start
  bool whole = false;                               // the current pair started inside this share
  PageCursor cur{-1, 0, 1, 1};
  ShareEnd<D>& E = stage[w];

  // The two parts' outputs added, every lane group's sums: the state of a pair that ends or is cut here.
  auto close = [&]() {
#pragma unroll
    for (int p = 0; p < TP; ++p)
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float x = oacc[p][e][i];            // (a bit cast of the element itself takes element 0)
          const int y = __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x128, 0xf, 0xf, false);   // row_ror:8
          oacc[p][e][i] = x + __builtin_bit_cast(float, y);
        }
    l_run += __shfl_xor(l_run, 16);
    l_run += __shfl_xor(l_run, 32);
  };
  auto leave = [&](int which) {                     // lane: head col, dims 32 p + 8 group ..
    if (!head_ok) return;
#pragma unroll
    for (int p = 0; p < TP; ++p) {
      float* o = &E.o[which][col][32 * p + 8 * group];
      *reinterpret_cast<f32x4*>(o) = f32x4{oacc[p][0][0], oacc[p][1][0], oacc[p][0][1], oacc[p][1][1]};
      *reinterpret_cast<f32x4*>(o + 4) = f32x4{oacc[p][0][2], oacc[p][1][2], oacc[p][0][3], oacc[p][1][3]};
    }
    if (group == 0) { E.ml[which][col][0] = m_run; E.ml[which][col][1] = l_run; }
  };

  if (r.n > 0) {
    const ConstI32Ptr bt = (ConstI32Ptr)a.block_table;
    const Lane<D, kBits> at(lane);
    const size_t page_bytes = (size_t)H * MX::kBytes;
    const uint8_t* const heads = a.cache + (size_t)g * MX::kBytes;
    struct Ids { int x[kUnitPages]; };
    // a unit: up to four pages of the cursor's sequence; `left` pages of the share from its first page on
    auto pages_of = [&](const PageCursor& c, int left) { return min(min(kUnitPages, c.np - c.p), left); };
    auto ids_of = [&](const PageCursor& c, int np) {
      Ids id;
#pragma unroll
      for (int i = 0; i < kUnitPages; ++i)
        id.x[i] = clamp_page(bt[(size_t)c.b * a.bt_stride + c.p + min(i, np - 1)], pages_seen);
      return id;
    };
    auto send = [&](U& u, const Ids& id) {
      const int pk = col >> 2;
      const int ik = pk < 2 ? (pk == 0 ? id.x[0] : id.x[1]) : (pk == 2 ? id.x[2] : id.x[3]);
      const int iv = group < 2 ? (group == 0 ? id.x[0] : id.x[1]) : (group == 2 ? id.x[2] : id.x[3]);
      at.load(u, heads + (size_t)ik * page_bytes, heads + (size_t)iv * page_bytes);
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
    U ua, ub;
    u32x4 q_next[KB];
    bf16x8 qop[KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) qop[kb] = zero_bf16x8();
    cur = locate(P, r.t0, B);
    int left = r.n, np_cur = pages_of(cur, left);
    Ids id = ids_of(cur, np_cur);
    send_q(q_next, cur);
    send(ua, id);
    bool fresh = true;                              // the unit is the first of its pair in this share
    PageCursor nxt = cur;
    step_past(nxt, np_cur);
    int np_nxt = pages_of(nxt, left - np_cur);
    if (left > np_cur) id = ids_of(nxt, np_nxt);
    // one unit: the next one's loads go out, then it is attended
    auto unit = [&](U& now, U& next) {
      if (fresh) {
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
          qop[kb] = hh < G ? as_bf16x8(q_next[kb]) : zero_bf16x8();
        }
#pragma unroll
        for (int p = 0; p < TP; ++p) oacc[p][0] = oacc[p][1] = f32x4{0.f, 0.f, 0.f, 0.f};
        m_run = -INFINITY;
        l_run = 0.f;
        whole = cur.p == 0;
      }
      const bool more = left > np_cur;
      PageCursor nn = nxt;
      int np_nn = 0;
      if (more) {
        if (nxt.p == 0) send_q(q_next, nxt);
        send(next, id);
        step_past(nn, np_nxt);
        np_nn = pages_of(nn, left - np_cur - np_nxt);
        if (left > np_cur + np_nxt) id = ids_of(nn, np_nn);
      }
      if (np_cur == kUnitPages && (cur.p + kUnitPages) * kPage <= cur.kv) {
        consume<D, kBits, false>(now, qop, oacc, m_run, l_run, a.scale_log2, kPage, part_hi, part_lo);
      } else {
        const int lim = group < np_cur ? cur.kv - (cur.p + group) * kPage : 0;
        consume<D, kBits, true>(now, qop, oacc, m_run, l_run, a.scale_log2, lim, part_hi, part_lo);
      }
      const bool ends_here = cur.p + np_cur == cur.np;
      if (ends_here) {
        close();
        if (whole) {
          if (head_ok) {
            const size_t row = (size_t)cur.b * H_q + g * G + col;
            const float inv = 1.0f / l_run;
#pragma unroll
            for (int p = 0; p < TP; ++p) {
              u32x4 x;
#pragma unroll
              for (int i = 0; i < 4; ++i)
                x[i] = (uint32_t)bf16_bits(oacc[p][0][i] * inv) | ((uint32_t)bf16_bits(oacc[p][1][i] * inv) << 16);
              *reinterpret_cast<u32x4*>(a.out + row * D + 32 * p + 8 * group) = x;
            }
            if (group == 0 && a.lse) a.lse[row] = (m_run + flog2(l_run)) * kLn2;
          }
        } else {                                    // only the first pair can have started earlier
          leave(0);
          first_b = cur.b;
        }
      }
      fresh = ends_here;
      left -= np_cur;
      if (!more) {
        if (ends_here) cur.b = -1;                  // the share ends with the pair's end
        return;
      }
      cur = nxt;
      np_cur = np_nxt;
      nxt = nn;
      np_nxt = np_nn;
    };
    for (;;) {
      unit(ua, ub);
      if (left == 0) break;
      unit(ub, ua);
      if (left == 0) break;
    }
    if (cur.b >= 0) {
      close();
      leave(1);
    }
  }
  finish_shares<D>(a, d, P, sh, r, reinterpret_cast<const char*>(stage), (int)sizeof(ShareEnd<D>),
                   SharePairs{first_b, cur.b, !whole, r.n > 0}, F);
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
