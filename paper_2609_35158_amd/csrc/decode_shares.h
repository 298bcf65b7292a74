// Decode of batches of up to kDecPlanMaxSeqs sequences in one launch of equal shares: the plan that
// every workgroup makes by itself, the cut of the page list and the merges, for decode_kernel
// (attn_kernels.hip) and decode_mx_kernel (decode_mx.hip).
#pragma once

#include "attn_device.h"

namespace pearl {

constexpr int kDecPlanChunks = kDecPlanMaxSeqs / kThreads;
static_assert(kDecPlanChunks * kThreads == kDecPlanMaxSeqs, "plan chunks");

struct DecPlanLds {
  int pre[kDecPlanMaxSeqs + 1];            // exclusive prefix sums of pages
  unsigned char tail[kDecPlanMaxSeqs];     // (attended keys - 1) % kPage
  int wsum[kWaves];
  int err;
  int over;                                // a sequence is longer than all_within's limit
};

// Pages and attended keys of one sequence from its length; false if it violates the host bounds.
__device__ __forceinline__ bool dec_seq(const AttnArgs& a, const DecPlanArgs& d, int b, int& pages, int& tail) {
  const int ctx = d.ctx_lens[b];
  const long long kv = (long long)ctx + 1;
  if (ctx < 0 || kv > d.max_kv_len || (kv + kPage - 1) / kPage > a.bt_stride) return false;
  pages = (int)((kv + kPage - 1) / kPage);
  tail = ctx % kPage;
  return true;
}

// Builds the prefix sums; returns the total pages, or -1 if a length violates the host bounds.
// most: the most pages of this thread's sequences (of this lane's: every wave holds them all).
// Batches of at most 64 sequences: every wave builds the same list (the same values to the same
// words), a lane per sequence, so no barrier is needed; a wave reads other lanes' words only after
// the fence that orders its own stores before them.
__device__ __forceinline__ int decode_plan(const AttnArgs& a, const DecPlanArgs& d, DecPlanLds& P, int& most) {
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, B = d.batch;
  // inclusive sums over the wave: inside rows of 16 lanes, then the rows' last lanes onto the rows after
  auto wave_scan = [&](int v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);     // row_shr:1, 2, 4, 8
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);     // row_bcast:15 to rows 1 and 3
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);     // row_bcast:31 to rows 2 and 3
    return v;
  };
  if (B <= 64) {
    int pages = 0, tail = 0;
    const bool bad = lane < B && !dec_seq(a, d, lane, pages, tail);
    const int incl = wave_scan(pages);
    if (lane < B) {
      P.pre[lane + 1] = incl;
      P.tail[lane] = (unsigned char)tail;
    }
    if (lane == 0) P.pre[0] = 0;
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    const int total = __builtin_amdgcn_readlane(incl, 63);
    most = pages;
    return __any(bad) ? -1 : total;
  }
  if (tid == 0) { P.err = 0; P.pre[0] = 0; P.over = 0; }
  __syncthreads();
  int carry = 0;
  most = 0;
#pragma unroll
  for (int c = 0; c < kDecPlanChunks; ++c) {
    if (c * kThreads >= B) break;                   // uniform
    const int b = c * kThreads + tid;
    int pages = 0, tail = 0;
    const bool bad = b < B && !dec_seq(a, d, b, pages, tail);
    most = max(most, pages);
    const int incl = wave_scan(pages);
    if (lane == 63) P.wsum[wv] = incl;
    if (__any(bad) && lane == 0) P.err = 1;
    __syncthreads();
    int before = carry, sum = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      if (w < wv) before += P.wsum[w];
      sum += P.wsum[w];
    }
    if (b < B) {
      P.pre[b + 1] = before + incl;
      P.tail[b] = (unsigned char)tail;
    }
    carry += sum;
    __syncthreads();
  }
  return P.err ? -1 : carry;
}

// A place in the page list: page p (of np) of sequence b, which attends to kv keys.  All members
// are uniform across the wave.
struct PageCursor {
  int b, p, np, kv;
};

// The last sequence b with pre[b] + kCost * b <= t, found by counting prefix sums with ballots (64 evenly spaced
// probes, then the gap between two).
template <int kCost> __device__ __forceinline__ int seq_at(const DecPlanLds& P, int t, int B) {
  const int lane = threadIdx.x & 63;
  const int gap = (B + 63) / 64;
  const int blk = __popcll(__ballot(lane * gap < B && P.pre[min(lane * gap, B)] + kCost * lane * gap <= t)) - 1;
  int b = blk * gap;
  if (gap > 1) {
    const int i1 = b + 1 + lane;
    b += __popcll(__ballot(lane < gap - 1 && i1 < B && P.pre[min(i1, B)] + kCost * i1 <= t));
  }
  return uni(b);
}

// The place of entry t (< pre[B]) of the list.
__device__ __forceinline__ PageCursor locate(const DecPlanLds& P, int t, int B) {
  const int b = seq_at<0>(P, t, B);
  const int first = uni(P.pre[b]);
  const int np = uni(P.pre[b + 1]) - first;
  return PageCursor{b, t - first, np, (np - 1) * kPage + uni(P.tail[b]) + 1};
}

// The next entry (never called on the list's last one).
__device__ __forceinline__ void advance(const DecPlanLds& P, PageCursor& c) {
  if (++c.p < c.np) return;
  c.p = 0;
  ++c.b;
  c.np = uni(P.pre[c.b + 1]) - uni(P.pre[c.b]);
  c.kv = (c.np - 1) * kPage + uni(P.tail[c.b]) + 1;
}

// Whether no sequence holds more than `limit` pages, `most` being decode_plan's: called once, by all
// threads.
__device__ __forceinline__ bool all_within(DecPlanLds& P, int B, int most, int limit) {
  const bool over = __any(most > limit);
  if (B <= 64) return !over;
  if (over && (threadIdx.x & 63) == 0) P.over = 1;
  __syncthreads();
  return P.over == 0;
}

// How a kernel's list of pages is cut: runs of at least kMinPages pages, or, where a wave takes units of
// kUnit > 1 pages, of as many pages as some number of units for each of its waves; several kv-heads share a
// workgroup if kPieceCost times the pieces of the longest sequence are at most the pages of a wave's
// share (DecShares); runs hold whole sequences if that makes none longer than an equal run by more than
// kWholePages (DecRun); where a workgroup holds 8 kv-heads, so that shares are runs and equal ones all there is, a
// sequence's start counts as kSeqCost pages.
struct PoolCut {                                    // bf16 pools: 8 KiB of K and V a page and kv-head (d = 128)
  static constexpr int kMinPages = 16, kPieceCost = 8, kWholePages = 28, kSeqCost = 0, kUnit = 1;
};

// What a workgroup of a decode launch takes: run x of the kv-heads [g0, g0 + heads), and its wave's share.
struct DecRun {
  int x, g0, dup;                                   // the first dup kv-heads are another workgroup's too
  int sub, j_w;                                     // the wave's share of the run and its kv-head, of the workgroup's
  int run0, t0, n;                                  // the run's first page, of all pages; the wave's first one and pages
  bool per_pair;
  int slot_stride;
};

// A pair cut by the workgroup's boundaries: its sequence (< 0: none), first run, runs, first slot.
struct CutPair {
  int b, x0, n, slot0;
};

// The cut of the page list.  A workgroup takes `heads` kv-heads (a power of two up to 8 that
// divides H) and one of n_runs runs of 8 / heads consecutive shares; the first `more` shares hold
// len + 1 entries, the others len, of the list in which `cost` entries stand before each sequence's
// pages.  Several heads per workgroup read the adjacent blocks of a page
// together, which HBM serves faster (2% of a share's time at 8 heads, 9% at 64).  But then every
// share's end cuts a pair between workgroups, and the last merges take longer the more pieces a pair
// is cut into.  So workgroups take several heads if the longest pair's pieces, longest / len, are few
// for the share's length: Cut::kPieceCost * longest / len <= len.  Measured (us a call with one head
// and with several; G = 4, G = 1 above 16 kv-heads; pages per share, pieces of the longest pair):
//   several are faster: 64 sequences of 2K-16K tokens, 8 kv-heads (144, 7) 363 and 355; 32 of 400-1600,
//     64 kv-heads (62, 1.6) 178 and 163; the same at 40 (39, 2.6) 110 and 107; 64 of 100-400, 64 kv-heads
//     (31, 1) 95.8 and 89.1; 256 of 1K-8K, 2 kv-heads (70, 7) 191 and 186;
//   one is faster: 48 of 2K-6K, 8 kv-heads (47, 8) 124 and 130; 32 of them (31, 12) 87 and 100; 16 of
//     2K-30K (64, 29) 171 and 188; 8 of 4K-16K, 16 kv-heads (39, 25) 116 and 135; 32 of 500-2000, 16
//     kv-heads (19, 6) 59 and 66; 200 of 500-2000, 4 kv-heads (30, 4) 89.5 and 90.1.
template <class Cut> struct DecShares {
  int cost;                                         // entries before a sequence's pages
  int heads, n_runs, len, more;
  __device__ __forceinline__ DecShares(DecPlanLds& P, int pages, int most, const DecPlanArgs& d) {
    // which form and how many runs: any wave and workgroup finds the same, exact quotients are not needed
    const int len_heads = min((int)((float)pages * d.inv_shares_heads), 1 << 15);
    const int longest = len_heads * len_heads / Cut::kPieceCost;            // at most, for several heads
    if (d.heads > 1 && (long long)longest * d.batch >= pages && all_within(P, d.batch, most, longest)) {
      heads = d.heads;
      n_runs = d.runs_heads;
    } else {
      heads = 1;
      if constexpr (Cut::kUnit > 1) {
        // Every wave takes at most so many units: one, and more where the longest sequence's merge would cost more than the
        // units it saves (a run more in it costs about as much as a third of a page in every wave).  The shares are cut
        // evenly, so they need not be whole units: 2731 tokens in 4 bits are 48 shares of 3 or 4 pages.  us a call with runs
        // of 32 pages and 1/64 of a sequence, as of bf16 pools, and so: one sequence at 8 kv-heads, 4 bits, 1500 tokens 14.6 and
        // 11.3, 2731 13.7 and 11.9, 10000 17.0 and 14.7, 30000 19.7 and 19.7; 8 bits 1500 16.8 and 12.1, 12000 16.5 and 17.2;
        // three of 5-20K at one kv-head 21.4 and 20.5.  With half a page for a third: 8 bits, 16000 17.9 for 17.3; with a
        // fifth: 4 bits, 16000 17.5 for 16.5.  (Beyond 64 sequences, where a wave does not hold all lengths, runs of one unit
        // a wave are only as many as fill the grid.)
        constexpr int kRun = kWaves * Cut::kUnit, kLong = 3 * Cut::kUnit * kRun;
        int units = 1;
        if (d.batch <= 64) while (__any(most > units * (units + 1) * kLong)) ++units;
        n_runs = max(1, min(d.runs_one, (int)((unsigned)(pages + units * kRun - 1) / (unsigned)(units * kRun))));
      } else {
        // Long sequences in few pairs take somewhat longer runs, so that a pair is not merged from 100
        // pieces: three of 5-20K tokens on one kv-head 22.0 us a call with kMinPages alone, 19.4 so.
        const int least = Cut::kMinPages + (int)((float)pages * d.inv_64_seqs);
        n_runs = max(1, min(d.runs_one, (int)((float)pages * __builtin_amdgcn_rcpf((float)least))));
      }
    }
    cost = Cut::kSeqCost > 0 && heads == kWaves ? Cut::kSeqCost : 0;
    const int n = n_runs * subs(), entries = pages + cost * d.batch;
    len = (int)((unsigned)entries / (unsigned)n);
    more = entries - len * n;
  }
  __device__ __forceinline__ int subs() const { return kWaves / heads; }   // shares per run
  __device__ __forceinline__ int begin(int share) const { return share * len + min(share, more); }
  __device__ __forceinline__ int first_page(const DecPlanLds& P, int t, int B) const {   // of all pages, from entry t on
    if (cost == 0) return t;
    const int b = seq_at<Cut::kSeqCost>(P, t, B), pre = uni(P.pre[b]);
    return uni(pre + max(t - (pre + cost * b) - cost, 0));
  }
  __device__ __forceinline__ int run_of(int t) const {                     // the run that holds entry t
    const int big = more * (len + 1);
    const int share = t < big ? (unsigned)t / (unsigned)(len + 1) : more + (unsigned)(t - big) / (unsigned)max(len, 1);
    return (unsigned)share / (unsigned)subs();
  }
  // The runs of sequence b's pages, cut between workgroups, and where its partials are: a run's first slot, or for a
  // start behind another sequence's pages the second one.
  __device__ __forceinline__ CutPair cut_of(const DecPlanLds& P, const DecRun& r, int b) const {
    const int at = uni(P.pre[b]) + cost * b, x0 = run_of(at + cost), x1 = run_of(uni(P.pre[b + 1]) + cost * b + cost - 1);
    const bool at_start = at <= begin(x0 * subs());
    return CutPair{b, x0, x1 - x0 + 1, at_start ? r.slot_stride * x0 : (r.per_pair ? n_runs + b : 2 * x0 + 1)};
  }
};

// A wave's partials at the end of its share, in the space of its own page stages: [0] the first
// pair's, [1] the last one's.
template <int D> struct ShareEnd {
  float o[2][8][D];
  float ml[2][8][2];
};
// What they are of: the sequences of the first pair (< 0: none) and the last one, whether the last
// one started before the share, and whether the share holds pages at all.
struct SharePairs {
  int first_b, last_b, before, used;
};

// Two adjacent floats as one device-scope access: stores are written through to the level where
// every XCD reads them, loads do not hit stale cache lines.
__device__ __forceinline__ void st_dev2(float* p, float x, float y) {
  const unsigned long long v = (unsigned long long)__builtin_bit_cast(unsigned, x) |
                               ((unsigned long long)__builtin_bit_cast(unsigned, y) << 32);
  __hip_atomic_store(reinterpret_cast<unsigned long long*>(p), v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// Four floats at a 16-byte aligned place, likewise; to be waited for by vmcnt, like any store.  (The nop: a store of over
// 8 bytes still reads its data in the cycle after, which the compiler cannot know of an asm statement.)
__device__ __forceinline__ void st_dev4(float* p, f32x4 x) {
  __asm__ volatile("global_store_dwordx4 %0, %1, off sc1\n\ts_nop 1" : : "v"(p), "v"(x) : "memory");
}
__device__ __forceinline__ void ld_dev2(const float* p, float& x, float& y) {
  const unsigned long long v = __hip_atomic_load(reinterpret_cast<const unsigned long long*>(p), __ATOMIC_RELAXED,
                                                 __HIP_MEMORY_SCOPE_AGENT);
  x = __builtin_bit_cast(float, (unsigned)v);
  y = __builtin_bit_cast(float, (unsigned)(v >> 32));
}

// Merge of a cut pair (kv-head g) from its partials, in the workgroup that counted itself in last:
//   o = sum_s 2^(m_s - m*) o~_s / sum_s 2^(m_s - m*) l_s,   lse = (m* + log2 l*) ln 2
// (of partials whose scores are all minus infinity m_s is too: weight 0).
// A lane takes D/16 dims of a q-head and the (m, l) of that head (4 heads a pass), up to kMergeBlock
// partials in flight at a time and no load beyond the pair's own (one sequence of 2732 keys, 10
// partials a pair: 13.8 us a call with blocks of 8, 13.15 with 12, 13.2 with 16; with the last
// partial loaded again to fill every block, 512 sequences of 2-3 partials took 195-200 us, now 190).
constexpr int kMergeBlock = 12;

template <int D>
__device__ __forceinline__ void merge_pair(const AttnArgs& a, const CutPair& c, int g, int stride, int max_dec, int pass) {
  constexpr int U = kMergeBlock, PER = D / 16;
  const int G = a.group, H_q = a.num_q_heads;
  const int ns = uni(c.n);
  const int lane = threadIdx.x & 63, head = 4 * pass + lane / 16, dim = lane % 16 * PER;
  if (head >= G) return;
  float M = -INFINITY, L = 0.f, acc[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) acc[i] = 0.f;
#pragma unroll 1
  for (int s0 = 0; s0 < ns; s0 += U) {
    float v[U][PER], m[U], l[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      m[u] = -INFINITY;
      if (s0 + u < ns) {                            // uniform
        const int s = s0 + u;
        const size_t slot = ((size_t)g * max_dec + (s == 0 ? c.slot0 : stride * (c.x0 + s))) * G + head;
        ld_dev2(&a.part_ml[2 * slot], m[u], l[u]);
#pragma unroll
        for (int i = 0; i < PER; i += 2) ld_dev2(&a.part_o[slot * D + dim + i], v[u][i], v[u][i + 1]);
      }
    }
    float M_new = M;
#pragma unroll
    for (int u = 0; u < U; ++u) M_new = fmaxf(M_new, m[u]);
    const float base = M_new == -INFINITY ? 0.f : M_new, alpha = fexp2(M - base);
    L *= alpha;
#pragma unroll
    for (int i = 0; i < PER; ++i) acc[i] *= alpha;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (s0 + u < ns) {                            // uniform
        const float f = fexp2(m[u] - base);
        L += f * l[u];
#pragma unroll
        for (int i = 0; i < PER; ++i) acc[i] += f * v[u][i];
      }
    }
    M = M_new;
  }
  const float inv = 1.0f / L;
  const size_t row = (size_t)c.b * H_q + g * G + head;
#pragma unroll
  for (int i = 0; i < PER; i += 4) {
    u32x2 pk;
    pk[0] = (uint32_t)bf16_bits(acc[i] * inv) | ((uint32_t)bf16_bits(acc[i + 1] * inv) << 16);
    pk[1] = (uint32_t)bf16_bits(acc[i + 2] * inv) | ((uint32_t)bf16_bits(acc[i + 3] * inv) << 16);
    *reinterpret_cast<u32x2*>(a.out + row * D + dim + i) = pk;
  }
  if (dim == 0 && a.lse) a.lse[row] = (M + flog2(L)) * kLn2;
}

// Finds a workgroup's run; false if it has none.
// Runs of whole sequences, as many sequences each (one, if the grid holds a workgroup for every
// (sequence, kv-head) pair), instead of equal runs, where no run gets much longer by it: then no pair
// is cut between workgroups, and the acknowledged stores, the count-in and the merge, which take
// about as long as 3 more pages a wave, fall away.  us a call with equal runs and so, 32 q-heads:
// 4 sequences of 200-400 tokens at 2 kv-heads 14.1 and 11.8; 24 of 500-1000 at 8 21.1 and 19.2; but
// one of 770 at 4, 30 pages over its run, 11.6 and 13.0; two sequences a run, 64 of 16-64 at 8 16.0 and
// 11.1.  The line at 28 pages more than an equal run, against 12 and 60: 32 of 200-700 at 8 16.4 / 18.6 /
// 16.4, 128 of 100-400 at 8 30.1 / 32.1 / 30.2, 300 of 100-500 at 2 25.2 / 25.2 / 26.2, 24 of 500-1200
// at 8 22.0 / 22.1 / 21.1.  It needs no partial slots: with short sequences the workspace holds one
// per sequence, which allows equal runs for half of them only.
template <class Cut>
__device__ __forceinline__ bool decode_run(const AttnArgs& a, const DecPlanArgs& d, const DecPlanLds& P, int most,
                                           int total_pages, DecShares<Cut>& sh, DecRun& r) {
  const int lane = threadIdx.x & 63, w = uni(threadIdx.x >> 6);
  const int H = a.num_kv_heads, B = d.batch;
  auto whole_begin = [&](int run) { return run * d.whole_seqs + min(run, d.whole_more); };
  // (up to 64 sequences every wave holds all lengths, and one that is too much by itself is seen there)
  bool whole_runs = sh.heads == 1 && !(B <= 64 && __any((most - Cut::kWholePages) * sh.n_runs > total_pages));
  if (whole_runs && (B > 64 || d.runs_whole < B)) {
    bool over = false;
#pragma unroll 1
    for (int i = lane; i < d.runs_whole; i += 64) {
      const int pages = P.pre[whole_begin(i + 1)] - P.pre[whole_begin(i)];
      over |= (long long)(pages - Cut::kWholePages) * sh.n_runs > total_pages;
    }
    whole_runs = !__any(over);
  }
  if (whole_runs) sh.n_runs = d.runs_whole;
  const int n_blk = (H + sh.heads - 1) / sh.heads;  // head blocks
  if ((int)blockIdx.x >= sh.n_runs * n_blk) return false;
  // Run x of a head block is workgroup x n_blk + (block - x) mod n_blk: the blocks of a run start
  // together, and every XCD (workgroup mod 8) sees all of them.
  r.x = blockIdx.x / n_blk;
  // The last block overlaps the one before if the kv-heads don't divide: the waves of its first `dup`
  // kv-heads go along, so that all keep pace, but read one page again and again and leave no results.
  const int blk0 = (blockIdx.x + r.x) % n_blk * sh.heads;
  r.g0 = min(blk0, H - sh.heads);
  r.dup = blk0 - r.g0;
  r.sub = w / sh.heads;
  r.j_w = w % sh.heads;
  int run0, t0, end;
  if (whole_runs) {
    run0 = uni(P.pre[whole_begin(r.x)]);
    const int len = uni(P.pre[whole_begin(r.x + 1)]) - run0, q = len / kWaves, rest = len % kWaves;
    t0 = run0 + w * q + min(w, rest);
    end = t0 + q + (w < rest);
  } else {
    const int share = r.x * sh.subs() + r.sub;
    t0 = sh.first_page(P, sh.begin(share), B);
    end = sh.first_page(P, sh.begin(share + 1), B);
    run0 = sh.first_page(P, sh.begin(r.x * sh.subs()), B);
  }
  r.run0 = run0;
  r.t0 = t0;
  r.n = end - t0;
  // partial slots and counters of a kv-head: two slots and a counter per run, or a slot per run,
  // and a slot and a counter per sequence, if that is fewer
  r.per_pair = B < sh.n_runs;
  r.slot_stride = r.per_pair ? 1 : 2;
  return true;
}

// Shared memory of finish_shares.
struct FinishLds {
  SharePairs ends[kWaves];                          // per share of the run
  CutPair cut[2];                                   // of the first and the second slot
  int last[2][kWaves];
};

// Merges the waves' partials per pair and stores what they give, after every wave has left its own, and
// what they are of, at its place in `stage` (stage_bytes each).
template <int D, class Cut>
__device__ __forceinline__ void finish_shares(const AttnArgs& a, const DecPlanArgs& d, const DecPlanLds& P,
                                              const DecShares<Cut>& sh, const DecRun& r, const char* stage,
                                              int stage_bytes, const SharePairs& mine, FinishLds& F) {
  const int lane = threadIdx.x & 63, w = uni(threadIdx.x >> 6);
  const int G = a.group;
  if (lane == 0) F.ends[r.sub] = mine;              // alike for all heads
  if (threadIdx.x < 2) F.cut[threadIdx.x].b = -1;
  // a barrier without the release fence of __syncthreads: output stores stay in flight
  __builtin_amdgcn_s_waitcnt(PEARL_LGKMCNT0);
  __asm__ volatile("s_barrier" ::: "memory");
  // A pair's partials form a chain: it starts in the share the pair starts in (or in the run's first
  // share), goes on through the last-pair partials of the following shares while the pair goes
  // on, and closes with the first-pair partial of the share the pair ends in.  Bit q of the masks
  // below is share q's.
  {
    const int subs = sh.subs();
    const SharePairs e = F.ends[lane & (kWaves - 1)];
    const unsigned used = (unsigned)__ballot(lane < subs && e.used);
    const unsigned has_first = (unsigned)__ballot(lane < subs && e.first_b >= 0);
    // bits 0..7: chains that start with share q's last pair; bit 8: the first share's first pair
    unsigned todo = (unsigned)__ballot(lane < subs && e.last_b >= 0 && (!e.before || lane == 0)) |
                    ((has_first & 1u) << kWaves);
    const int rows = sh.heads * G;                  // q-heads of the workgroup
    while (todo) {
      const int q0 = __builtin_ctz(todo);
      todo &= todo - 1;
      const bool is_first = q0 == kWaves;
      const int qb = is_first ? 0 : q0;
      const unsigned after = is_first ? 0u : ~0u << (q0 + 1);
      const unsigned close = has_first & after;     // its lowest bit: the share that closes the chain
      const unsigned mid = is_first ? 0u : (used & after & ((close & -close) - 1u)) | (1u << q0);
      const int q_close = is_first ? 0 : (close ? __builtin_ctz(close) : -1);
      const int b = __builtin_amdgcn_readlane(is_first ? e.first_b : e.last_b, qb);
      const bool before = is_first || __builtin_amdgcn_readlane(e.before, qb);
      const bool cut = before || q_close < 0;       // other workgroups hold parts of it
      const int pu = uni(P.pre[b]);                 // the pair's first entry
      const int second = pu > r.run0;
      const int slot2 = r.per_pair ? sh.n_runs + b : 2 * r.x + 1;   // the run's second slot
      for (int t = threadIdx.x + r.dup * G * (D / 2); t < rows * (D / 2); t += kThreads) {
        const int row_w = t / (D / 2), dim = 2 * (t - row_w * (D / 2));
        const int j = row_w / G, head = row_w - j * G;      // kv-head of the workgroup, q-head of the group
        float M = -INFINITY, L = 0.f, o0 = 0.f, o1 = 0.f;
        auto add = [&](int q, int which) {
          const ShareEnd<D>& E = *reinterpret_cast<const ShareEnd<D>*>(stage + (q * sh.heads + j) * stage_bytes);
          const float m = E.ml[which][head][0], l = E.ml[which][head][1];
          const float M_new = fmaxf(M, m);
          const float base = M_new == -INFINITY ? 0.f : M_new, fa = fexp2(M - base), fb = fexp2(m - base);
          L = fa * L + fb * l;
          o0 = fa * o0 + fb * E.o[which][head][dim];
          o1 = fa * o1 + fb * E.o[which][head][dim + 1];
          M = M_new;
        };
        for (unsigned rest = mid; rest; rest &= rest - 1) add(__builtin_ctz(rest), 1);
        if (q_close >= 0) add(q_close, 0);
        if (!cut) {
          const size_t row = (size_t)b * a.num_q_heads + r.g0 * G + row_w;
          const float inv = 1.0f / L;
          *reinterpret_cast<uint32_t*>(a.out + row * D + dim) =
              (uint32_t)bf16_bits(o0 * inv) | ((uint32_t)bf16_bits(o1 * inv) << 16);
          if (dim == 0 && a.lse) a.lse[row] = (M + flog2(L)) * kLn2;
        } else {
          const size_t slot = ((size_t)(r.g0 + j) * d.max_dec + (second ? slot2 : r.slot_stride * r.x)) * G + head;
          st_dev2(&a.part_o[slot * D + dim], o0, o1);
          if (dim == 0) st_dev2(&a.part_ml[2 * slot], M, L);
        }
      }
      if (cut && threadIdx.x == 0) {
        F.cut[second] = sh.cut_of(P, r, b);
      }
    }
  }
  // Count the run in on its cut pairs once its stores are acknowledged; the last one merges.  The
  // counter of a pair is its sequence's, or (of as many counters as runs) that of the run it starts
  // in: at most one pair goes on past a run's end.
  __builtin_amdgcn_s_waitcnt(PEARL_VMCNT(0));
  __syncthreads();
  const int task = threadIdx.x;                     // (slot kind, kv-head of the workgroup)
  if (task < 2 * sh.heads) {
    const int j = task >> 1;
    const CutPair c = F.cut[task & 1];
    int last = 0;
    if (c.b >= 0 && j >= r.dup) {
      const int ctr = r.per_pair ? (r.g0 + j) * d.batch + c.b : (r.g0 + j) * sh.n_runs + c.x0;
      last = __hip_atomic_fetch_add(&a.split_cnt[ctr], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == c.n - 1;
    }
    F.last[task & 1][j] = last;
  }
  __syncthreads();
  const int passes = (G + 3) / 4;
#pragma unroll 1
  for (int t = w; t < 2 * sh.heads * passes; t += kWaves) {
    const int pair = t / passes;
    if (F.last[pair & 1][pair >> 1])
      merge_pair<D>(a, F.cut[pair & 1], r.g0 + (pair >> 1), r.slot_stride, d.max_dec, t - pair * passes);
  }
}

}  // namespace pearl
