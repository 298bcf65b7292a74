// The cache in MX blocks: 32 neighbouring channels of one token and kv-head share a scale 2^(s - 127)
// (one byte s; 255: every element is NaN), elements are E2M1 (4 bits) or E4M3 (8 bits).
//
// One block of the cache holds the 16 tokens of a (page, kv-head), nb = D / 32 scales a token:
//   K codes   16 rows of D * bits / 8 bytes: a token's channels in order (4 bits: even channel low);
//   V codes   units of 16 bytes, one pair of neighbouring channels for TPU tokens (16 at 4 bits, 8 at
//             8): the pair's two codes of a token side by side, units ordered (token group, pair);
//   K scales  [slot % 4][32-channel block][slot / 4];
//   V scales  [32-channel block][slot].
// The layout is the attention kernels': a lane's K operand is 16 bytes of a token row, its V operand
// 16 bytes of a channel pair, i.e. V comes transposed without passing through LDS, and the scales of a
// lane's four K rows are one dword.  No two tokens share a byte, so a token is appended without
// reading its neighbours.  At D = 128 and 4 bits a block is 2176 bytes, 17 lines of 128.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "pearl_internal.h"

namespace pearl {

template <int D, int kBits> struct MxBlock {
  static_assert(D == 64 || D == 128, "head_dim");
  static_assert(kBits == 4 || kBits == 8, "element bits");
  static constexpr int kRow = D * kBits / 8;        // bytes of a token's codes
  static constexpr int kCodes = kPage * kRow;
  static constexpr int kBlocks = D / 32;            // scales of a token
  static constexpr int kTokensPerUnit = 64 / kBits;
  static constexpr int kVCodes = kCodes;            // offsets
  static constexpr int kKScales = 2 * kCodes;
  static constexpr int kVScales = kKScales + kPage * kBlocks;
  static constexpr int kBytes = kVScales + kPage * kBlocks;
  static_assert(kBytes % 64 == 0, "blocks stay aligned");
  __device__ static __forceinline__ int k_scale(int slot, int blk) {
    return kKScales + ((slot & 3) * kBlocks + blk) * 4 + (slot >> 2);
  }
  __device__ static __forceinline__ int v_scale(int slot, int blk) { return kVScales + blk * kPage + slot; }
  // the unit of a channel pair that holds a token, and the token's place in it
  __device__ static __forceinline__ int v_code(int slot, int pair) {
    return kVCodes + (slot / kTokensPerUnit * (D / 2) + pair) * 16 + slot % kTokensPerUnit * (kBits / 4);
  }
};

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x2 __attribute__((ext_vector_type(2)));

// 2^(s - 127) as the conversion instructions take it: a float of which only the exponent bits count, 0 for
// 2^-127 and 255 for NaN (every code and scale, and other bits set beside the exponent: checked on the
// device against the definition).
__device__ __forceinline__ float mx_scale(uint32_t s) { return __builtin_bit_cast(float, s << 23); }
// the same for byte k of a word
template <int k> __device__ __forceinline__ float mx_scale_of(uint32_t w) {
  return __builtin_bit_cast(float, k < 3 ? w << (23 - 8 * k) : w >> 1);
}

// Whether one of a word's four scales may make elements infinite or NaN (a bit per byte).  All are finite up to scales of
// 252 at 4 bits (6 * 2^125) and 246 at 8 (448 * 2^119); some scales below are taken along, for fewer instructions.
template <int kBits> __device__ __forceinline__ uint32_t mx_large_scale(uint32_t w) {
  if constexpr (kBits == 4) return ((w >> 2 & 0x3f3f3f3fu) + 0x01010101u) & 0x40404040u;   // 252 and more
  else return ((w >> 4 & 0x0f0f0f0fu) + 0x01010101u) & 0x10101010u;                        // 240 and more
}
// Whether one of a word's four 8-bit elements is E4M3's NaN, 0x7f or 0xff: its byte's bit in kMxNanBits.
constexpr uint32_t kMxNanBits = 0x80808080u;
__device__ __forceinline__ uint32_t mx_nan_code(uint32_t w) { return (w & 0x7f7f7f7fu) + 0x01010101u; }

// Whether the low or the high one of two bf16 in a dword is infinite or NaN.
__device__ __forceinline__ bool mx_low_not_finite(uint32_t w) { return (w & 0x7f80u) == 0x7f80u; }
__device__ __forceinline__ bool mx_high_not_finite(uint32_t w) { return (w & 0x7f800000u) == 0x7f800000u; }

// 16 bits of a buffer that is read in other types too.
typedef uint16_t u16_any __attribute__((may_alias));

// Two elements (byte kSel of w, or 16-bit half kSel at 8 bits) as bf16 in a dword: exact, except values
// under 2^-133, the least bf16, which are rounded to it.
template <int kBits, int kSel> __device__ __forceinline__ uint32_t mx_up(uint32_t w, float scale) {
  if constexpr (kBits == 4) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, kSel));
  else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, kSel != 0));
}

}  // namespace pearl
