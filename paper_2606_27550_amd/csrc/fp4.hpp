// Four-bit rows: groups of 32 values along a row share a scale byte b, the
// power of two 2^(b - 127) (255: not a number), and every value is a code of
// sign and one of 0, 1/2, 1, 3/2, 2, 3, 4, 6, two codes a byte, the first in the
// lower half.  The matrix instructions take codes and scale bytes as they are;
// as bf16 numbers the values are exact.
#pragma once

#include "common.hpp"

namespace entmtp {

constexpr int kFp4Group = 32;
constexpr int kFp4RowBytes = ENTMTP_HEAD_DIM / 2 + ENTMTP_HEAD_DIM / kFp4Group;   // of a head's row: 68
static_assert(kFp4RowBytes == ENTMTP_FP4_ROW, "the header's row");
constexpr uint32_t kFp4NaN = 255;
constexpr uint32_t kFp4Top = 252;   // from here on 6 steps pass bf16's largest number

typedef __bf16 bf16v2 __attribute__((ext_vector_type(2)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

// Scale byte of a group whose largest magnitude has the bf16 bits top: the
// largest value comes to lie in [3.5, 7) steps of the scale, so that it is off by
// at most one (rounding it up to 4 from 3.5, down to 6 from 7: the same).  Held
// in [2, 252], so that every value is a normal bf16 number or zero; 255 where a
// value is not finite.
__device__ __forceinline__ uint32_t fp4_scale(uint32_t top) {
  const int e = static_cast<int>((top + 0x20u) >> 7) - 2;   // (the carry is that of a mantissa of 1.75 or more)
  return top >= 0x7f80u ? kFp4NaN : static_cast<uint32_t>(e < 2 ? 2 : (e > static_cast<int>(kFp4Top) ? kFp4Top : e));
}
__device__ __forceinline__ float fp4_step(uint32_t b) { return __uint_as_float(b << 23); }   // b in [1, 254]

// Codes of eight bf16 values (one to a half word) at scale step: the nearest, of
// two equally near ones the even code, beyond 6 steps 6; zero where the scale
// byte is 255.
__device__ __forceinline__ uint32_t fp4_codes(u32x4 x, uint32_t b) {
  const float step = fp4_step(b == kFp4NaN ? 127u : b);
  uint32_t w = 0u;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16v2, static_cast<uint32_t>(x[0])), step, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16v2, static_cast<uint32_t>(x[1])), step, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16v2, static_cast<uint32_t>(x[2])), step, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16v2, static_cast<uint32_t>(x[3])), step, 3);
  return b == kFp4NaN ? 0u : w;
}

// The eight values of a word of codes, in bf16.
__device__ __forceinline__ u32x4 fp4_values(uint32_t w, float step) {
  u32x4 v;
  v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, step, 0));
  v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, step, 1));
  v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, step, 2));
  v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, step, 3));
  return v;
}

// The largest magnitude's bits among eight bf16 values (NaN above infinity above the rest).
__device__ __forceinline__ uint32_t bf16_top(u32x4 x) {
  uint32_t m = 0u;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t lo = x[e] & 0x7fffu, hi = x[e] >> 16 & 0x7fffu;
    m = max(m, max(lo, hi));
  }
  return m;
}

}  // namespace entmtp
