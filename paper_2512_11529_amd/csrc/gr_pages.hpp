// What the calls over pages of a pool share: their element types, how FP4 pages are laid out, and the conversions to and from codes.  Not part of the ABI.
#pragma once
#include <math.h>
#include "gr_internal.hpp"

static inline bool gr_page_size_ok(int32_t ps) { return ps >= 16 && ps <= 1024 && (ps & (ps - 1)) == 0; }
static inline bool gr_scale_ok(float s) { return s > 0.f && s < INFINITY; }

// GR_KV_FP4: for each page and KV head a record of its own: the tokens' codes, d / 2 bytes each (element 2 i in the low half of byte i), and behind them the
// tokens' scales, d / 32 bytes each.  (A head's tokens lie together because half a byte an element leaves a token's head shorter than a line of 128 bytes, whose
// other half would be another KV head's, which another XCD reads.)
static constexpr uint32_t gr_fp4_codes(uint32_t page_size, uint32_t d) { return page_size * (d / 2); }
static constexpr uint32_t gr_fp4_record(uint32_t page_size, uint32_t d) { return page_size * (d / 2 + d / 32); }

#ifdef __HIPCC__
namespace {

typedef __bf16 kv_bf16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t kv_u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t kv_u32x2 __attribute__((ext_vector_type(2)));

// x / scale, within +-448; NaN stays NaN.
// FAST: the quotient from the scale's reciprocal r (rounded to nearest) and one correction by the exact remainder, q = q0 + (x - q0 scale) r with q0 = x r, which rounds as the
// division does for every bf16 x (Markstein's theorem; of the 2^30 pairs of a scale's significand and a bf16 value's none differs from the division.  Powers of two beside them change nothing
// for scales from 2^-60 to 2^60, where the remainder of a value whose code is not 0 is far from underflow); for other x it is the division's or a neighbour of it.
// q0 is held within +-512, so that an infinite one does not make the remainder NaN: the result saturates all the same.  16 x 60-700 rows of 8 x 128 from a fused projection
// 10.0 us with the division.
template <bool FAST>
__device__ __forceinline__ float fp8_quotient(float x, float scale, float r) {
  float y;
  if (FAST) {
    const float q0 = fminf(fmaxf(x * r, -512.f), 512.f);
    y = copysignf(fmaf(fmaf(-q0, scale, x), r, q0), x);        // (-0 lost its sign)
  } else {
    y = x / scale;
  }
  return x != x ? x : fminf(fmaxf(y, -448.f), 448.f);
}
// Four quotients as E4M3 codes, rounded to nearest even.
__device__ __forceinline__ uint32_t fp8_codes4(float a, float b, float c, float d) {
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
}

__device__ __forceinline__ float bf16_at(uint32_t w, int odd) { return __uint_as_float(odd ? w & 0xffff0000u : w << 16); }
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  const kv_bf16x2 h = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, h);
}
// Eight FP4 codes (the first in the low bits) under the scale 2^(power - 127), in bf16: exact for powers from 7 to 252, which are those that are written.
__device__ __forceinline__ kv_u32x4 fp4_values8(uint32_t codes, uint32_t power) {
  const float scale = __uint_as_float(power << 23);
  return kv_u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1)),
                  __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3))};
}

}  // namespace
#endif
