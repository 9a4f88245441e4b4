// 4-bit rows: d codes of the float format E2M1 (1 sign, 2 exponent bits with bias 1, 1 fraction bit: magnitudes 0, 0.5, 1, 1.5, 2, 3, 4
// and 6), two to a byte, the even element in the low half, and one power of two for every 32 of them, value = code * 2^e.
#pragma once

#include "device_utils.h"

namespace d2o {

struct Code4 {  // two elements
  uint8_t two;
};
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

constexpr int kBlock4 = 32;      // elements that share a power of two
constexpr int kNan4 = -128;      // exponent of a block with an infinity or NaN: all of it is NaN

// A block's exponent from the bits of its largest magnitude: the smallest e with amax <= 6 * 2^e (6 = 1.5 * 2^2), within [-120, 125]
// (6 * 2^125 is the largest power that bf16 holds with all codes; values above it, up to 1.33 times as large, become it); 0 for a block of zeros.
__device__ __forceinline__ int fp4_exponent(uint32_t amax) {
  if (amax >= 0x7F800000u) return kNan4;
  const int e = int(amax >> 23) - 127 - ((amax & 0x7FFFFFu) <= 0x400000u ? 2 : 1);
  return amax == 0 ? 0 : min(max(e, -120), 125);
}
// 2^e as the conversion instructions take it, which look at the exponent bits only; kNan4 gives an infinity, with which every code becomes NaN.
__device__ __forceinline__ float fp4_scale(int e) { return __uint_as_float(uint32_t(e + 127) << 23); }

// Eight bf16 elements (pairs in x) to eight codes: to nearest, in the middle of two to the even code.
__device__ __forceinline__ uint32_t fp4_encode8(const u32x4& x, int e) {
  const float scale = fp4_scale(e == kNan4 ? 0 : e);
  const uint32_t x0 = x[0], x1 = x[1], x2 = x[2], x3 = x[3];  // (a bit cast of a vector's element itself takes the first one)
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, x0), scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, x1), scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, x2), scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, x3), scale, 3);
}
// Eight codes to bf16 (exact: two significant bits).
__device__ __forceinline__ u32x4 fp4_decode8(uint32_t w, float scale) {
  return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3))};
}
// The largest magnitude of eight bf16 elements, as the bits of a float (NaN above infinity).
__device__ __forceinline__ uint32_t fp4_amax8(const u32x4& x) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) m = max(m, max((x[i] << 16) & 0x7FFF0000u, x[i] & 0x7FFF0000u));
  return m;
}
// Eight bf16 elements of each lane, four neighbouring lanes a block: codes and the block's exponent.
__device__ __forceinline__ uint32_t fp4_encode_block(const u32x4& x, int& e) {
  uint32_t m = fp4_amax8(x);
  m = max(m, uint32_t(dpp_i32<kDppXor1>(int(m))));
  m = max(m, uint32_t(dpp_i32<kDppXor2>(int(m))));
  e = fp4_exponent(m);
  return fp4_encode8(x, e);
}

}  // namespace d2o
