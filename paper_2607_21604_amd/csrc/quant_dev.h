// Device helpers of the group-64 quantiser: a lane holds 8 consecutive elements, a group of 64 sits
// on 8 aligned lanes of one DPP row.
#pragma once
#include "common.h"

namespace akvs {

template <int CTRL>
__device__ __forceinline__ float dpp_f32(float x) {
  return __int_as_float(
      __builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, false));
}
__device__ __forceinline__ float oct_max(float x) {  // over aligned groups of 8 lanes
  x = fmaxf(x, dpp_f32<0xB1>(x));    // lane ^ 1
  x = fmaxf(x, dpp_f32<0x4E>(x));    // lane ^ 2
  return fmaxf(x, dpp_f32<0x141>(x));  // the two quads of the 8 lanes
}
__device__ __forceinline__ float oct_min(float x) {
  x = fminf(x, dpp_f32<0xB1>(x));
  x = fminf(x, dpp_f32<0x4E>(x));
  return fminf(x, dpp_f32<0x141>(x));
}
__device__ __forceinline__ float oct_sum(float x) {
  x += dpp_f32<0xB1>(x);
  x += dpp_f32<0x4E>(x);
  return x + dpp_f32<0x141>(x);
}

// Quotient rounded to an integer code 0..levels (rne), from v = x - zero.
__device__ __forceinline__ uint32_t int_code(float tq, float levels) {
  return (uint32_t)(int)fminf(fmaxf(rintf(tq), 0.f), levels);
}

// The 4-bit codes (element i at bits 4 i) and (scale, zero) of a lane's octet; all lanes of its
// group call. The quotients are formed with the group's reciprocal, off by at most 2 ulp, and by
// division only where that lies near a rounding boundary: the codes are those of the division.
__device__ __forceinline__ void u4_octet(const float (&v)[8], uint32_t &word, uint32_t &meta) {
  float lo = v[0], hi = v[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) {
    lo = fminf(lo, v[i]);
    hi = fmaxf(hi, v[i]);
  }
  lo = oct_min(lo);
  hi = oct_max(hi);
  const _Float16 z16 = (_Float16)lo, s16 = (_Float16)__fdiv_rn(hi - lo, 15.f);
  const float scale = (float)s16, zero = (float)z16;
  word = 0;
  if (scale != 0.f) {
    const float rs = __fdiv_rn(1.0f, scale);
    float t[8];
    bool near = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      t[i] = (v[i] - zero) * rs;
      near |= fabsf(__builtin_amdgcn_fractf(t[i]) - 0.5f) < 2e-5f;
    }
    if (near) {
#pragma unroll
      for (int i = 0; i < 8; ++i) t[i] = __fdiv_rn(v[i] - zero, scale);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) word |= int_code(t[i], 15.f) << (4 * i);
  }
  meta = (uint32_t)__builtin_bit_cast(uint16_t, s16) |
         ((uint32_t)__builtin_bit_cast(uint16_t, z16) << 16);
}

}  // namespace akvs
