// The INT4 recipe of PIPO_KV_INT4_G64 (pipo.h) on eight elements per lane,
// eight adjacent lanes per group of 64.
#pragma once

#include "device.h"

namespace pipo {

// largest of the 8 lanes of a group, by DPP moves within a row of 16 lanes
// (swap neighbours, swap pairs, mirror within 8)
template <int CTRL>
__device__ __forceinline__ float lane_move(float v) {
  return __uint_as_float(
      __builtin_amdgcn_update_dpp(0u, __float_as_uint(v), CTRL, 0xF, 0xF, false));
}
__device__ __forceinline__ float group_max8(float v) {
  v = fmaxf(v, lane_move<0xB1>(v));
  v = fmaxf(v, lane_move<0x4E>(v));
  return fmaxf(v, lane_move<0x141>(v));
}
__device__ __forceinline__ float group_min8(float v) {
  v = fminf(v, lane_move<0xB1>(v));
  v = fminf(v, lane_move<0x4E>(v));
  return fminf(v, lane_move<0x141>(v));
}

// Codes as the low bits of kCodeBits + code, for pack8.
constexpr uint32_t kCodeBits = 0x4B000000u;  // 2^23, whose last bit counts 1
struct Quant8 {
  uint32_t c[8];
  uint16_t scale, min;
};

// of elements v of a group whose least and largest are mn and mx.  FINITE: all are,
// and then the two divisions are multiplications by a correctly rounded
// reciprocal with one residual step each (Markstein, IBM J. Res. Dev. 34, 1990),
// the same bits; for 1 / s, from the hardware's approximation, because s has 11
// bits, so that 1 / s is never within 2^-36 of the middle between two floats.
template <bool FINITE>
__device__ __forceinline__ Quant8 quantize8(const float (&v)[8], float mn, float mx) {
  float s32, inv;
  if constexpr (FINITE) {
    constexpr float r15 = 1.f / 15.f;
    const float x = mx - mn, q0 = x * r15;
    s32 = __builtin_fmaf(__builtin_fmaf(-q0, 15.f, x), r15, q0);
  } else {
    s32 = (mx - mn) / 15.f;
  }
  const _Float16 s16 = (_Float16)s32, m16 = (_Float16)mn;
  const float s = (float)s16, m = (float)m16;
  // (x - min) / scale, correctly rounded in the same way from the correctly
  // rounded reciprocal: an eighth of a division per element.  A scale of 0 gives
  // code 0, and so do infinite inputs (NaN, as the division would).  Adding 2^23
  // rounds half to even.
  if constexpr (FINITE) {
    const float r = __builtin_amdgcn_rcpf(s);
    inv = s != 0.f ? __builtin_fmaf(__builtin_fmaf(-s, r, 1.f), r, r) : 0.f;
  } else {
    inv = s != 0.f ? 1.f / s : 0.f;
  }
  Quant8 out;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float x = v[j] - m, q0 = x * inv;
    const float q = __builtin_fmaf(__builtin_fmaf(-q0, s, x), inv, q0);
    out.c[j] = __float_as_uint(__builtin_amdgcn_fmed3f(q, 0.f, 15.f) + 8388608.f);
  }
  out.scale = __builtin_bit_cast(uint16_t, s16);
  out.min = __builtin_bit_cast(uint16_t, m16);
  return out;
}

// code j to nibble at(j) of a word: sums of shifted bits, the constant's share
// taken off at the end
template <typename At>
__device__ __forceinline__ uint32_t pack8(const Quant8& q, At at) {
  uint32_t w = 0, bias = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    w += q.c[j] << (4 * at(j));
    bias += kCodeBits << (4 * at(j));
  }
  return w - bias;
}

}  // namespace pipo
