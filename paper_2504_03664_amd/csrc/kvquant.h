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

struct Quant8 {
  uint32_t c[8];
  uint16_t scale, min;
};

__device__ __forceinline__ Quant8 quantize8(const float (&v)[8]) {
  float mn = v[0], mx = v[0];
#pragma unroll
  for (int j = 1; j < 8; ++j) {
    mn = fminf(mn, v[j]);
    mx = fmaxf(mx, v[j]);
  }
  mn = group_min8(mn);
  mx = group_max8(mx);
  const _Float16 s16 = (_Float16)((mx - mn) / 15.f);
  const _Float16 m16 = (_Float16)mn;
  const float s = (float)s16, m = (float)m16;
  // (x - min) / scale, correctly rounded from the correctly rounded reciprocal
  // and one residual step (Markstein, IBM J. Res. Dev. 34, 1990): an eighth of
  // a division per element.  Infinite inputs give NaN and code 0, as the
  // division would.
  const float inv = s != 0.f ? 1.f / s : 0.f;
  Quant8 out;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float x = v[j] - m, q0 = x * inv;
    const float q = __builtin_fmaf(__builtin_fmaf(-q0, s, x), inv, q0);
    out.c[j] = (uint32_t)(s != 0.f ? fminf(fmaxf(__builtin_rintf(q), 0.f), 15.f) : 0.f);
  }
  out.scale = __builtin_bit_cast(uint16_t, s16);
  out.min = __builtin_bit_cast(uint16_t, m16);
  return out;
}

}  // namespace pipo
