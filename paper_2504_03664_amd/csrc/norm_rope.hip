// Per-head RMSNorm of q and k with the rotary positions in the same pass:
//   y = x / sqrt(mean(x^2) + eps) * gamma                        (a head's D elements)
//   out_i = y_i cos - y_{i + D/2} sin,  out_{i + D/2} = y_{i + D/2} cos + y_i sin
// (q then times q_scale), in fp32 from fp16 and rounded once.  D/16 lanes hold
// a head, eight pairs each, so the sum of squares is three (two) DPP moves and
// the pairs never leave a lane.  Bound by HBM: each element is read and written
// once, cos and sin come from the caches (8192 rows of 32 + 8 heads of 128: 168 MB
// in 32.4 us, 5.2 TB/s, where a large copy moves 4.86), and by the launch for a decode
// step (16 rows: 3.2 us).
#include <algorithm>

#include "common.h"
#include "device.h"
#include "kvquant.h"

namespace pipo {

struct NormRope {
  const uint16_t *q, *k, *gq, *gk;
  uint16_t *qo, *ko;
  const float* cs;
  const int32_t* pos;
  int64_t ldq, ldk, ldqo, ldko, M, n_pos;
  int H, Hkv;
  float eps, q_scale;
};

constexpr int64_t kL2Bytes = 8 << 22;  // of all XCDs

// eight halves; VEC: 16-byte aligned
template <bool VEC>
__device__ __forceinline__ h8 load8(const uint16_t* p) {
  if constexpr (VEC) return load_h8(p);
  h8 v;
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = __builtin_bit_cast(_Float16, p[j]);
  return v;
}
// STREAM: past the L2, which the rows would not stay in
template <bool VEC, bool STREAM>
__device__ __forceinline__ void store8(uint16_t* p, h8 v) {
  if constexpr (VEC && STREAM) {
    __builtin_nontemporal_store(__builtin_bit_cast(u32x4, v), reinterpret_cast<u32x4*>(p));
  } else if constexpr (VEC) {
    *reinterpret_cast<u32x4*>(p) = __builtin_bit_cast(u32x4, v);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const _Float16 x = v[j];  // (clang's bit_cast of a vector's element reads element 0)
      p[j] = __builtin_bit_cast(uint16_t, x);
    }
  }
}

template <int D, bool VEC, bool STREAM>
__global__ __launch_bounds__(256) void norm_rope_k(NormRope a) {
  constexpr int LPH = D / 16, GPB = 256 / LPH;  // lanes per head, heads of a block
  const uint32_t NH = a.H + a.Hkv;
  const int64_t unit =
      ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * GPB + threadIdx.x / LPH;
  if (unit >= a.M * NH) return;
  int64_t m;
  uint32_t h;
  if (a.M * NH < ((int64_t)1 << 32)) {
    const uint32_t row = (uint32_t)unit / NH;
    m = row;
    h = (uint32_t)unit - row * NH;
  } else {
    m = unit / NH;
    h = (uint32_t)(unit - m * NH);
  }
  const int64_t p = a.pos[m];
  if (p < 0 || p >= a.n_pos) return;
  const int i = 8 * (threadIdx.x % LPH);
  const float* c = a.cs + p * D + 2 * i;  // D/2 (cos, sin) pairs per position
  const bool is_q = h < (uint32_t)a.H;
  const uint16_t* x = is_q ? a.q + m * a.ldq + (int64_t)h * D
                           : a.k + m * a.ldk + (int64_t)(h - a.H) * D;
  uint16_t* y = is_q ? a.qo + m * a.ldqo + (int64_t)h * D
                     : a.ko + m * a.ldko + (int64_t)(h - a.H) * D;
  const uint16_t* gamma = is_q ? a.gq : a.gk;
  const float scale = is_q ? a.q_scale : 1.f;
  const h8 xa = load8<VEC>(x + i), xb = load8<VEC>(x + i + D / 2);
  float u[8], v[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    u[j] = (float)xa[j];
    v[j] = (float)xb[j];
  }
  if (gamma) {
    const h8 ga = load8<VEC>(gamma + i), gb = load8<VEC>(gamma + i + D / 2);
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) s += u[j] * u[j] + v[j] * v[j];
    s += lane_move<0xB1>(s);
    s += lane_move<0x4E>(s);
    if constexpr (LPH == 8) s += lane_move<0x141>(s);
    const float r = 1.f / sqrtf(s * (1.f / D) + a.eps);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      u[j] *= r * (float)ga[j];
      v[j] *= r * (float)gb[j];
    }
  }
  h8 oa, ob;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float co = c[2 * j], si = c[2 * j + 1];
    oa[j] = (_Float16)((u[j] * co - v[j] * si) * scale);
    ob[j] = (_Float16)((v[j] * co + u[j] * si) * scale);
  }
  store8<VEC, STREAM>(y + i, oa);
  store8<VEC, STREAM>(y + i + D / 2, ob);
}

pipo_status launch_qk_norm_rope(const NormRope& a, int D, hipStream_t st) {
  if (a.M == 0) return PIPO_OK;
  const bool vec = (reinterpret_cast<uintptr_t>(a.q) | reinterpret_cast<uintptr_t>(a.k) |
                    reinterpret_cast<uintptr_t>(a.qo) | reinterpret_cast<uintptr_t>(a.ko) |
                    reinterpret_cast<uintptr_t>(a.gq) | reinterpret_cast<uintptr_t>(a.gk)) % 16 == 0 &&
                   (a.ldq | a.ldk | a.ldqo | a.ldko) % 8 == 0;
  const auto go = [&](auto kernel) {
    const int64_t gpb = 256 / (D / 16), blocks = (a.M * (a.H + a.Hkv) + gpb - 1) / gpb;
    // (a launch takes under 2^32 threads in a dimension)
    const int64_t row = (int64_t)1 << 22;
    const dim3 grid((unsigned)std::min(blocks, row), (unsigned)((blocks + row - 1) / row));
    launch(kernel, grid, dim3(256), 0, st, a);
  };
  // (8192 rows of 32 + 8 heads of 128: 37.9 us with ordinary stores, 32.4 with these)
  const bool stream = vec && a.M * (a.H + a.Hkv) * D * 2 > kL2Bytes;
  if (D == 128)
    stream ? go(norm_rope_k<128, true, true>)
           : vec ? go(norm_rope_k<128, true, false>) : go(norm_rope_k<128, false, false>);
  else
    stream ? go(norm_rope_k<64, true, true>)
           : vec ? go(norm_rope_k<64, true, false>) : go(norm_rope_k<64, false, false>);
  PIPO_HIP_TRY(hipGetLastError());
  return PIPO_OK;
}

}  // namespace pipo

extern "C" pipo_status pipo_op_qk_norm_rope(
    const uint16_t* q, int64_t ldq, const uint16_t* k, int64_t ldk, const uint16_t* q_gamma,
    const uint16_t* k_gamma, const float* cos_sin, int64_t n_pos, const int32_t* pos,
    uint16_t* q_out, int64_t ldqo, uint16_t* k_out, int64_t ldko, int64_t M, int32_t n_heads,
    int32_t n_kv_heads, int32_t head_dim, float eps, float q_scale, void* stream) {
  using namespace pipo;
  clear_error();
  if (M < 0 || n_heads < 1 || n_kv_heads < 1 || n_pos < 1 || !(eps >= 0.f)) {
    set_error("qk_norm_rope: M %lld, heads %d/%d, %lld positions, eps %g", (long long)M, n_heads,
              n_kv_heads, (long long)n_pos, (double)eps);
    return PIPO_ERR_ARG;
  }
  if (head_dim != 64 && head_dim != 128) {
    set_error("qk_norm_rope: head_dim %d not supported (64 or 128)", head_dim);
    return PIPO_ERR_UNSUPPORTED;
  }
  const int64_t dq = (int64_t)n_heads * head_dim, dk = (int64_t)n_kv_heads * head_dim;
  if (!q || !k || !cos_sin || !pos || !q_out || !k_out || ldq < dq || ldqo < dq || ldk < dk ||
      ldko < dk) {
    set_error("qk_norm_rope: NULL pointer, or rows (%lld, %lld, %lld, %lld) shorter than the heads",
              (long long)ldq, (long long)ldk, (long long)ldqo, (long long)ldko);
    return PIPO_ERR_ARG;
  }
  // (the second: a grid of 2^16 rows of 2^22 blocks at most)
  if (M >= ((int64_t)1 << 31) || M * (n_heads + (int64_t)n_kv_heads) >= ((int64_t)1 << 40)) {
    set_error("qk_norm_rope: %lld rows of %d + %d heads", (long long)M, n_heads, n_kv_heads);
    return PIPO_ERR_UNSUPPORTED;
  }
  NormRope a{q, k, q_gamma, k_gamma, q_out, k_out, cos_sin, pos, ldq, ldk, ldqo, ldko, M, n_pos,
             n_heads, n_kv_heads, eps, q_scale};
  return launch_qk_norm_rope(a, head_dim, static_cast<hipStream_t>(stream));
}
