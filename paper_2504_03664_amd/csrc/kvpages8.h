// Pages of an 8-bit KV cache (pipo_kv8_pages in pipo_ops.h): addressing and codes,
// shared by the kernels that fill, read and attend to them.
//
// A page holds page_size positions of every key/value head, head after head,
// each head's positions in tiles of 16, and behind all of them two floats a tile
// (head after head again): the scales of its keys and of its values.  A tile
// is 32 D bytes, K codes and then V codes, in the order in which lanes (r, g), lane
// r + 16 g, hold operands of the 16 x 16 x 32 matrix products, 16 bytes a lane and 1 KiB
// a load:
//   K: bytes 1024 c + 16 (key + 16 g) + 8 j + b: dimension 64 c + 32 j + 8 g + b;
//   V: bytes 1024 c + 16 (r + 16 g) + 4 m + b: key 4 g + b, dimension 64 c + 16 m + r.
// Scales are powers of two within bounds for which code * scale is an fp16 number
// for every code: products may take the values themselves, and reading rounds nothing.
#pragma once

#include "common.h"
#include "device.h"

namespace pipo {

constexpr float kKv8Clamp = 57344.f;  // 448 * 2^7: of an element before it is quantized

// one layer of a pipo_kv8_pages as kernels take it
struct Pages8 {
  uint8_t* pool;
  const int32_t* table;
  int64_t stride;       // of the table's rows
  int64_t page_bytes;
  uint32_t scales_at;   // in a page
  int n_pages, ps_log2, Hkv, n_seq;
};

template <int D>
constexpr int kTile8 = 32 * D;

__device__ __forceinline__ uint32_t tile8_index(const Pages8& c, int head, int pos) {
  const int log2 = c.ps_log2 - 4;
  return ((uint32_t)head << log2) + ((pos >> 4) & ((1 << log2) - 1));
}
template <int D>
__device__ __forceinline__ uint8_t* tile8_at(const Pages8& c, int page, int head, int pos) {
  return c.pool + (int64_t)page * c.page_bytes + tile8_index(c, head, pos) * (uint32_t)kTile8<D>;
}
__device__ __forceinline__ float* scales8_at(const Pages8& c, int page, int head, int pos) {
  return reinterpret_cast<float*>(c.pool + (int64_t)page * c.page_bytes + c.scales_at +
                                  8 * tile8_index(c, head, pos));
}

// exponents of scales, and the largest magnitude in units of the scale
template <bool INT8>
struct Kv8 {
  static constexpr int kLow = INT8 ? -24 : -15, kHigh = INT8 ? 9 : 7;
  static constexpr int kTopExp = INT8 ? 6 : 8;                      // of 127 and 448,
  static constexpr uint32_t kTopFrac = INT8 ? 0x7E0000 : 0x600000;  // and their fraction
};
__device__ __forceinline__ int exponent(float x) {
  return (int)(__float_as_uint(x) >> 23 & 255) - 127;
}
__device__ __forceinline__ float power(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// two codes (bytes 0 and 1 or, HI, 2 and 3 of a word) as halves, times a scale in
// range.  E4M3: one instruction, which takes the scale along.  INT8: c + 128 under the
// exponent of 1024, where the last bit counts one, less 1152.
template <bool HI>
__device__ __forceinline__ h2 e4m3_halves(uint32_t w, float scale) {
  return __builtin_bit_cast(h2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, HI));
}
template <bool HI>
__device__ __forceinline__ h2 int8_halves(uint32_t w_flipped) {  // w ^ 0x80808080
  const uint32_t u = __builtin_amdgcn_perm(0x64646464u, w_flipped, HI ? 0x04030402u : 0x04010400u);
  return __builtin_bit_cast(h2, u) - h2{(_Float16)1152.f, (_Float16)1152.f};
}

// eight codes of two words -> halves; UNIT: in units of the scale
template <bool INT8, bool UNIT>
__device__ __forceinline__ h8 halves8(uint32_t w0, uint32_t w1, float s0, float s1) {
  h2 p[4];
  if constexpr (INT8) {
    const uint32_t f0 = w0 ^ 0x80808080u, f1 = w1 ^ 0x80808080u;
    p[0] = int8_halves<false>(f0);
    p[1] = int8_halves<true>(f0);
    p[2] = int8_halves<false>(f1);
    p[3] = int8_halves<true>(f1);
    if constexpr (!UNIT) {
      const _Float16 a = (_Float16)s0, b = (_Float16)s1;
      p[0] *= h2{a, a};
      p[1] *= h2{a, a};
      p[2] *= h2{b, b};
      p[3] *= h2{b, b};
    }
  } else {
    p[0] = e4m3_halves<false>(w0, UNIT ? 1.f : s0);
    p[1] = e4m3_halves<true>(w0, UNIT ? 1.f : s0);
    p[2] = e4m3_halves<false>(w1, UNIT ? 1.f : s1);
    p[3] = e4m3_halves<true>(w1, UNIT ? 1.f : s1);
  }
  return h8{p[0][0], p[0][1], p[1][0], p[1][1], p[2][0], p[2][1], p[3][0], p[3][1]};
}

pipo_status check_pages8(const char* what, const pipo_kv8_pages* c, int32_t layer, Pages8* v);

}  // namespace pipo
