// Rows into and out of the pages of an 8-bit KV cache (layout in kvpages8.h;
// pipo_kv8_pages in pipo_ops.h).
//
//   pages8_append_k: a wave for each tile of 16 positions that gets rows, head, and K
//                    or V: it alone holds what decides the tile's scale.
//   pages8_read_k:   slots -> fp16 rows, a thread on 32 elements of two heads.
// Both are bound by HBM (4096 rows of 56 heads of 128: append 44 us, 4.0 TB/s; read 40 us, 4.4
// TB/s of which two thirds are stores), a step's 16 rows by the launch (5 us each).
// With scales that are powers of two every product here is exact; only the
// conversions to codes round.
#include "kvpages8.h"

#include <algorithm>
#include <type_traits>

#include "kvpages.h"

namespace pipo {

struct Rows8 {
  Pages8 c;
  const uint16_t *k, *v;
  int64_t ldk, ldv, M;
  const int32_t *q_start, *kv_len;
};

__device__ __forceinline__ int start_of(const Rows8& a, int i) {
  return (int)min(max((int64_t)a.q_start[i], (int64_t)0), a.M);
}
// Slots of work: sequence i's tiles with new rows are slots q_start[i] / 16 + 2 i and on,
// of which there are enough (n rows touch at most n / 16 + 2 tiles), so that a slot's
// sequence is found by a search and no sums over sequences: 64 candidates at a time.
// The last i with q_start[i] / 16 + 2 i <= slot; -1: none.
__device__ __forceinline__ int seq_of_slot(const Rows8& a, int64_t slot) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = a.c.n_seq;
  for (;;) {
    const int step = (n + 63) / 64, i = lo + lane * step;
    const bool in = lane * step < n;
    const uint64_t below =
        __ballot(in && start_of(a, in ? i : 0) / 16 + 2 * (int64_t)i <= slot);
    const int k = __popcll(below) - 1;
    if (k < 0) return -1;
    lo += k * step;
    n = min(step, n - k * step);
    if (n <= 1) return lo;
  }
}

// bits of the largest magnitude of a wave's halves (finite)
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v = max(v, (uint32_t)__shfl_xor((int)v, d, 64));
  return v;
}

// eight elements clamped, NaN as 0, and the largest of their magnitudes' bits
__device__ __forceinline__ void clamp8(h8& x, uint32_t& top) {
  u32x4 w = __builtin_bit_cast(u32x4, x);
  typedef uint16_t us2 __attribute__((ext_vector_type(2)));
  constexpr uint16_t kLimit = 0x7B00;  // kKv8Clamp's bits
  us2 t = us2{0, 0};
#pragma unroll
  for (int j = 0; j < 4; ++j)
    t = __builtin_elementwise_max(t, __builtin_bit_cast(us2, w[j] & 0x7FFF7FFFu));
  if (__any(max(t[0], t[1]) > kLimit)) {  // hardly ever
    t = us2{0, 0};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float f = (float)x[j];
      x[j] = (_Float16)(f == f ? fminf(fmaxf(f, -kKv8Clamp), kKv8Clamp) : 0.f);
    }
    w = __builtin_bit_cast(u32x4, x);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      t = __builtin_elementwise_max(t, __builtin_bit_cast(us2, w[j] & 0x7FFF7FFFu));
  }
  top = max(top, (uint32_t)max(t[0], t[1]));
}

template <bool INT8>
__device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d) {
  if constexpr (INT8) {
    const uint32_t x = (uint8_t)(int)__builtin_rintf(a) | (uint32_t)(uint8_t)(int)__builtin_rintf(b) << 8;
    return x | (uint32_t)(uint8_t)(int)__builtin_rintf(c) << 16 |
           (uint32_t)(uint8_t)(int)__builtin_rintf(d) << 24;
  } else {
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false),
                                                     true);
  }
}
// elements 4 i .. 4 i + 3 over a scale (inv: its reciprocal) -> codes
template <bool INT8>
__device__ __forceinline__ uint32_t codes4(h8 x, int i, float inv) {
  return pack4<INT8>((float)x[4 * i] * inv, (float)x[4 * i + 1] * inv, (float)x[4 * i + 2] * inv,
                     (float)x[4 * i + 3] * inv);
}
// codes of a smaller scale, ratio f at most 1
template <bool INT8>
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float f) {
  if constexpr (INT8) {
    return pack4<true>((float)(int8_t)w * f, (float)(int8_t)(w >> 8) * f, (float)(int8_t)(w >> 16) * f,
                       (float)(int8_t)(w >> 24) * f);
  } else {
    const h2 lo = e4m3_halves<false>(w, 1.f), hi = e4m3_halves<true>(w, 1.f);
    return pack4<false>((float)lo[0] * f, (float)lo[1] * f, (float)hi[0] * f, (float)hi[1] * f);
  }
}

template <int CTRL>
__device__ __forceinline__ uint32_t quad_move(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, false);
}
// four lanes' words as a 4 x 4 matrix of bytes, transposed
__device__ __forceinline__ uint32_t transpose4(uint32_t w, int lane) {
  const uint32_t o = quad_move<0xB1>(w);
  w = lane & 1 ? __builtin_amdgcn_perm(w, o, 0x07030501u) : __builtin_amdgcn_perm(o, w, 0x06020400u);
  const uint32_t p = quad_move<0x4E>(w);
  return lane & 2 ? __builtin_amdgcn_perm(w, p, 0x07060302u) : __builtin_amdgcn_perm(p, w, 0x05040100u);
}

// eight codes as halves to a row
template <bool INT8, bool VEC>
__device__ __forceinline__ void store8(uint16_t* dst, uint32_t w0, uint32_t w1, float scale) {
  const h8 x = halves8<INT8, false>(w0, w1, scale, scale);
  if constexpr (VEC) {
    *reinterpret_cast<u32x4*>(dst) = __builtin_bit_cast(u32x4, x);
  } else {
    const u32x4 y = __builtin_bit_cast(u32x4, x);
#pragma unroll
    for (int j = 0; j < 8; ++j) dst[j] = (uint16_t)(y[j / 2] >> (16 * (j & 1)));
  }
}

template <bool VEC>
__device__ __forceinline__ h8 row8(const uint16_t* p) {
  if constexpr (VEC) return load_h8(p);
  h8 v;
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = __builtin_bit_cast(_Float16, p[j]);
  return v;
}

template <int D, bool INT8, bool VEC>
__global__ __launch_bounds__(256) void pages8_append_k(Rows8 a) {
  constexpr int C = D / 64;
  using F = Kv8<INT8>;
  const Pages8& c = a.c;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t groups = (2 * c.Hkv + 3) / 4;  // of four heads' waves
  const int64_t block = (int64_t)blockIdx.y * gridDim.x + blockIdx.x, slot = block / groups;
  const int hv = (int)(block - slot * groups) * 4 + wave;
  if (hv >= 2 * c.Hkv) return;
  const bool value = hv >= c.Hkv;
  const int head = value ? hv - c.Hkv : hv;
  const int i = __builtin_amdgcn_readfirstlane(seq_of_slot(a, slot));
  if (i < 0) return;
  const int r0 = start_of(a, i), r1 = max(start_of(a, i + 1), r0);
  const int64_t len = a.kv_len[i], p0 = len - (r1 - r0);   // position of row r0
  const int64_t t = max(p0, (int64_t)0) / 16 + (slot - (r0 / 16 + 2 * (int64_t)i));
  const int64_t first = 16 * t;   // position of the tile's first key
  if (r0 == r1 || first >= len || (first >> c.ps_log2) >= c.stride) return;
  const int page = c.table[i * c.stride + (first >> c.ps_log2)];
  if (page < 0 || page >= c.n_pages) return;
  // keys [kf, ke) are new, those below are the cache's
  const int kf = (int)max(max(p0, (int64_t)0) - first, (int64_t)0);
  const int ke = (int)min(len - first, (int64_t)16);
  uint8_t* tile = tile8_at<D>(c, page, head, (int)first) + (value ? 16 * D : 0);
  float* scale_at = scales8_at(c, page, head, (int)first) + (value ? 1 : 0);

  // this lane's key and the dimension of its piece n: for keys in operand order, for
  // values so that four neighbours hold four keys
  const int key = value ? 4 * (lane >> 2 & 3) + (lane & 3) : lane & 15;
  const auto dim = [&](int n) {
    return value ? 64 * (lane >> 5) + 16 * n + 8 * (lane >> 4 & 1) : 64 * (n / 2) + 32 * (n % 2) + 8 * (lane >> 4);
  };
  const bool fresh = key >= kf && key < ke && (!value || lane < 32 * C);
  const int64_t row = r0 + first + key - p0;
  const uint16_t* src = value ? a.v + row * a.ldv : a.k + row * a.ldk;
  constexpr int N = 4;   // pieces of a value's lane; a key's has 2 C
  const int pieces = value ? N : 2 * C;
  h8 x[N];
  u32x4 old[2 * C];
  float before = 0.f;
  const bool merge = kf > 0 || ke < 16;
#pragma unroll
  for (int n = 0; n < N; ++n)
    x[n] = fresh && n < pieces ? row8<VEC>(src + (int64_t)head * D + dim(n)) : zero_h8();
  // the lane's 16-byte parts of the tile: keys chunk n; values two dimensions four apart
  const int vr = 8 * (lane >> 4 & 1) + (lane & 3) + 16 * (lane >> 2 & 3);
  const auto part = [&](int n) {
    return value ? 1024 * (lane >> 5) + 16 * (vr + 4 * n) : 1024 * n + 16 * lane;
  };
  const int parts = value ? (lane < 32 * C ? 2 : 0) : C;
  if (merge) {
#pragma unroll
    for (int n = 0; n < 2; ++n)
      if (n < parts) old[n % (2 * C)] = *reinterpret_cast<const u32x4*>(tile + part(n));
    if (kf > 0) before = *scale_at;
  }
  uint32_t top = 0;
#pragma unroll
  for (int n = 0; n < N; ++n) clamp8(x[n], top);
  const float amax = h2f((uint16_t)wave_max(top));
  int e = exponent(amax) - F::kTopExp + ((__float_as_uint(amax) & 0x7FFFFF) > F::kTopFrac);
  e = min(max(e, F::kLow), F::kHigh);
  const int e0 = min(max(exponent(before), F::kLow), F::kHigh);
  const bool grows = kf > 0 && e > e0;
  if (kf > 0) e = max(e, e0);
  const float inv = power(-e), ratio = power(e0 - e);

  if (!value) {
#pragma unroll
    for (int n = 0; n < C; ++n) {
      u32x4 w;
      w[0] = codes4<INT8>(x[2 * n], 0, inv);
      w[1] = codes4<INT8>(x[2 * n], 1, inv);
      w[2] = codes4<INT8>(x[2 * n + 1], 0, inv);
      w[3] = codes4<INT8>(x[2 * n + 1], 1, inv);
      if (grows && key < kf) {
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = rescale4<INT8>(old[n][j], ratio);
      }
      if (fresh || (grows && key < kf)) *reinterpret_cast<u32x4*>(tile + part(n)) = w;
    }
  } else {
    // bytes of this lane's words: keys 4 g .. 4 g + 3
    uint32_t is_new = 0, is_old = 0;
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      const int kk = (key & ~3) + b;
      if (kk >= kf && kk < ke) is_new |= 0xFFu << (8 * b);
      if (kk < kf) is_old |= 0xFFu << (8 * b);
    }
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      u32x4 w;
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = transpose4(codes4<INT8>(x[j], n, inv), lane);
      if (merge) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t y = old[n % (2 * C)][j];
          w[j] = (w[j] & is_new) | (y & ~is_new);
          if (grows) w[j] = (w[j] & ~is_old) | (rescale4<INT8>(y, ratio) & is_old);
        }
      }
      if (n < parts && (is_new || grows)) *reinterpret_cast<u32x4*>(tile + part(n)) = w;
    }
  }
  if (lane == 0) *scale_at = power(e);
}

// A thread on 32 elements of a row's heads h0, h0 + step .. (values behind keys), D / 32
// threads a head, sixteen rows of a head side by side: rows that are consecutive positions,
// as of a prefix, then read the same words of values, a byte each of 16 bytes that a
// thread loads, out of the first-level cache (byte by byte, eight a thread, 70 us where this
// takes 40 to 46: eight prompts of 512
// rows, 56 heads of 128; stored past the L2, in its pieces of 32 bytes, 96).
constexpr int kReadHeads = 2;
__host__ __device__ constexpr int64_t read_step(int Hkv) {
  return (2 * (int64_t)Hkv + kReadHeads - 1) / kReadHeads;
}
template <int D, bool INT8, bool VEC>
__global__ __launch_bounds__(256) void pages8_read_k(Pages8 c, const int32_t* __restrict__ seq,
                                                     const int32_t* __restrict__ pos,
                                                     uint16_t* __restrict__ k, int64_t ldk,
                                                     uint16_t* __restrict__ v, int64_t ldv, int64_t M) {
  constexpr int UN = D / 32;
  const int64_t e = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 256 + threadIdx.x;
  const uint32_t step = (uint32_t)read_step(c.Hkv), per_group = step * 16 * UN;
  const int64_t group = e < ((int64_t)1 << 32) ? (uint32_t)e / per_group : e / per_group;
  const uint32_t r = (uint32_t)(e - group * per_group);
  const int64_t m = 16 * group + r / UN % 16;
  if (m >= M) return;
  const int unit = r % UN, cc = unit / 2, h = unit % 2;
  const int i = seq[m], p = pos[m];
  if (i < 0 || i >= c.n_seq || p < 0 || (p >> c.ps_log2) >= c.stride) return;
  const int page = c.table[i * c.stride + (p >> c.ps_log2)];
  if (page < 0 || page >= c.n_pages) return;
  const int key = p & 15;
  float scale[kReadHeads];
  u32x4 w[kReadHeads][8];
#pragma unroll
  for (int t = 0; t < kReadHeads; ++t) {
    const int hv = (int)(r / (16 * UN) + t * step);
    if (hv >= 2 * c.Hkv) break;
    const bool value = hv >= c.Hkv;
    const int head = value ? hv - c.Hkv : hv;
    const uint8_t* tile = tile8_at<D>(c, page, head, p) + 1024 * cc;
    scale[t] = scales8_at(c, page, head, p)[value ? 1 : 0];
    if (value) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        w[t][j] = *reinterpret_cast<const u32x4*>(tile + 16 * D + 16 * (8 * h + j + 16 * (key >> 2)));
    } else {
#pragma unroll
      for (int j = 0; j < 2; ++j)
        w[t][j] = *reinterpret_cast<const u32x4*>(tile + 16 * (key + 16 * (2 * h + j)));
    }
  }
#pragma unroll
  for (int t = 0; t < kReadHeads; ++t) {
    const int hv = (int)(r / (16 * UN) + t * step);
    if (hv >= 2 * c.Hkv) break;
    const bool value = hv >= c.Hkv;
    const int head = value ? hv - c.Hkv : hv;
    uint16_t* dst = (value ? v + m * ldv : k + m * ldk) + (int64_t)head * D + 64 * cc;
    if (value) {   // the key's byte of each word: words of four dimensions
      const uint32_t two = 0x0C0C0400u + 0x0101u * (key & 3);
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        uint32_t y[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const uint32_t lo = __builtin_amdgcn_perm(w[t][4 * j + 1][n], w[t][4 * j][n], two);
          const uint32_t hi = __builtin_amdgcn_perm(w[t][4 * j + 3][n], w[t][4 * j + 2][n], two);
          y[j] = lo | hi << 16;
        }
        store8<INT8, VEC>(dst + 16 * n + 8 * h, y[0], y[1], scale[t]);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int n = 0; n < 2; ++n)
          store8<INT8, VEC>(dst + 32 * n + 8 * (2 * h + j), w[t][j][2 * n], w[t][j][2 * n + 1], scale[t]);
    }
  }
}

static int64_t codes_bytes(int32_t page_size, int32_t n_kv_heads, int32_t head_dim) {
  return 2 * (int64_t)n_kv_heads * page_size * head_dim;
}

pipo_status check_pages8(const char* what, const pipo_kv8_pages* c, int32_t layer, Pages8* v) {
  if (!c || !c->pool || !c->table || reinterpret_cast<uintptr_t>(c->pool) % 16 != 0 ||
      (c->fmt != PIPO_KV8_E4M3 && c->fmt != PIPO_KV8_INT8)) {
    set_error("%s: NULL cache, pool or table, a pool off 16-byte alignment, or an unknown format", what);
    return PIPO_ERR_ARG;
  }
  const int64_t page = pipo_kv8_page_bytes(c->page_size, c->n_kv_heads, c->head_dim);
  if (page == 0 || c->n_seq > 65535) {
    set_error("%s: pages of %d positions of %d heads of %d, or %d sequences, not supported (16, 32, 64, "
              "128 or 256 positions, heads of 64 or 128, under 2^31 bytes; 65535 sequences)", what,
              c->page_size, c->n_kv_heads, c->head_dim, c->n_seq);
    return PIPO_ERR_UNSUPPORTED;
  }
  if (c->n_pages < 1 || c->n_layers < 1 || layer < 0 || layer >= c->n_layers || c->n_seq < 1 ||
      c->table_stride < 1 || c->layer_bytes % 16 != 0 || c->layer_bytes / page < c->n_pages) {
    set_error("%s: %d pages of %lld bytes, layer %d of %d every %lld bytes, %d sequences, table "
              "rows of %lld", what, c->n_pages, (long long)page, layer, c->n_layers,
              (long long)c->layer_bytes, c->n_seq, (long long)c->table_stride);
    return PIPO_ERR_ARG;
  }
  if (v) {
    v->pool = static_cast<uint8_t*>(c->pool) + layer * c->layer_bytes;
    v->table = c->table;
    v->stride = c->table_stride;
    v->page_bytes = page;
    v->scales_at = (uint32_t)codes_bytes(c->page_size, c->n_kv_heads, c->head_dim);
    v->n_pages = c->n_pages;
    v->ps_log2 = __builtin_ctz((unsigned)c->page_size);
    v->Hkv = c->n_kv_heads;
    v->n_seq = c->n_seq;
  }
  return PIPO_OK;
}

static pipo_status check_rows8(const char* what, const pipo_kv8_pages* c, const void* p0,
                               const void* p1, const void* k, int64_t ldk, const void* v, int64_t ldv,
                               int64_t M) {
  const int64_t dkv = (int64_t)c->n_kv_heads * c->head_dim;
  if (!p0 || !p1 || !k || !v || M < 0 || ldk < dkv || ldv < dkv) {
    set_error("%s: NULL pointer, %lld rows, or rows (%lld, %lld) shorter than %lld", what,
              (long long)M, (long long)ldk, (long long)ldv, (long long)dkv);
    return PIPO_ERR_ARG;
  }
  if (M >= ((int64_t)1 << 31)) {
    set_error("%s: %lld rows", what, (long long)M);
    return PIPO_ERR_UNSUPPORTED;
  }
  return PIPO_OK;
}

static bool rows_aligned8(const void* k, int64_t ldk, const void* v, int64_t ldv) {
  return (reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) % 16 == 0 &&
         (ldk | ldv) % 8 == 0;
}

// blocks in rows of 2^22 (a launch takes under 2^32 threads in a dimension)
static dim3 grid_of(int64_t blocks) {
  const int64_t row = (int64_t)1 << 22;
  return dim3((unsigned)std::min(blocks, row), (unsigned)((blocks + row - 1) / row));
}

// fn(head_dim, whether INT8, whether rows are aligned) as constants
template <typename F>
static void pick8(int head_dim, bool int8, bool vec, F fn) {
  const auto with_vec = [&](auto d, auto f) {
    vec ? fn(d, f, std::true_type{}) : fn(d, f, std::false_type{});
  };
  const auto with_fmt = [&](auto d) {
    int8 ? with_vec(d, std::true_type{}) : with_vec(d, std::false_type{});
  };
  head_dim == 128 ? with_fmt(std::integral_constant<int, 128>{})
                  : with_fmt(std::integral_constant<int, 64>{});
}

}  // namespace pipo

using namespace pipo;

extern "C" {

int64_t pipo_kv8_page_bytes(int32_t page_size, int32_t n_kv_heads, int32_t head_dim) {
  if (page_size < 16 || page_size > 256 || (page_size & (page_size - 1)) != 0 || n_kv_heads < 1 ||
      (head_dim != 64 && head_dim != 128))
    return 0;
  const int64_t scales = (int64_t)n_kv_heads * page_size / 2;
  const int64_t n = codes_bytes(page_size, n_kv_heads, head_dim) + (scales + 127) / 128 * 128;
  return n < ((int64_t)1 << 31) ? n : 0;
}

pipo_status pipo_op_kv8_pages_append(const pipo_kv8_pages* c, int32_t layer, const int32_t* q_start,
                                     const int32_t* kv_len, const uint16_t* k, int64_t ldk,
                                     const uint16_t* v, int64_t ldv, int64_t M, void* stream) {
  clear_error();
  Rows8 a;
  PIPO_TRY(check_pages8("kv8_pages_append", c, layer, &a.c));
  PIPO_TRY(check_rows8("kv8_pages_append", c, q_start, kv_len, k, ldk, v, ldv, M));
  if (M == 0) return PIPO_OK;
  a.k = k;
  a.v = v;
  a.ldk = ldk;
  a.ldv = ldv;
  a.M = M;
  a.q_start = q_start;
  a.kv_len = kv_len;
  const int64_t blocks = (M / 16 + 2 * (int64_t)c->n_seq) * ((2 * (int64_t)c->n_kv_heads + 3) / 4);
  if (blocks >= ((int64_t)1 << 37)) {
    set_error("kv8_pages_append: %lld rows of %d heads", (long long)M, c->n_kv_heads);
    return PIPO_ERR_UNSUPPORTED;
  }
  pick8(c->head_dim, c->fmt == PIPO_KV8_INT8, rows_aligned8(k, ldk, v, ldv), [&](auto d, auto f, auto al) {
    launch(pages8_append_k<decltype(d)::value, decltype(f)::value, decltype(al)::value>, grid_of(blocks),
           dim3(256), 0, static_cast<hipStream_t>(stream), a);
  });
  PIPO_HIP_TRY(hipGetLastError());
  return PIPO_OK;
}

pipo_status pipo_op_kv8_pages_read(const pipo_kv8_pages* c, int32_t layer, const int32_t* seq,
                                   const int32_t* pos, uint16_t* k, int64_t ldk, uint16_t* v,
                                   int64_t ldv, int64_t M, void* stream) {
  clear_error();
  Pages8 view;
  PIPO_TRY(check_pages8("kv8_pages_read", c, layer, &view));
  PIPO_TRY(check_rows8("kv8_pages_read", c, seq, pos, k, ldk, v, ldv, M));
  if (M == 0) return PIPO_OK;
  const int64_t per_group = read_step(c->n_kv_heads) * (c->head_dim / 2), groups = (M + 15) / 16;
  const int64_t blocks = (groups * per_group + 255) / 256;
  if (per_group >= ((int64_t)1 << 31) || blocks >= ((int64_t)1 << 37)) {
    set_error("kv8_pages_read: %lld rows of %d heads", (long long)M, c->n_kv_heads);
    return PIPO_ERR_UNSUPPORTED;
  }
  pick8(c->head_dim, c->fmt == PIPO_KV8_INT8, rows_aligned8(k, ldk, v, ldv), [&](auto d, auto f, auto al) {
    launch(pages8_read_k<decltype(d)::value, decltype(f)::value, decltype(al)::value>, grid_of(blocks),
           dim3(256), 0, static_cast<hipStream_t>(stream), view, seq, pos, k, ldk, v, ldv, M);
  });
  PIPO_HIP_TRY(hipGetLastError());
  return PIPO_OK;
}

pipo_status pipo_op_kv8_pages_copy(const pipo_kv8_pages* c, const int32_t* pairs,
                                   const int32_t* n_pairs, int32_t max_pairs, void* stream) {
  clear_error();
  Pages8 view;
  PIPO_TRY(check_pages8("kv8_pages_copy", c, 0, &view));
  if (!pairs || !n_pairs || max_pairs < 0) {
    set_error("kv8_pages_copy: NULL pointer or %d pairs", max_pairs);
    return PIPO_ERR_ARG;
  }
  if (max_pairs == 0) return PIPO_OK;
  launch_pages_copy(view.pool, c->layer_bytes, view.page_bytes, c->n_layers, c->n_pages, pairs, n_pairs,
                    max_pairs, static_cast<hipStream_t>(stream));
  PIPO_HIP_TRY(hipGetLastError());
  return PIPO_OK;
}

}  // extern "C"
