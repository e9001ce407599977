// Rows into and out of the pages of a 4-bit KV cache, and copies of pages
// (layout in kvpages.h; pipo_kv_pages in pipo_ops.h).
//
//   pages_append_k: fp16 rows -> their slots, with the recipe of kv_quant_k
//                   (kvquant.h) on elements clamped to +-kKvClamp (NaN: 0).
//   pages_read_k:   slots -> fp16 rows, code * scale + min rounded once.
//   pages_copy_k:   whole pages of every layer.
// D/8 lanes hold one head's key (or value) of a row, eight elements each; the
// lanes of one head in four rows follow each other, so that prompts, whose rows
// are consecutive positions, write whole words of four keys' codes and 64 bytes
// at a time.  Bound by HBM for prompts, by the launch for a decode step.
#include "kvpages.h"

#include <algorithm>

#include "kvquant.h"

namespace pipo {

// the head's key or value that this thread works at; false past the end or
// where the row has no slot.  (All lanes of a head agree.)
struct Slot {
  int64_t m;
  int head, x, key;   // x: eight-element piece
  bool value;
  int seq, pos;
  const uint8_t* tile;
};
template <int D>
__device__ __forceinline__ bool slot_of(const PagesView& c, const int32_t* seq, const int32_t* pos,
                                        int64_t M, Slot& s) {
  constexpr int LANES = D / 8;
  const uint32_t per_quad = (uint32_t)c.Hkv * 2 * 4 * LANES;  // of four rows
  const int64_t e = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 256 + threadIdx.x;
  const int64_t quads = (M + 3) / 4;
  if (e >= quads * per_quad) return false;
  uint32_t r;
  if (quads * per_quad < ((int64_t)1 << 32)) {
    const uint32_t quad = (uint32_t)e / per_quad;
    s.m = 4 * (int64_t)quad;
    r = (uint32_t)e - quad * per_quad;
  } else {
    s.m = e / per_quad;
    r = (uint32_t)(e - s.m * per_quad);
    s.m *= 4;
  }
  s.x = r % LANES;
  s.m += r / LANES % 4;
  // value heads behind key heads, as a fused projection's rows have them
  s.head = r / LANES / 4;
  s.value = s.head >= c.Hkv;
  if (s.value) s.head -= c.Hkv;
  if (s.m >= M) return false;
  const int i = seq[s.m], p = pos[s.m];
  if (i < 0 || i >= c.n_seq || p < 0 || (p >> c.ps_log2) >= c.stride) return false;
  const int page = c.table[i * c.stride + (p >> c.ps_log2)];
  if (page < 0 || page >= c.n_pages) return false;
  s.seq = i;
  s.pos = p;
  s.key = p & (kTileKeys - 1);
  s.tile = tile_at<D>(c, page, s.head, p);
  return true;
}

template <int D, bool VEC>
__global__ __launch_bounds__(256) void pages_append_k(PagesView c, const int32_t* __restrict__ seq,
                                                      const int32_t* __restrict__ pos,
                                                      const uint16_t* __restrict__ k, int64_t ldk,
                                                      const uint16_t* __restrict__ v, int64_t ldv,
                                                      int64_t M) {
  constexpr int LANES = D / 8;
  Slot s;
  const bool ok = slot_of<D>(c, seq, pos, M, s);
  // whether the four rows of these 4 LANES lanes are the four keys of a word: each
  // finds its own place counted from the first's
  const int k4 = threadIdx.x / LANES % 4, first = (threadIdx.x & 63) - k4 * LANES;
  const int at0 = ok ? s.pos - k4 : -1;
  const uint64_t fit = __ballot(ok && at0 % 4 == 0 && at0 == __shfl(at0, first, 64) &&
                                s.seq == __shfl(ok ? s.seq : -1, first, 64));
  const uint64_t mask = LANES == 16 ? ~0ull : 0xFFFFFFFFull << (threadIdx.x & 32);
  const bool whole = (fit & mask) == mask;
  if (!ok) return;
  const uint16_t* src = (s.value ? v + s.m * ldv : k + s.m * ldk) + s.head * D + 8 * s.x;
  float f[8];
  if constexpr (VEC) {
    const h8 h = load_h8(src);
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = (float)h[j];
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = h2f(src[j]);
  }
#pragma unroll
  for (int j = 0; j < 8; ++j)
    f[j] = f[j] == f[j] ? fminf(fmaxf(f[j], -kKvClamp), kKvClamp) : 0.f;
  const Quant8 q = quantize8(f);
  uint8_t* tile = const_cast<uint8_t*>(s.tile);
  if (!s.value) {
    uint32_t w = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) w |= q.c[j] << (4 * (4 * (j & 1) + j / 2));
    *reinterpret_cast<uint32_t*>(tile + (s.key + 16 * (s.x & 3)) * (D / 8) + 4 * (s.x >> 2)) = w;
  } else {
    // dimensions 16 apart share a byte: lanes x and x ^ 2 exchange their codes
    // and write four of the eight bytes each
    uint32_t w = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) w |= q.c[j] << (4 * j);
    const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)w, 0x4E, 0xF, 0xF, false);
    const bool high = s.x & 2;
    const uint32_t lo = high ? o >> 16 : w, hi = high ? w >> 16 : o;
    uint8_t* at = tile + 8 * D + (8 * (s.x & 1) + (high ? 4 : 0) + 16 * (s.key >> 2)) * (D / 8) +
                  4 * (s.x >> 2);
    uint32_t b = 0;  // byte j: of the j-th of the four
#pragma unroll
    for (int j = 0; j < 4; ++j)
      b |= (((lo >> (4 * j)) & 15) | (((hi >> (4 * j)) & 15) << 4)) << (8 * j);
    if (whole) {
      // the four rows' bytes transposed: the lane of key k writes the word of the
      // k-th, first by pairs of keys, then by halves
      const uint32_t o1 = (uint32_t)__shfl_xor((int)b, LANES, 64);
      b = k4 & 1 ? __builtin_amdgcn_perm(b, o1, 0x07030501u) : __builtin_amdgcn_perm(o1, b, 0x06020400u);
      const uint32_t o2 = (uint32_t)__shfl_xor((int)b, 2 * LANES, 64);
      b = k4 & 2 ? __builtin_amdgcn_perm(b, o2, 0x07060302u) : __builtin_amdgcn_perm(o2, b, 0x05040100u);
      *reinterpret_cast<uint32_t*>(at + k4 * (D / 8)) = b;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) at[j * (D / 8) + (s.key & 3)] = (uint8_t)(b >> (8 * j));
    }
  }
  if (s.x % 8 == 0)
    *reinterpret_cast<uint32_t*>(tile + (s.value ? 17 : 16) * D + s.key * (D / 16) + s.x / 8 * 4) =
        (uint32_t)q.min | ((uint32_t)q.scale << 16);
}

template <int D, bool VEC>
__global__ __launch_bounds__(256) void pages_read_k(PagesView c, const int32_t* __restrict__ seq,
                                                    const int32_t* __restrict__ pos,
                                                    uint16_t* __restrict__ k, int64_t ldk,
                                                    uint16_t* __restrict__ v, int64_t ldv,
                                                    int64_t M) {
  Slot s;
  if (!slot_of<D>(c, seq, pos, M, s)) return;
  const uint32_t pair = *reinterpret_cast<const uint32_t*>(
      s.tile + (s.value ? 17 : 16) * D + s.key * (D / 16) + s.x / 8 * 4);
  const float mn = h2f((uint16_t)pair), sc = h2f((uint16_t)(pair >> 16));
  uint32_t code[8];
  if (!s.value) {
    const uint32_t w = *reinterpret_cast<const uint32_t*>(
        s.tile + (s.key + 16 * (s.x & 3)) * (D / 8) + 4 * (s.x >> 2));
#pragma unroll
    for (int j = 0; j < 8; ++j) code[j] = (w >> (4 * (4 * (j & 1) + j / 2))) & 15;
  } else {
    const uint8_t* at = s.tile + 8 * D + (8 * (s.x & 1) + 16 * (s.key >> 2)) * (D / 8) +
                        4 * (s.x >> 2) + (s.key & 3);
    const int shift = s.x & 2 ? 4 : 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) code[j] = (at[j * (D / 8)] >> shift) & 15;
  }
  uint16_t* dst = (s.value ? v + s.m * ldv : k + s.m * ldk) + s.head * D + 8 * s.x;
  u32x4 h;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    h[j] = (uint32_t)f2h(__builtin_fmaf((float)code[2 * j], sc, mn)) |
           ((uint32_t)f2h(__builtin_fmaf((float)code[2 * j + 1], sc, mn)) << 16);
  if constexpr (VEC) {
    *reinterpret_cast<u32x4*>(dst) = h;
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) dst[j] = (uint16_t)(h[j / 2] >> (16 * (j & 1)));
  }
}

// page pairs[i][0] onto page pairs[i][1], i < *n_pairs, in every layer; work
// items of 16 KiB taken in turn by a fixed grid, since the host does not know
// how many pairs there are
constexpr int kCopyBytes = 16384;
__global__ __launch_bounds__(256) void pages_copy_k(uint8_t* pool, int64_t layer_bytes,
                                                    int64_t page_bytes, int n_layers, int n_pages,
                                                    const int32_t* __restrict__ pairs,
                                                    const int32_t* __restrict__ n_pairs,
                                                    int max_pairs) {
  const int n = min(max(*n_pairs, 0), max_pairs);
  const int pieces = (int)((page_bytes + kCopyBytes - 1) / kCopyBytes);
  const int64_t items = (int64_t)n * n_layers * pieces;
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int piece = (int)(it % pieces);
    const int64_t r = it / pieces;
    const int layer = (int)(r % n_layers), i = (int)(r / n_layers);
    const int src = pairs[2 * i], dst = pairs[2 * i + 1];
    if (src < 0 || src >= n_pages || dst < 0 || dst >= n_pages || src == dst) continue;
    const uint8_t* a = pool + layer * layer_bytes + src * page_bytes;
    uint8_t* b = pool + layer * layer_bytes + dst * page_bytes;
    u32x4 x[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t at = (int64_t)piece * kCopyBytes + j * 4096 + threadIdx.x * 16;
      if (at < page_bytes) x[j] = *reinterpret_cast<const u32x4*>(a + at);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t at = (int64_t)piece * kCopyBytes + j * 4096 + threadIdx.x * 16;
      if (at < page_bytes) *reinterpret_cast<u32x4*>(b + at) = x[j];
    }
  }
}

pipo_status check_pages(const char* what, const pipo_kv_pages* c, int32_t layer, PagesView* v) {
  if (!c || !c->pool || !c->table || reinterpret_cast<uintptr_t>(c->pool) % 16 != 0) {
    set_error("%s: NULL cache, pool or table, or a pool off 16-byte alignment", what);
    return PIPO_ERR_ARG;
  }
  const int64_t page = pipo_kv_page_bytes(c->page_size, c->n_kv_heads, c->head_dim);
  if (page == 0) {
    set_error("%s: pages of %d positions of %d heads of %d not supported (16, 32, 64, 128 or 256 "
              "positions, heads of 64 or 128, under 2^31 bytes)", what, c->page_size,
              c->n_kv_heads, c->head_dim);
    return PIPO_ERR_UNSUPPORTED;
  }
  if (c->n_pages < 1 || c->n_layers < 1 || layer < 0 || layer >= c->n_layers || c->n_seq < 1 ||
      c->table_stride < 1 || c->layer_bytes % 16 != 0 || c->layer_bytes < c->n_pages * page) {
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
    v->n_pages = c->n_pages;
    v->ps_log2 = __builtin_ctz((unsigned)c->page_size);
    v->Hkv = c->n_kv_heads;
    v->n_seq = c->n_seq;
  }
  return PIPO_OK;
}

static pipo_status check_rows(const char* what, const pipo_kv_pages* c, const int32_t* seq,
                              const int32_t* pos, const void* k, int64_t ldk, const void* v,
                              int64_t ldv, int64_t M) {
  const int64_t dkv = (int64_t)c->n_kv_heads * c->head_dim;
  if (!seq || !pos || !k || !v || M < 0 || ldk < dkv || ldv < dkv) {
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

// a thread per 8 elements of four rows at a time, in rows of 2^22 blocks (a launch
// takes under 2^32 threads in a dimension)
static dim3 rows_grid(const PagesView& c, int D, int64_t M) {
  const int64_t blocks = ((M + 3) / 4 * 4 * c.Hkv * 2 * (D / 8) + 255) / 256, row = (int64_t)1 << 22;
  return dim3((unsigned)std::min(blocks, row), (unsigned)((blocks + row - 1) / row));
}

static bool rows_aligned(const void* k, int64_t ldk, const void* v, int64_t ldv) {
  return (reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) % 16 == 0 &&
         (ldk | ldv) % 8 == 0;
}

}  // namespace pipo

using namespace pipo;

extern "C" {

int64_t pipo_kv_page_bytes(int32_t page_size, int32_t n_kv_heads, int32_t head_dim) {
  if (page_size < 16 || page_size > 256 || (page_size & (page_size - 1)) != 0 || n_kv_heads < 1 ||
      (head_dim != 64 && head_dim != 128))
    return 0;
  const int64_t n = (int64_t)n_kv_heads * page_size * (head_dim + head_dim / 8);
  return n < ((int64_t)1 << 31) ? n : 0;
}

pipo_status pipo_op_kv_pages_append(const pipo_kv_pages* c, int32_t layer, const int32_t* seq,
                                    const int32_t* pos, const uint16_t* k, int64_t ldk,
                                    const uint16_t* v, int64_t ldv, int64_t M, void* stream) {
  clear_error();
  PagesView view;
  PIPO_TRY(check_pages("kv_pages_append", c, layer, &view));
  PIPO_TRY(check_rows("kv_pages_append", c, seq, pos, k, ldk, v, ldv, M));
  if (M == 0) return PIPO_OK;
  const auto go = [&](auto kernel) {
    launch(kernel, rows_grid(view, c->head_dim, M), dim3(256), 0, static_cast<hipStream_t>(stream),
           view, seq, pos, k, ldk, v, ldv, M);
  };
  const bool vec = rows_aligned(k, ldk, v, ldv);
  if (c->head_dim == 128)
    vec ? go(pages_append_k<128, true>) : go(pages_append_k<128, false>);
  else
    vec ? go(pages_append_k<64, true>) : go(pages_append_k<64, false>);
  PIPO_HIP_TRY(hipGetLastError());
  return PIPO_OK;
}

pipo_status pipo_op_kv_pages_read(const pipo_kv_pages* c, int32_t layer, const int32_t* seq,
                                  const int32_t* pos, uint16_t* k, int64_t ldk, uint16_t* v,
                                  int64_t ldv, int64_t M, void* stream) {
  clear_error();
  PagesView view;
  PIPO_TRY(check_pages("kv_pages_read", c, layer, &view));
  PIPO_TRY(check_rows("kv_pages_read", c, seq, pos, k, ldk, v, ldv, M));
  if (M == 0) return PIPO_OK;
  const auto go = [&](auto kernel) {
    launch(kernel, rows_grid(view, c->head_dim, M), dim3(256), 0, static_cast<hipStream_t>(stream),
           view, seq, pos, k, ldk, v, ldv, M);
  };
  const bool vec = rows_aligned(k, ldk, v, ldv);
  if (c->head_dim == 128)
    vec ? go(pages_read_k<128, true>) : go(pages_read_k<128, false>);
  else
    vec ? go(pages_read_k<64, true>) : go(pages_read_k<64, false>);
  PIPO_HIP_TRY(hipGetLastError());
  return PIPO_OK;
}

pipo_status pipo_op_kv_pages_copy(const pipo_kv_pages* c, const int32_t* pairs,
                                  const int32_t* n_pairs, int32_t max_pairs, void* stream) {
  clear_error();
  PagesView view;
  PIPO_TRY(check_pages("kv_pages_copy", c, 0, &view));
  if (!pairs || !n_pairs || max_pairs < 0) {
    set_error("kv_pages_copy: NULL pointer or %d pairs", max_pairs);
    return PIPO_ERR_ARG;
  }
  if (max_pairs == 0) return PIPO_OK;
  const int64_t pieces = (view.page_bytes + kCopyBytes - 1) / kCopyBytes;
  const int64_t items = (int64_t)max_pairs * c->n_layers * pieces;
  launch(pages_copy_k, dim3((unsigned)std::min<int64_t>(items, 2048)), dim3(256), 0,
         static_cast<hipStream_t>(stream), view.pool, c->layer_bytes, view.page_bytes, c->n_layers,
         c->n_pages, pairs, n_pairs, max_pairs);
  PIPO_HIP_TRY(hipGetLastError());
  return PIPO_OK;
}

}  // extern "C"
