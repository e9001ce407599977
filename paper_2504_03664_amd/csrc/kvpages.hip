// Rows into and out of the pages of a 4-bit KV cache, and copies of pages
// (layout in kvpages.h; pipo_kv_pages in pipo_ops.h).
//
//   pages_append_k: fp16 rows -> their slots, with the recipe of kv_quant_k
//                   (kvquant.h) on elements clamped to +-kKvClamp (NaN: 0).
//   pages_read_k:   slots -> fp16 rows, code * scale + min rounded once.
//   pages_copy_k:   whole pages of every layer.
// D/8 lanes hold one head's key (or value) of a row, eight elements each; the
// lanes of one head in sixteen rows follow each other, so that prompts, whose rows
// are consecutive positions, write whole words of four keys' codes, and a tile's
// lines from one workgroup.  For prompts append is bound by the quantizer's arithmetic
// (4096 rows of 56 heads of 128: vector instructions issue in 76 % of the cycles), read
// by HBM (150 MB in 28 us, vector instructions in 65 %); for a decode step both by the
// launch.
#include "kvpages.h"

#include <algorithm>
#include <type_traits>

#include "kvquant.h"

namespace pipo {

// The row that this thread works at, and its slot.  HEADS: of the 2 Hkv heads (values
// behind keys, as a fused projection's rows have them) a thread takes h0, h0 + step,
// .., so that one look at the table serves several.
struct Slot {
  int64_t m;      // (>= M: none)
  int x, h0;      // eight-element piece, first head
  int seq, pos;   // -1: no slot
  const uint8_t* tile;  // of head 0
};
template <int D, int HEADS>
__device__ __forceinline__ uint32_t head_step(const PagesView& c) {
  return (2 * c.Hkv + HEADS - 1) / HEADS;
}
template <int D, int HEADS>
__device__ __forceinline__ void row_of(const PagesView& c, int64_t M, Slot& s) {
  constexpr int LANES = D / 8;
  const uint32_t per_group = head_step<D, HEADS>(c) * kTileKeys * LANES;  // of sixteen rows
  const int64_t e = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 256 + threadIdx.x;
  uint32_t r;
  if ((M + kTileKeys - 1) / kTileKeys * per_group < ((int64_t)1 << 31)) {
    const uint32_t group = (uint32_t)e / per_group;
    s.m = kTileKeys * (int64_t)group;
    r = (uint32_t)e - group * per_group;
  } else {
    s.m = e / per_group;
    r = (uint32_t)(e - s.m * per_group);
    s.m *= kTileKeys;
  }
  s.x = r % LANES;
  s.m += r / LANES % kTileKeys;
  s.h0 = r / LANES / kTileKeys;
}
template <int D>
__device__ __forceinline__ void slot_of(const PagesView& c, const int32_t* seq, const int32_t* pos,
                                        int64_t M, Slot& s) {
  s.seq = s.pos = -1;
  if (s.m >= M) return;
  const int i = seq[s.m], p = pos[s.m];
  if (i < 0 || i >= c.n_seq || p < 0 || (p >> c.ps_log2) >= c.stride) return;
  const int page = c.table[i * c.stride + (p >> c.ps_log2)];
  if (page < 0 || page >= c.n_pages) return;
  s.seq = i;
  s.pos = p;
  s.tile = tile_at<D>(c, page, 0, p);
}
// bytes from a head's tile to the next head's
template <int D>
__device__ __forceinline__ uint32_t head_bytes(const PagesView& c) {
  return kTileBytes<D> << (c.ps_log2 - 4);
}

// elements to +-kKvClamp, NaN to 0; hardly ever needed, so one test of the largest
// magnitude's bits decides for the wave
__device__ __forceinline__ void clamp8(h8& x) {
  typedef uint16_t us2 __attribute__((ext_vector_type(2)));
  constexpr uint32_t kLimit = 0x7B00;  // kKvClamp's bits
  const u32x4 w = __builtin_bit_cast(u32x4, x);
  us2 top = __builtin_bit_cast(us2, w[0] & 0x7FFF7FFFu);
#pragma unroll
  for (int j = 1; j < 4; ++j)
    top = __builtin_elementwise_max(top, __builtin_bit_cast(us2, w[j] & 0x7FFF7FFFu));
  if (!__any(top[0] > kLimit || top[1] > kLimit)) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float f = (float)x[j];
    x[j] = (_Float16)(f == f ? fminf(fmaxf(f, -kKvClamp), kKvClamp) : 0.f);
  }
}
// (in assembly: the compiler would quiet every operand first)
__device__ __forceinline__ h2 pk_max(h2 a, h2 b) {
  h2 d;
  asm("v_pk_max_f16 %0, %1, %2" : "=v"(d) : "v"(a), "v"(b));
  return d;
}
template <int CTRL>
__device__ __forceinline__ h2 pk_move(h2 v) {
  return __builtin_bit_cast(h2, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}
// largest and least of the group's 64 finite halves, eight lanes of eight: both at
// once, the least as the largest of the negated
__device__ __forceinline__ void group_range(h8 x, float& least, float& most) {
  const u32x4 w = __builtin_bit_cast(u32x4, x), n = w ^ 0x80008000u;
  h2 p[4], q[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t y = w[j], z = n[j];
    p[j] = __builtin_bit_cast(h2, y);
    q[j] = __builtin_bit_cast(h2, z);
  }
  const h2 a = pk_max(pk_max(p[0], p[1]), pk_max(p[2], p[3]));
  const h2 b = pk_max(pk_max(q[0], q[1]), pk_max(q[2], q[3]));
  h2 m = pk_max(h2{a[0], b[0]}, h2{a[1], b[1]});
  m = pk_max(m, pk_move<0xB1>(m));
  m = pk_max(m, pk_move<0x4E>(m));
  m = pk_max(m, pk_move<0x141>(m));
  most = (float)m[0];
  least = -(float)m[1];
}

template <int D, bool VEC, int HEADS>
__global__ __launch_bounds__(256) void pages_append_k(PagesView c, const int32_t* __restrict__ seq,
                                                      const int32_t* __restrict__ pos,
                                                      const uint16_t* __restrict__ k, int64_t ldk,
                                                      const uint16_t* __restrict__ v, int64_t ldv,
                                                      int64_t M) {
  constexpr int LANES = D / 8;
  Slot s;
  row_of<D, HEADS>(c, M, s);
  const int step = head_step<D, HEADS>(c);
  h8 in[HEADS];
#pragma unroll
  for (int t = 0; t < HEADS; ++t) {
    const int h = s.h0 + t * step;
    if (s.m >= M || h >= 2 * c.Hkv) continue;
    const uint16_t* src =
        (h < c.Hkv ? k + s.m * ldk + h * D : v + s.m * ldv + (h - c.Hkv) * D) + 8 * s.x;
    if constexpr (VEC) {
      in[t] = load_h8(src);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) in[t][j] = __builtin_bit_cast(_Float16, src[j]);
    }
  }
  slot_of<D>(c, seq, pos, M, s);
  // whether the four rows of these 4 LANES lanes are the four keys of a word: each
  // finds its own place counted from the first's
  const int k4 = threadIdx.x / LANES % 4, first = (threadIdx.x & 63) - k4 * LANES;
  const int at0 = s.seq >= 0 ? s.pos - k4 : -1;
  const uint64_t fit = __ballot(s.seq >= 0 && at0 % 4 == 0 && at0 == __shfl(at0, first, 64) &&
                                s.seq == __shfl(s.seq, first, 64));
  const uint64_t mask = LANES == 16 ? ~0ull : 0xFFFFFFFFull << (threadIdx.x & 32);
  const bool whole = (fit & mask) == mask;
  if (s.seq < 0) return;
  const int key = s.pos & (kTileKeys - 1);
#pragma unroll
  for (int t = 0; t < HEADS; ++t) {
    const int h = s.h0 + t * step;
    if (h >= 2 * c.Hkv) break;  // (all lanes of a row's head agree, and the four rows')
    const bool value = h >= c.Hkv;
    uint8_t* tile = const_cast<uint8_t*>(s.tile) + (uint32_t)(value ? h - c.Hkv : h) * head_bytes<D>(c);
    clamp8(in[t]);
    float least, most, f[8];
    group_range(in[t], least, most);
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = (float)in[t][j];
    const Quant8 q = quantize8<true>(f, least, most);
    if (!value) {
      *reinterpret_cast<uint32_t*>(tile + (key + 16 * (s.x & 3)) * (D / 8) + 4 * (s.x >> 2)) =
          pack8(q, [](int j) { return 4 * (j & 1) + j / 2; });
    } else {
      // dimensions 16 apart share a byte: lanes x and x ^ 2 exchange their codes
      // and write four of the eight bytes each
      const uint32_t w = pack8(q, [](int j) { return j; });
      const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)w, 0x4E, 0xF, 0xF, false);
      const bool high = s.x & 2;
      const uint32_t lo = high ? o >> 16 : w, hi = high ? w >> 16 : o;
      uint8_t* at = tile + 8 * D + (8 * (s.x & 1) + (high ? 4 : 0) + 16 * (key >> 2)) * (D / 8) +
                    4 * (s.x >> 2);
      // byte j: of the j-th of the four (the nibbles of 16 bits spread over 32)
      const auto spread = [](uint32_t y) {
        y = (y & 0xFFu) | (y << 8 & 0xFF0000u);
        return (y & 0x000F000Fu) | (y << 4 & 0x0F000F00u);
      };
      uint32_t b = spread(lo) | spread(hi) << 4;
      if (whole) {
        // the four rows' bytes transposed: the lane of key k writes the word of the
        // k-th, first by pairs of keys, then by halves
        const uint32_t o1 = (uint32_t)__shfl_xor((int)b, LANES, 64);
        b = k4 & 1 ? __builtin_amdgcn_perm(b, o1, 0x07030501u)
                   : __builtin_amdgcn_perm(o1, b, 0x06020400u);
        const uint32_t o2 = (uint32_t)__shfl_xor((int)b, 2 * LANES, 64);
        b = k4 & 2 ? __builtin_amdgcn_perm(b, o2, 0x07060302u)
                   : __builtin_amdgcn_perm(o2, b, 0x05040100u);
        *reinterpret_cast<uint32_t*>(at + k4 * (D / 8)) = b;
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) at[j * (D / 8) + (key & 3)] = (uint8_t)(b >> (8 * j));
      }
    }
    if (s.x % 8 == 0)
      *reinterpret_cast<uint32_t*>(tile + (value ? 17 : 16) * D + key * (D / 16) + s.x / 8 * 4) =
          (uint32_t)q.min | ((uint32_t)q.scale << 16);
  }
}

template <int D, bool VEC, int HEADS>
__global__ __launch_bounds__(256) void pages_read_k(PagesView c, const int32_t* __restrict__ seq,
                                                    const int32_t* __restrict__ pos,
                                                    uint16_t* __restrict__ k, int64_t ldk,
                                                    uint16_t* __restrict__ v, int64_t ldv,
                                                    int64_t M) {
  Slot s;
  row_of<D, HEADS>(c, M, s);
  slot_of<D>(c, seq, pos, M, s);
  if (s.seq < 0) return;
  const int key = s.pos & (kTileKeys - 1), step = head_step<D, HEADS>(c);
  uint32_t pair[HEADS], w[HEADS][8];  // of a key one word, of a value its eight bytes
#pragma unroll
  for (int t = 0; t < HEADS; ++t) {
    const int h = s.h0 + t * step;
    if (h >= 2 * c.Hkv) break;
    const bool value = h >= c.Hkv;
    const uint8_t* tile = s.tile + (uint32_t)(value ? h - c.Hkv : h) * head_bytes<D>(c);
    pair[t] = *reinterpret_cast<const uint32_t*>(tile + (value ? 17 : 16) * D + key * (D / 16) +
                                                 s.x / 8 * 4);
    if (!value) {
      w[t][0] = *reinterpret_cast<const uint32_t*>(tile + (key + 16 * (s.x & 3)) * (D / 8) +
                                                   4 * (s.x >> 2));
    } else {
      const uint8_t* at =
          tile + 8 * D + (8 * (s.x & 1) + 16 * (key >> 2)) * (D / 8) + 4 * (s.x >> 2) + (key & 3);
#pragma unroll
      for (int j = 0; j < 8; ++j) w[t][j] = at[j * (D / 8)];
    }
  }
#pragma unroll
  for (int t = 0; t < HEADS; ++t) {
    const int h = s.h0 + t * step;
    if (h >= 2 * c.Hkv) break;
    const bool value = h >= c.Hkv;
    const float mn = h2f((uint16_t)pair[t]), sc = h2f((uint16_t)(pair[t] >> 16));
    uint16_t* dst =
        (value ? v + s.m * ldv + (h - c.Hkv) * D : k + s.m * ldk + h * D) + 8 * s.x;
    u32x4 o;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float y[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t code = value ? w[t][2 * j + i] >> (s.x & 2 ? 4 : 0) : w[t][0] >> (4 * (4 * i + j));
        y[i] = __builtin_fmaf((float)(code & 15), sc, mn);
      }
      o[j] = (uint32_t)f2h(y[0]) | ((uint32_t)f2h(y[1]) << 16);
    }
    if constexpr (VEC) {
      if constexpr (HEADS > 1)  // (many rows: past the L2, 30 -> 27 us)
        __builtin_nontemporal_store(o, reinterpret_cast<u32x4*>(dst));
      else
        *reinterpret_cast<u32x4*>(dst) = o;
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) dst[j] = (uint16_t)(o[j / 2] >> (16 * (j & 1)));
    }
  }
}

// page pairs[i][0] onto page pairs[i][1], i < *n_pairs, in every layer; work
// items of 16 KiB taken in turn by a fixed grid, since the host does not know
// how many pairs there are.  Stores go past the L2, of a few pages too: 45 MB of pages
// take 18.5 us, 23 with ordinary stores, and 28 MB 7.4 and 8.5; with the attention that
// reads the copies next 28 MB take 62.8 and 62.2, 7 MB 19.0 and 19.2.
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
      if (at < page_bytes) __builtin_nontemporal_store(x[j], reinterpret_cast<u32x4*>(b + at));
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

// Sixteen rows at a time, D/8 threads for a head of each, in rows of 2^22 blocks (a
// launch takes under 2^32 threads in a dimension).  Four heads a thread where that
// leaves the chip full, eight blocks a CU (4096 rows of 56 heads: append 68 -> 59
// us, read 43 -> 32, now 47 and 28).
constexpr int kRowHeads = 4;
static bool many_rows(const PagesView& c, int D, int64_t M) {
  return M * 2 * c.Hkv * (D / 8) >= (int64_t)kRowHeads * 256 * 8 * 256;
}
static dim3 rows_grid(const PagesView& c, int D, int64_t M) {
  const int heads = many_rows(c, D, M) ? kRowHeads : 1;
  const int64_t units =
      (M + kTileKeys - 1) / kTileKeys * kTileKeys * ((2 * c.Hkv + heads - 1) / heads);
  const int64_t blocks = (units * (D / 8) + 255) / 256, row = (int64_t)1 << 22;
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
  const auto pick = [&](auto d) {
    constexpr int D = decltype(d)::value;
    if (many_rows(view, D, M))
      vec ? go(pages_append_k<D, true, kRowHeads>) : go(pages_append_k<D, false, kRowHeads>);
    else
      vec ? go(pages_append_k<D, true, 1>) : go(pages_append_k<D, false, 1>);
  };
  if (c->head_dim == 128)
    pick(std::integral_constant<int, 128>{});
  else
    pick(std::integral_constant<int, 64>{});
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
  const auto pick = [&](auto d) {
    constexpr int D = decltype(d)::value;
    if (many_rows(view, D, M))
      vec ? go(pages_read_k<D, true, kRowHeads>) : go(pages_read_k<D, false, kRowHeads>);
    else
      vec ? go(pages_read_k<D, true, 1>) : go(pages_read_k<D, false, 1>);
  };
  if (c->head_dim == 128)
    pick(std::integral_constant<int, 128>{});
  else
    pick(std::integral_constant<int, 64>{});
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
