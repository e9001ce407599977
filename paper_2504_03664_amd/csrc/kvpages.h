// Pages of a 4-bit KV cache (pipo_kv_pages in pipo_ops.h): addressing shared
// by the kernels that fill, read, move and attend to them.
//
// A page holds page_size positions of every key/value head, head after head,
// each head's positions in tiles of 16.  A tile is 18 D bytes: K codes (8 D),
// V codes (8 D), the 16 x D/64 (min, scale) pairs of K (D) and those of V (D).
// Codes lie as the matrix instructions take them, so that attention loads a
// tile straight into operand registers, a wave 16 D/16 contiguous bytes at a
// time, and never transposes:
//   K: byte (key + 16 g) D/8 + 4 kk + j is lane (key, g)'s: dimensions 32 kk +
//      8 g + 0..7 in a 32-bit word, dimension 2 i + h of them in nibble 4 h + i
//      (one shift, mask and or then gives two neighbours as halves);
//   V: byte (r + 16 g) D/8 + 4 w + i is lane (r, g)'s: key 4 g + i, dimension
//      32 w + r in the low nibble and 32 w + 16 + r in the high one.  A byte
//      belongs to one key, so rows are written without reading their neighbours.
// A pair word has the scale in its high half: words order as scales do.
#pragma once

#include "common.h"
#include "device.h"

namespace pipo {

constexpr int kTileKeys = 16;
constexpr float kKvClamp = 57344.f;  // of an element before it is quantized: code * scale +
                                     // min then stays below the largest fp16 (57376 at most)

// one layer of a pipo_kv_pages as kernels take it
struct PagesView {
  uint8_t* pool;
  const int32_t* table;
  int64_t stride;      // of the table's rows
  int64_t page_bytes;
  int n_pages, ps_log2, Hkv, n_seq;
};

template <int D>
constexpr int kTileBytes = 18 * D;

// (32-bit: a page has at most 2^31 bytes)
template <int D>
__device__ __forceinline__ const uint8_t* tile_at(const PagesView& v, int page, int head, int pos) {
  const int tiles = 1 << (v.ps_log2 - 4);
  return v.pool + (int64_t)page * v.page_bytes +
         (uint32_t)((head << (v.ps_log2 - 4)) + ((pos >> 4) & (tiles - 1))) * kTileBytes<D>;
}

// whole pages of every layer, of any format (pages of a multiple of 16 bytes)
void launch_pages_copy(uint8_t* pool, int64_t layer_bytes, int64_t page_bytes, int n_layers,
                       int n_pages, const int32_t* pairs, const int32_t* n_pairs, int max_pairs,
                       hipStream_t st);

pipo_status check_pages(const char* what, const pipo_kv_pages* c, int32_t layer, PagesView* v);

}  // namespace pipo
