// Attention over the pages of a 4-bit KV cache (layout in kvpages.h): sequences
// of different lengths, from one query each to whole pieces of a prompt.
//
// The G query heads of a key/value head times a sequence's queries are columns
// (column c: query c / G, head c % G), 16 to a matrix product.  With a group's
// K = c s + m (c: codes, 0..15) a score is
//   q . k = sum over groups g of s_g (q_g . c_g) + m_g sum(q_g),
// and the output, with p the softmax weights,
//   o = sum over keys of (p s_g) c_g + p m_g,
// so the matrix products run on codes, which are exact as halves, and scale and
// min enter in fp32 per key and column.  That costs four multiply-adds a score
// where expanding the cache to halves costs four a key and eight dimensions
// and rounds every key and value.
#include <algorithm>
#include <type_traits>

#include "attention_common.h"
#include "kvpages.h"

namespace pipo {

struct AttnPages {
  PagesView c;
  const uint16_t* q;
  uint16_t* o;
  const int32_t *q_start, *kv_len;
  float* part;      // [row][head][split][D] sums and, behind them, their (R, l)
  float2* part_rl;
  int64_t ldq, ldo, M;
  int H, G, max_q, max_len;
  int few_cols;               // up to this many are attn_pages_few_k's, or none
  int chunk_few, chunk_many;  // keys of a split, by the sequence's columns
  int splits;                 // of a row's partials in `part`
  bool q_vec, o_vec;          // q rows 16-byte aligned, o rows 8-byte
};

// Up to this many columns a sequence is attn_pages_few_k's, above it
// attn_pages_many_k's; all of them where every row of the call may be one of
// max_q equal shares, which saves a launch.
constexpr int kFewCols = 64;
constexpr int kPackCols = 8;  // columns with which 64 keys at a time can be taken
constexpr int kCentreBlocks = 32;  // after which attn_pages_few_k centres its sums
constexpr int kMaxSplits = 64;  // a wave's lanes, in attn_pages_merge_k
constexpr float kLog2e = 1.4426950408889634f;
// p is held times 2^15 / (a bound of the block's value scales), so that p s fits a
// half with 29 bits of range below the largest (where the scales of a block's keys and
// groups are far apart, the smaller ones' have what is left of them: 11 at 2^18)
constexpr float kPBits = 15.f;

// a sequence's rows [row0, row0 + nq), how many of them count (up to max_q), and
// keys
struct Seq {
  int row0, nq, rows, len;
};
__device__ __forceinline__ Seq sequence(const AttnPages& a, int i) {
  Seq s;
  const int64_t r0 = min(max((int64_t)a.q_start[i], (int64_t)0), a.M);
  const int64_t r1 = min(max((int64_t)a.q_start[i + 1], r0), a.M);
  s.row0 = (int)r0;
  s.nq = (int)(r1 - r0);
  s.rows = min(s.nq, a.max_q);
  s.len = min(max(a.kv_len[i], 0), a.max_len);
  return s;
}

template <int D>
__device__ __forceinline__ h8 load_q(const AttnPages& a, int64_t row, int head, int dim) {
  const uint16_t* p = a.q + row * a.ldq + (int64_t)head * D + dim;
  if (a.q_vec) return load_h8(p);
  h8 v;
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = __builtin_bit_cast(_Float16, p[j]);
  return v;
}

// codes under exponents that place them at their value: nibble bits 2..5 of a
// half are 256 + c, bits 6..9 are 16 + c
struct Magic {
  uint32_t e256, e16, m256, m16;
};
__device__ __forceinline__ Magic magic() {
  return Magic{vgpr_const(0x5C005C00u), vgpr_const(0x4C004C00u), sgpr_const(0x003C003Cu),
               sgpr_const(0x03C003C0u)};
}
// codes as subnormal halves: nibble bits 4..7 of a half are c 2^-20, which the
// matrix instructions take as it is
constexpr float kCodeUnit = 0x1p-20f;
// a word of K codes -> eight dimensions in order
__device__ __forceinline__ h8 k_codes(uint32_t w, uint32_t nibble) {
  u32x4 o;
  o[0] = (w << 4) & nibble;
  o[1] = w & nibble;
  o[2] = (w >> 4) & nibble;
  o[3] = (w >> 8) & nibble;
  return __builtin_bit_cast(h8, o);
}
// V words of two tiles -> the eight keys' codes of dimension 32 w + r (half 0) or
// 32 w + 16 + r (half 1); key order 0, 2, 1, 3 in each tile
template <int HALF>
__device__ __forceinline__ h8 v_codes(uint32_t w0, uint32_t w1, uint32_t nibble) {
  u32x4 o;
  o[0] = (HALF ? w0 : w0 << 4) & nibble;
  o[1] = (HALF ? w0 >> 8 : w0 >> 4) & nibble;
  o[2] = (HALF ? w1 : w1 << 4) & nibble;
  o[3] = (HALF ? w1 >> 8 : w1 >> 4) & nibble;
  return __builtin_bit_cast(h8, o);
}

__device__ __forceinline__ float lo_half(uint32_t w) { return h2f((uint16_t)w); }
__device__ __forceinline__ float hi_half(uint32_t w) { return h2f((uint16_t)(w >> 16)); }

__device__ __forceinline__ float cols_max(float x) {  // over the four lanes of a column
  x = pair_max(__builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false));
  return pair_max(__builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
}
__device__ __forceinline__ float cols_sum(float x) {
  x = pair_sum(__builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false));
  return pair_sum(__builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
}

// a tile from the cache into LDS, as it lies: 16 bytes a lane, the pairs with a
// part of the lanes
template <int D>
__device__ __forceinline__ void issue_tile(const uint8_t* tile, uint8_t* lds, int lane) {
#pragma unroll
  for (int i = 0; i < D / 64; ++i)
    lds_dma16_w<true>(tile + 1024 * i + 16 * lane, lds + 1024 * i);
  if (lane < D / 8) lds_dma16_w<true>(tile + 16 * D + 16 * lane, lds + 16 * D);
}
template <int D>
constexpr int kTileLoads = D / 64 + 1;

template <int N>
__device__ __forceinline__ void load_words(uint32_t (&w)[N], const uint8_t* p) {
  if constexpr (N == 2) {
    const u32x2 x = *reinterpret_cast<const u32x2*>(p);
    w[0] = x[0];
    w[1] = x[1];
  } else {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(p + 16 * i);
#pragma unroll
      for (int j = 0; j < 4; ++j) w[4 * i + j] = x[j];
    }
  }
}

// what a lane holds of two tiles' keys (or values): operand words of codes, and
// the pairs of keys 4 g .. 4 g + 3
template <int D>
struct Part {
  uint32_t c[2][D / 32], pair[2][D / 16];
};
// Reads it at LDS offsets `codes` + OFF (this lane's codes of the first tile) and
// `pairs` + POFF, and waits for it.  In assembly, because the compiler waits for
// every load into LDS under way before any LDS read it knows of, the next
// block's among them.
template <int D, int OFF, int POFF>
__device__ __forceinline__ void read_part(Part<D>& t, uint32_t codes, uint32_t pairs) {
  constexpr int T = kTileBytes<D>;
  if constexpr (D == 128) {
    u32x4 c0, c1, a0, a1, b0, b1;
    asm volatile(
        "ds_read_b128 %0, %6 offset:%8\n"
        "ds_read_b128 %1, %6 offset:%9\n"
        "ds_read_b128 %2, %7 offset:%10\n"
        "ds_read_b128 %3, %7 offset:%11\n"
        "ds_read_b128 %4, %7 offset:%12\n"
        "ds_read_b128 %5, %7 offset:%13\n"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(c0), "=&v"(c1), "=&v"(a0), "=&v"(a1), "=&v"(b0), "=&v"(b1)
        : "v"(codes), "v"(pairs), "n"(OFF), "n"(OFF + T), "n"(POFF), "n"(POFF + 16), "n"(POFF + T),
          "n"(POFF + T + 16)
        : "memory");
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      t.c[0][i] = c0[i];
      t.c[1][i] = c1[i];
      t.pair[0][i] = a0[i];
      t.pair[0][4 + i] = a1[i];
      t.pair[1][i] = b0[i];
      t.pair[1][4 + i] = b1[i];
    }
  } else {
    u32x2 c0, c1;
    u32x4 a, b;
    asm volatile(
        "ds_read_b64 %0, %4 offset:%6\n"
        "ds_read_b64 %1, %4 offset:%7\n"
        "ds_read_b128 %2, %5 offset:%8\n"
        "ds_read_b128 %3, %5 offset:%9\n"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(c0), "=&v"(c1), "=&v"(a), "=&v"(b)
        : "v"(codes), "v"(pairs), "n"(OFF), "n"(OFF + T), "n"(POFF), "n"(POFF + T)
        : "memory");
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      t.pair[0][i] = a[i];
      t.pair[1][i] = b[i];
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      t.c[0][i] = c0[i];
      t.c[1][i] = c1[i];
    }
  }
}

// the codes of two tiles alone
template <int D, int OFF>
__device__ __forceinline__ void read_codes(uint32_t (&c)[2][D / 32], uint32_t codes) {
  constexpr int T = kTileBytes<D>;
  if constexpr (D == 128) {
    u32x4 c0, c1;
    asm volatile(
        "ds_read_b128 %0, %2 offset:%3\n"
        "ds_read_b128 %1, %2 offset:%4\n"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(c0), "=&v"(c1)
        : "v"(codes), "n"(OFF), "n"(OFF + T)
        : "memory");
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      c[0][i] = c0[i];
      c[1][i] = c1[i];
    }
  } else {
    u32x2 c0, c1;
    asm volatile(
        "ds_read_b64 %0, %2 offset:%3\n"
        "ds_read_b64 %1, %2 offset:%4\n"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(c0), "=&v"(c1)
        : "v"(codes), "n"(OFF), "n"(OFF + T)
        : "memory");
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      c[0][i] = c0[i];
      c[1][i] = c1[i];
    }
  }
}

// result of column r of a tile of 16 columns: straight to o, or a partial
template <int D>
__device__ __forceinline__ void put(const AttnPages& a, const Seq& s, int h, int row, int sp, int ns,
                                    int dim, float acc, float R, float l) {
  if (ns == 1) {
    a.o[(int64_t)row * a.ldo + (int64_t)h * D + dim] = f2h(l > 0.f ? acc / l : (l == l ? 0.f : l));
  } else {
    const int64_t at = ((int64_t)row * a.H + h) * a.splits + sp;
    a.part[at * D + dim] = acc;
    if (dim == 0) a.part_rl[at] = make_float2(R, l);
  }
}

// Few columns: a workgroup is W waves on (sequence, key/value head, 16 / PACK
// columns, split) that take the split's keys by turns, 32 PACK at a time, through
// LDS of their own: two blocks each, the next loaded while one is worked on.
// PACK 2, for at most eight columns: the operands of a block's first 32 keys have
// the queries in columns 0..7 and zeros in the others, those of its second 32 the
// reverse, so the products of both meet in one register, and everything per score
// is done once for 64 keys.
// Codes are operands at their value, as subnormal halves: under an exponent, as 256 + c,
// the sums would have to be corrected by up to 17 times what is left of them (relative
// error of the output where scores hardly differ, 4 heads of 128: 2.1e-4 now at
// scores of 190 and 2.5e-4 at 1800, where those sums left 7.3e-4 and 4.6e-3; for 1 to 2 %
// of the time, 64 keys' instructions being 32 more).
// The sums of p s c, c 0 to 15, grow with the keys where the output does not, and so
// would their rounding: every kCentreBlocks blocks they are centred.  Relative error
// of the output over 16384, 65536 and 262144 nearly equal weights (its own rounding:
// 2e-4): 2.1e-4, 2.1e-4 and 1.8e-4; corrected at the end only, 1.4e-3, 3.7e-3 and 9.2e-3
// with p s (256 + c).
// With many sequences bound by HBM (64 of 513 to 544 keys of 56 heads of 128: 274 MB
// in 65 us, 4.2 TB/s, where a large copy moves 4.86), with few by vector arithmetic
// (580 instructions for 64 keys) and the loads that wait for each other.
template <int D, int W, int PACK>
struct FewLds {  // two blocks a wave; the waves' sums at the end
  __attribute__((aligned(1024))) uint8_t ring[W][2 * 2 * PACK * kTileBytes<D>];
  float R[W][16], l[W][16];
};

template <int D, int W, int PACK>
__device__ __forceinline__ void few_columns(const AttnPages& a, int pair, int sp, int ct,
                                            FewLds<D, W, PACK>& lds) {
  constexpr int KK = D / 32, NG = D / 64, NF = D / 16;
  constexpr int T = 2 * PACK, KEYS = 16 * T, COLS = 16 / PACK;  // tiles and keys of a block, columns
  const int kh = pair % a.c.Hkv, si = pair / a.c.Hkv;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // the wave's blocks are p0 + KEYS (wave + W i); lane T i + j holds the page of
  // tile j of block i, 64 / T blocks at a time, the first of them read beside the
  // sequence's length
  const int32_t* row = a.c.table + si * a.c.stride;
  const int p0 = sp * a.chunk_few, step = W * KEYS;
  int p = p0 + wave * KEYS;
  const auto ahead = [&](int p) { return (int64_t)p + lane / T * step + 16 * (lane % T); };
  const auto entry = [&](int64_t pos, int end) { return pos < end ? row[pos >> a.c.ps_log2] : -1; };
  int pages = entry(ahead(p), a.max_len), block = 0;

  const Seq s = sequence(a, si);
  const int cols = s.rows * a.G;
  if (COLS * ct >= cols || cols > a.few_cols) return;
  const int ns = max(1, (s.len + a.chunk_few - 1) / a.chunk_few);
  if (sp >= ns) return;
  const int r = lane & 15, g = lane >> 4;
  const uint32_t nibble = sgpr_const(0x00F000F0u);
  constexpr int BLK = T * kTileBytes<D>, ROW = D + 4;
  static_assert(16 * ROW * 4 <= 2 * BLK, "a wave's sums fit its blocks");
  uint8_t* const ring = lds.ring[wave];
  const uint32_t ring_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)ring;

  // this lane's column: keys [0, vis) are visible
  // (PACK 2: of the first half block, or for r >= 8 of the second)
  const int half = r / COLS, col = COLS * ct + r % COLS, qj = col / a.G, h = kh * a.G + col % a.G;
  const int vis = col < cols ? max(0, s.len - s.nq + qj + 1) : 0;
  const int jmin = COLS * ct / a.G, jmax = min(s.rows - 1, (COLS * ct + COLS - 1) / a.G);
  const int all = max(0, s.len - s.nq + jmin + 1);      // visible to every column
  const int end = max(0, s.len - s.nq + jmax + 1);      // to any
  const int p1 = min(end, p0 + a.chunk_few);

  f4 acc[NF];
#pragma unroll
  for (int n = 0; n < NF; ++n) acc[n] = f4{0.f, 0.f, 0.f, 0.f};
  float R = -INFINITY, l = 0.f, msum[NG] = {};  // sums of p and p m
  f4 psum[NG];                                  // of p s, in every element, since
  int blocks = 0;                               // so many blocks
#pragma unroll
  for (int n = 0; n < NG; ++n) psum[n] = f4{0.f, 0.f, 0.f, 0.f};
  const h8 ones = h8(1);

  uint32_t valid = 0;  // bit T s + j: tile j in slot s is a page's
  if (ahead(p) >= p1) pages = -1;
  const auto issue = [&](int p, int slot) {
    if (block == 64 / T) {
      block = 0;
      pages = entry(ahead(p), p1);
    }
#pragma unroll
    for (int j = 0; j < T; ++j) {
      const int page = __builtin_amdgcn_readlane(pages, T * block + j);
      const bool ok = page >= 0 && page < a.c.n_pages;
      valid = (valid & ~(1u << (T * slot + j))) | ((uint32_t)ok << (T * slot + j));
      issue_tile<D>(tile_at<D>(a.c, ok ? page : 0, kh, p + 16 * j),
                    ring + slot * BLK + j * kTileBytes<D>, lane);
    }
    ++block;
  };

  int slot = 0;
  if (p < p1) issue(p, 0);
  if (p + step < p1) issue(p + step, 1);

  h8 qf[PACK][KK];  // of the column in its own half, 0 in the other
  float qsum[NG];  // of the column's q, in units of the codes
#pragma unroll
  for (int n = 0; n < NG; ++n) {
    float sum = 0.f;
#pragma unroll
    for (int kk = 2 * n; kk < 2 * n + 2; ++kk) {
      const h8 q = col < cols ? load_q<D>(a, s.row0 + qj, h, 32 * kk + 8 * g) : zero_h8();
#pragma unroll
      for (int j = 0; j < 8; ++j) sum += (float)q[j];
#pragma unroll
      for (int u = 0; u < PACK; ++u) qf[u][kk] = half == u ? q : zero_h8();
    }
    qsum[n] = cols_sum(sum) * kCodeUnit;
  }

  const auto compute = [&](int p, int slot, auto edge_c) {
    constexpr bool EDGE = decltype(edge_c)::value;
    const uint32_t codes = ring_at + slot * BLK + lane * (D / 8);
    const uint32_t scales = ring_at + slot * BLK + half * (2 * kTileBytes<D>) + g * (D / 4);
    const int pos = p + 32 * half;  // of this lane's scores
    int lim[2];                     // keys of its tiles that exist
#pragma unroll
    for (int j = 0; j < 2; ++j)
      lim[j] = EDGE && !(valid >> (T * slot + 2 * half + j) & 1) ? 0 : p1 - pos - 16 * j;
    float x[2][4], bm = -INFINITY;  // scores times kCodeUnit
    Part<D> t;
    uint32_t c2[2][KK];  // the second half's codes
    read_part<D, 0, 16 * D>(t, codes, scales);
    if constexpr (PACK == 2) read_codes<D, 2 * kTileBytes<D>>(c2, codes);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      f4 sc[NG];
#pragma unroll
      for (int n = 0; n < NG; ++n) {
        sc[n] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 2 * n; kk < 2 * n + 2; ++kk) {
          sc[n] = mfma16(k_codes(t.c[j][kk], nibble), qf[0][kk], sc[n]);
          if constexpr (PACK == 2) sc[n] = mfma16(k_codes(c2[j][kk], nibble), qf[1][kk], sc[n]);
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float v = 0.f;
#pragma unroll
        for (int n = 0; n < NG; ++n) {
          const uint32_t w = t.pair[j][e * NG + n];
          v = n == 0 ? lo_half(w) * qsum[0] : __builtin_fmaf(lo_half(w), qsum[n], v);
          v = __builtin_fmaf(hi_half(w), sc[n][e], v);
        }
        if constexpr (EDGE) {
          const int key = 4 * g + e;
          v = key < lim[j] && pos + 16 * j + key < vis ? v : -INFINITY;
        }
        x[j][e] = v;
        bm = fmaxf(bm, v);
      }
    }
    uint32_t top = 0;
    read_part<D, 8 * D, 17 * D>(t, codes, scales);
    if constexpr (PACK == 2) read_codes<D, 2 * kTileBytes<D> + 8 * D>(c2, codes);
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int n = 0; n < NG; ++n) {
          uint32_t& w = t.pair[j][e * NG + n];
          if constexpr (EDGE) w = 4 * g + e < lim[j] ? w : 0u;  // past the end: anything
          top = max(top, w);
        }
    bm = cols_max(bm);
    // scales are below 2^(exponent field - 14)
    const float es = cols_max((float)((int)(top >> 26) - 14));
    const float Rn = fmaxf(R, __builtin_fmaf(bm, kLog2e / kCodeUnit, es));
    const float Rs = EDGE && Rn == -INFINITY ? 0.f : Rn;
    const float alpha = __builtin_amdgcn_exp2f(R - Rs);
    R = Rn;
    if (__any(alpha != 1.f)) {  // the running maxima rarely grow after the first blocks
      l *= alpha;
#pragma unroll
      for (int n = 0; n < NG; ++n) {
        psum[n] *= alpha;
        msum[n] *= alpha;
      }
#pragma unroll
      for (int n = 0; n < NF; ++n) acc[n] *= alpha;
    }
    const float shift = kPBits - Rs;
    h8 hi[NG], lo[NG];
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        constexpr int kOrder[4] = {0, 2, 1, 3};  // of v_codes
        const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(x[j][e], kLog2e / kCodeUnit, shift));
        l += y;
#pragma unroll
        for (int n = 0; n < NG; ++n) {
          const uint32_t w = t.pair[j][e * NG + n];
          // p s in two halves, 22 bits of it (fused, so that each is one
          // instruction with its rounding)
          const _Float16 a16 = (_Float16)__builtin_fmaf(y, hi_half(w), 0.f);
          hi[n][4 * j + kOrder[e]] = a16;
          lo[n][4 * j + kOrder[e]] = (_Float16)__builtin_fmaf(y, hi_half(w), -(float)a16);
          msum[n] = __builtin_fmaf(y, lo_half(w), msum[n]);
        }
      }
#pragma unroll
    for (int n = 0; n < NG; ++n) {
      psum[n] = mfma16(ones, hi[n], psum[n]);
      psum[n] = mfma16(ones, lo[n], psum[n]);
    }
#pragma unroll
    for (int u = 0; u < PACK; ++u) {
      h8 phi[NG], plo[NG];  // the half block's weights in its own columns
#pragma unroll
      for (int n = 0; n < NG; ++n) {
        phi[n] = PACK == 1 || half == u ? hi[n] : zero_h8();
        plo[n] = PACK == 1 || half == u ? lo[n] : zero_h8();
      }
#pragma unroll
      for (int w = 0; w < KK; ++w) {
        const int n = w / 2;
        const uint32_t w0 = u ? c2[0][w] : t.c[0][w], w1 = u ? c2[1][w] : t.c[1][w];
        const h8 v0 = v_codes<0>(w0, w1, nibble), v1 = v_codes<1>(w0, w1, nibble);
        acc[2 * w] = mfma16(v0, phi[n], acc[2 * w]);
        acc[2 * w] = mfma16(v0, plo[n], acc[2 * w]);
        acc[2 * w + 1] = mfma16(v1, phi[n], acc[2 * w + 1]);
        acc[2 * w + 1] = mfma16(v1, plo[n], acc[2 * w + 1]);
      }
    }
  };

  // 7.5 p s from the sums of p s c to those of p m (a quarter of it in each of a
  // column's lanes): both then have values' own size, not that of 7.5 scales
  const auto centre = [&] {
#pragma unroll
    for (int n = 0; n < NF; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        acc[n][e] = __builtin_fmaf(-7.5f * kCodeUnit, psum[n / 4][e], acc[n][e]);
#pragma unroll
    for (int n = 0; n < NG; ++n) {
      msum[n] = __builtin_fmaf(1.875f, psum[n][0], msum[n]);
      psum[n] = f4{0.f, 0.f, 0.f, 0.f};
    }
    blocks = 0;
  };

  // first the blocks that every column sees whole, up to one without a page
  const auto run = [&](auto edge_c) {
    constexpr bool EDGE = decltype(edge_c)::value;
    for (; p < p1; p += step, slot ^= 1) {
      if (!EDGE && (p + KEYS > all || (valid >> (T * slot) & ((1 << T) - 1)) != (1 << T) - 1)) return;
      if (p + step < p1)  // this block has landed, the next may still travel
        __builtin_amdgcn_s_waitcnt(waitcnt_imm(T * kTileLoads<D>, false));
      else
        __builtin_amdgcn_s_waitcnt(waitcnt_imm(0, false));
      __builtin_amdgcn_sched_barrier(0);
      compute(p, slot, edge_c);
      __builtin_amdgcn_sched_barrier(0);  // (the slot is read)
      if (p + 2 * step < p1) issue(p + 2 * step, slot);
      if (++blocks == kCentreBlocks) centre();
    }
  };
  run(std::false_type{});
  run(std::true_type{});

  // merge the waves (and halves): element e of acc[n] is dimension 16 n + 4 g + e of
  // column r
  centre();
  l = cols_sum(l);
#pragma unroll
  for (int n = 0; n < NG; ++n) msum[n] = cols_sum(msum[n]);
#pragma unroll
  for (int n = 0; n < NF; ++n) {
    f4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = __builtin_fmaf(acc[n][e], 1.f / kCodeUnit, msum[n / 4]);
    *reinterpret_cast<f4*>(reinterpret_cast<float*>(ring) + r * ROW + 16 * n + 4 * g) = v;
  }
  if (g == 0) {
    lds.R[wave][r] = R;
    lds.l[wave][r] = l;
  }
  __syncthreads();
  for (int c = tid; c < COLS * D; c += W * 64) {
    const int cr = c / D, dim = c % D, cc = COLS * ct + cr;
    if (cc >= cols) break;
    float Rm = -INFINITY;
#pragma unroll
    for (int w = 0; w < W * PACK; ++w) Rm = fmaxf(Rm, lds.R[w / PACK][w % PACK * COLS + cr]);
    const float Rs = Rm == -INFINITY ? 0.f : Rm;
    float A = 0.f, L = 0.f;
#pragma unroll
    for (int w = 0; w < W * PACK; ++w) {
      const int i = w % PACK * COLS + cr;
      const float f = __builtin_amdgcn_exp2f(lds.R[w / PACK][i] - Rs);
      const float* acc_w = reinterpret_cast<const float*>(lds.ring[w / PACK]);
      A = __builtin_fmaf(acc_w[i * ROW + dim], f, A);
      L = __builtin_fmaf(lds.l[w / PACK][i], f, L);
    }
    put<D>(a, s, kh * a.G + cc % a.G, s.row0 + cc / a.G, sp, ns, dim, A, Rm, L);
  }
}

// Many columns: a workgroup is one or two teams of four waves of 32 columns each
// on (sequence, key/value head, 128 columns, split).  Two teams take the split's
// keys by turns, 64 at a time, and meet in LDS at the end.  In a team each wave
// unpacks a tile of the next block into LDS, in operand order (keys as c, values as
// c - 7.5), while all of them work on this one, so a block is unpacked once for 128
// columns and every LDS access is a wave's contiguous kilobyte.  The weights p s
// go to the second product rounded to a half: with the codes centred, and the
// rest of a value, p (m + 7.5 s), summed in fp32, that is one rounding of the
// size of the output's own.
// Bound by vector instructions, 590 of a wave beside 64 matrix ones for a block
// (eight sequences of 509 rows over 4099 keys, 32/8 heads: 452 us, 567 TFLOP/s, the
// vector pipe issues in 67 % of the cycles, the matrix pipe is busy in 23 %).
constexpr int kManyCols = 128, kManyKeys = 64;

// a word of K codes -> eight dimensions, c
__device__ __forceinline__ h8 k_plain(uint32_t w, const Magic& g) {
  const uint32_t a = w << 2, b = w >> 6;
  u32x4 o;
  o[0] = (a & g.m256) | g.e256;
  o[1] = (a & g.m16) | g.e16;
  o[2] = (b & g.m256) | g.e256;
  o[3] = (b & g.m16) | g.e16;
  const h8 bias = {256.f16, 256.f16, 16.f16, 16.f16, 256.f16, 256.f16, 16.f16, 16.f16};
  return __builtin_bit_cast(h8, o) - bias;
}
// a V word -> four keys (0, 2, 1, 3) of dimension 32 w + r (half 0) or 32 w + 16
// + r, c - 7.5
template <int HALF>
__device__ __forceinline__ h4 v_centred(uint32_t w, const Magic& g) {
  const uint32_t m = HALF ? g.m16 : g.m256, e = HALF ? g.e16 : g.e256;
  u32x2 o;
  o[0] = ((w << 2) & m) | e;
  o[1] = ((w >> 6) & m) | e;
  constexpr _Float16 b = HALF ? 23.5f16 : 263.5f16;
  return __builtin_bit_cast(h4, o) - h4{b, b, b, b};
}

// The t-th column tile of the launch: its sequence (-1: none) and which of the
// sequence's tiles.  Only sequences of many columns have tiles, so that a batch of
// which a few are prompts launches little else (a workgroup with nothing to do
// waits for as much LDS as the others).  Up to 64 sequences go by their keys, the
// most first (16 prompts' 509 rows each over 509 to 4099 keys: 556 -> 489 us).
// Of a sequence the tiles with the most keys come first.
struct Place {
  int seq, tile;
};
__device__ __forceinline__ int many_tiles(const AttnPages& a, int i) {
  const int cols = sequence(a, i).rows * a.G;
  return cols > a.few_cols ? (cols + kManyCols - 1) / kManyCols : 0;
}
__device__ __forceinline__ Place place_of(const AttnPages& a, int t) {
  const int n = a.c.n_seq, lane = threadIdx.x & 63;
  if (n <= 64) {
    const int tiles = lane < n ? many_tiles(a, lane) : 0, keys = tiles ? a.kv_len[lane] : 0;
    int before = 0;
    for (int i = 0; i < n; ++i) {
      const int k = __builtin_amdgcn_readlane(keys, i), w = __builtin_amdgcn_readlane(tiles, i);
      before += k > keys || (k == keys && i < lane) ? w : 0;
    }
    const uint64_t hit = __ballot(t >= before && t < before + tiles);
    if (!hit) return Place{-1, 0};
    const int i = __ffsll((unsigned long long)hit) - 1;
    return Place{i, __builtin_amdgcn_readlane(before + tiles - 1, i) - t};
  }
  const int each = (n + 63) / 64, first = lane * each, last = min(n, first + each);
  int sum = 0;
  for (int i = first; i < last; ++i) sum += many_tiles(a, i);
  int end = sum;  // of this lane's tiles
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int y = __shfl_up(end, d, 64);
    if (lane >= d) end += y;
  }
  const uint64_t hit = __ballot(t >= end - sum && t < end);
  if (!hit) return Place{-1, 0};
  const int src = __ffsll((unsigned long long)hit) - 1;
  int r = t - __builtin_amdgcn_readlane(end - sum, src);
  for (int i = src * each;; ++i) {  // (ends: r is below the sum of these)
    const int tiles = many_tiles(a, i);
    if (r < tiles) return Place{i, tiles - 1 - r};
    r -= tiles;
  }
}

template <int CTRL>
__device__ __forceinline__ uint32_t lane_move_u(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, false);
}

// Makes the compiler forget that it has converted these halves, so that the next
// use takes them as operands of a mixed multiply-add instead of as floats kept in
// registers.
template <int N>
__device__ __forceinline__ void as_halves(uint32_t (&w)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+v"(w[i]));
}

// K operands [tile][kk][lane], V operands [pair of tiles][fragment][lane], the
// (min, scale) words [K, V][tile][key][group] (0 past the end), the largest of
// each tile's V and which tiles are pages'
template <int D>
struct ManyStage {
  h8 k[kManyKeys / 16][D / 32][64];
  h8 v[kManyKeys / 32][D / 16][64];
  uint32_t pair[2][kManyKeys / 16][16 * (D / 64)];
  uint32_t top[kManyKeys / 16], valid[kManyKeys / 16];
};
template <int D, int TEAMS>
struct ManyLds {
  static constexpr int ROW = D + 4;  // floats of a column's sums, where the teams meet
  union {
    ManyStage<D> st[TEAMS][2];
    float sums[TEAMS - 1 ? kManyCols : 1][ROW];
  };
  float2 rl[TEAMS - 1 ? kManyCols : 1];
};

template <int D, int TEAMS>
__device__ __forceinline__ void many_columns(const AttnPages& a, int pair, int sp,
                                             ManyLds<D, TEAMS>& lds) {
  constexpr int KK = D / 32, NG = D / 64, NF = D / 16, T = kManyKeys / 16, U = 2;
  using Stage = ManyStage<D>;
  const int kh = pair % a.c.Hkv;
  const Place at = place_of(a, pair / a.c.Hkv);
  if (at.seq < 0) return;
  const int si = __builtin_amdgcn_readfirstlane(at.seq);
  const int ct = __builtin_amdgcn_readfirstlane(at.tile);
  const Seq s = sequence(a, si);
  const int cols = s.rows * a.G;
  const int ns = max(1, (s.len + a.chunk_many - 1) / a.chunk_many);
  if (sp >= ns) return;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6) & 3;
  const int team = __builtin_amdgcn_readfirstlane(tid >> 8);
  const int r = lane & 15, g = lane >> 4;
  const Magic mg = magic();

  Stage* const st = lds.st[team];

  const int c0 = kManyCols * ct + 32 * wave;  // this wave's first column
  const int q_last = min(s.rows - 1, (kManyCols * ct + kManyCols - 1) / a.G);
  const int end = max(0, s.len - s.nq + q_last + 1);  // keys visible to any column
  const int p0 = sp * a.chunk_many, p1 = min(end, p0 + a.chunk_many);
  const int blocks = p1 > p0 ? (p1 - p0 + kManyKeys - 1) / kManyKeys : 0;
  // this team's are blocks team, team + TEAMS .., and all waves go through as many
  const int turns = (blocks + TEAMS - 1) / TEAMS, mine = (blocks + TEAMS - 1 - team) / TEAMS;
  // keys visible to all of the wave's columns, and to any
  const int all = max(0, s.len - s.nq + c0 / a.G + 1);
  const int end_w = c0 < cols ? min(p1, s.len - s.nq + min(s.rows - 1, (c0 + 31) / a.G) + 1) : 0;

  // this wave's tile of the next block, on its way
  uint32_t kw[KK], vw[KK];
  u32x4 pw;
  uint32_t ok;
  int lim;
  // lane i holds the page of its tile in the team's block i, 64 at a time
  const int32_t* row = a.c.table + si * a.c.stride;
  int pages = -1;
  const auto fetch = [&](int blk) {
    const int pos = p0 + (TEAMS * blk + team) * kManyKeys + 16 * wave;
    if ((blk & 63) == 0) {
      const int64_t at = (int64_t)pos + (int64_t)lane * (TEAMS * kManyKeys);
      pages = at < p1 ? row[at >> a.c.ps_log2] : -1;
    }
    const int page = __builtin_amdgcn_readlane(pages, blk & 63);
    ok = page >= 0 && page < a.c.n_pages;
    lim = ok ? p1 - pos : 0;  // keys of the tile that exist
    const uint8_t* tile = tile_at<D>(a.c, ok ? page : 0, kh, pos);
    load_words(kw, tile + lane * (D / 8));
    load_words(vw, tile + 8 * D + lane * (D / 8));
    if (lane < D / 8) pw = *reinterpret_cast<const u32x4*>(tile + 16 * D + 16 * lane);
  };
  const auto unpack = [&](Stage& x) {
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) x.k[wave][kk][lane] = k_plain(kw[kk], mg);
#pragma unroll
    for (int w = 0; w < KK; ++w) {
      h4* v0 = reinterpret_cast<h4*>(&x.v[wave / 2][2 * w][lane]);
      h4* v1 = reinterpret_cast<h4*>(&x.v[wave / 2][2 * w + 1][lane]);
      v0[wave % 2] = v_centred<0>(vw[w], mg);
      v1[wave % 2] = v_centred<1>(vw[w], mg);
    }
    if (lane < D / 8) {  // the first half of these lanes has K's, the others V's
      const int at = 4 * (lane % (D / 16));
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if ((at + i) / NG >= lim) pw[i] = 0;  // past the end, or page 0's: anything
      *reinterpret_cast<u32x4*>(x.pair[lane / (D / 16)][wave] + at) = pw;
      uint32_t top = max(max(pw[0], pw[1]), max(pw[2], pw[3]));
      top = max(top, lane_move_u<0xB1>(top));
      top = max(top, lane_move_u<0x4E>(top));
      if constexpr (D == 128) top = max(top, lane_move_u<0x141>(top));
      if (lane == D / 16) {
        x.top[wave] = top;
        x.valid[wave] = ok;
      }
    }
  };

  h8 qf[U][KK];
  float qsum[U][NG];
  int vis[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int col = c0 + 16 * u + r, qj = col / a.G;
    vis[u] = col < cols ? max(0, s.len - s.nq + qj + 1) : 0;
#pragma unroll
    for (int n = 0; n < NG; ++n) {
      float sum = 0.f;
#pragma unroll
      for (int kk = 2 * n; kk < 2 * n + 2; ++kk) {
        qf[u][kk] = col < cols ? load_q<D>(a, s.row0 + qj, kh * a.G + col % a.G, 32 * kk + 8 * g)
                               : zero_h8();
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += (float)qf[u][kk][j];
      }
      qsum[u][n] = cols_sum(sum);
    }
  }
  f4 acc[U][NF];
  float R[U], l[U], msum[U][NG];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    R[u] = -INFINITY;
    l[u] = 0.f;
#pragma unroll
    for (int n = 0; n < NG; ++n) msum[u][n] = 0.f;
#pragma unroll
    for (int n = 0; n < NF; ++n) acc[u][n] = f4{0.f, 0.f, 0.f, 0.f};
  }

  const auto compute = [&](const Stage& x, int k0, auto edge_c) {
    constexpr bool EDGE = decltype(edge_c)::value;
    float sc[U][T][4];
    h8 kf[2][KK];
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) kf[0][kk] = x.k[0][kk][lane];
#pragma unroll
    for (int j = 0; j < T; ++j) {
      f4 d[U][NG];
      uint32_t w[4 * NG];
      load_words(w, reinterpret_cast<const uint8_t*>(&x.pair[0][j][4 * g * NG]));
      if (j + 1 < T) {
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) kf[(j + 1) & 1][kk] = x.k[j + 1][kk][lane];
      }
      __builtin_amdgcn_sched_barrier(0);  // (these loads travel beside this tile's work)
#pragma unroll
      for (int kk = 0; kk < KK; ++kk)
#pragma unroll
        for (int u = 0; u < U; ++u)
          d[u][kk / 2] =
              mfma16(kf[j & 1][kk], qf[u][kk], kk % 2 ? d[u][kk / 2] : f4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (u > 0) as_halves(w);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float v = 0.f;
#pragma unroll
          for (int n = 0; n < NG; ++n) {
            v = __builtin_fmaf(lo_half(w[e * NG + n]), qsum[u][n], v);
            v = __builtin_fmaf(hi_half(w[e * NG + n]), d[u][n][e], v);
          }
          if constexpr (EDGE) v = x.valid[j] && k0 + 16 * j + 4 * g + e < vis[u] ? v : -INFINITY;
          sc[u][j][e] = v;
        }
      }
    }
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < T; ++j) top = max(top, x.top[j]);
    // scales are below 2^(exponent field - 14)
    const float es = (float)((int)(top >> 26) - 14);
    float shift[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float bm = -INFINITY;
#pragma unroll
      for (int j = 0; j < T; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) bm = fmaxf(bm, sc[u][j][e]);
      bm = cols_max(bm);
      const float Rn = fmaxf(R[u], __builtin_fmaf(bm, kLog2e, es));
      const float Rs = EDGE && Rn == -INFINITY ? 0.f : Rn;
      const float alpha = __builtin_amdgcn_exp2f(R[u] - Rs);
      R[u] = Rn;
      shift[u] = kPBits - Rs;
      if (__any(alpha != 1.f)) {
        l[u] *= alpha;
#pragma unroll
        for (int n = 0; n < NG; ++n) msum[u][n] *= alpha;
#pragma unroll
        for (int n = 0; n < NF; ++n) acc[u][n] *= alpha;
      }
    }
#pragma unroll
    for (int t = 0; t < T / 2; ++t) {
      h8 pf[U][NG];
      uint32_t vp[2][4 * NG];
#pragma unroll
      for (int jj = 0; jj < 2; ++jj)
        load_words(vp[jj], reinterpret_cast<const uint8_t*>(&x.pair[1][2 * t + jj][4 * g * NG]));
      h8 vf[NF];
#pragma unroll
      for (int n = 0; n < NF; ++n) vf[n] = x.v[t][n][lane];
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int jj = 0; jj < 2; ++jj)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          constexpr int kOrder[4] = {0, 2, 1, 3};  // of v_centred
          const int j = 2 * t + jj;
          float y[U];
#pragma unroll
          for (int u = 0; u < U; ++u) {
            y[u] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[u][j][e], kLog2e, shift[u]));
            l[u] += y[u];
          }
#pragma unroll
          for (int n = 0; n < NG; ++n) {
            uint32_t w[1] = {vp[jj][e * NG + n]};
            const float mu = __builtin_fmaf(hi_half(w[0]), 7.5f, lo_half(w[0]));
#pragma unroll
            for (int u = 0; u < U; ++u) {
              as_halves(w);
              pf[u][n][4 * jj + kOrder[e]] = (_Float16)__builtin_fmaf(y[u], hi_half(w[0]), 0.f);
              msum[u][n] = __builtin_fmaf(y[u], mu, msum[u][n]);
            }
          }
        }
#pragma unroll
      for (int n = 0; n < NF; ++n) {
#pragma unroll
        for (int u = 0; u < U; ++u) acc[u][n] = mfma16(vf[n], pf[u][n / 4], acc[u][n]);
      }
      // (else these sums sink behind the next block's unpacking, and keep y and vp alive)
#pragma unroll
      for (int u = 0; u < U; ++u) {
        asm volatile("" : "+v"(l[u]));
#pragma unroll
        for (int n = 0; n < NG; ++n) asm volatile("" : "+v"(msum[u][n]));
      }
    }
  };

  if (mine > 0) {
    fetch(0);
    unpack(st[0]);
  }
  __syncthreads();
  int blk = 0;
  // first the blocks that all columns of the wave see whole, up to one with a
  // tile that is no page's; every wave goes through every block
  const auto run = [&](auto edge_c) {
    constexpr bool EDGE = decltype(edge_c)::value;
    for (; blk < turns; ++blk) {
      const Stage& x = st[blk & 1];
      const int k0 = p0 + (TEAMS * blk + team) * kManyKeys;
      if constexpr (!EDGE) {
        uint32_t v = 1;
#pragma unroll
        for (int j = 0; j < T; ++j) v &= x.valid[j];
        if (blk >= mine || k0 + kManyKeys > all || !__builtin_amdgcn_readfirstlane(v)) return;
      }
      if (blk + 1 < mine) fetch(blk + 1);
      if (!EDGE || (blk < mine && k0 < end_w)) compute(x, k0, edge_c);
      if (blk + 1 < mine) unpack(st[(blk + 1) & 1]);
      __syncthreads();
    }
  };
  run(std::false_type{});
  run(std::true_type{});

  // element e of acc[u][n]: dimension 16 n + 4 g + e of column c0 + 16 u + r.  The
  // second team's sums go to LDS (every block there is read), the first adds them.
#pragma unroll
  for (int u = 0; u < U; ++u) {
    l[u] = cols_sum(l[u]);
#pragma unroll
    for (int n = 0; n < NG; ++n) msum[u][n] = cols_sum(msum[u][n]);
#pragma unroll
    for (int n = 0; n < NF; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[u][n][e] += msum[u][n / 4];
    const int c = 32 * wave + 16 * u + r;
    if (team == 1) {
#pragma unroll
      for (int n = 0; n < NF; ++n)
        *reinterpret_cast<f4*>(&lds.sums[c][16 * n + 4 * g]) = acc[u][n];
      if (g == 0) lds.rl[c] = make_float2(R[u], l[u]);
    }
  }
  if constexpr (TEAMS == 2) {
    __syncthreads();
    if (team == 1) return;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int c = 32 * wave + 16 * u + r;
      const float2 rl = lds.rl[c];
      const float Rn = fmaxf(R[u], rl.x), Rs = Rn == -INFINITY ? 0.f : Rn;
      const float f0 = __builtin_amdgcn_exp2f(R[u] - Rs), f1 = __builtin_amdgcn_exp2f(rl.x - Rs);
      R[u] = Rn;
      l[u] = l[u] * f0 + rl.y * f1;
#pragma unroll
      for (int n = 0; n < NF; ++n) {
        const f4 y = *reinterpret_cast<const f4*>(&lds.sums[c][16 * n + 4 * g]);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[u][n][e] = acc[u][n][e] * f0 + y[e] * f1;
      }
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int col = c0 + 16 * u + r;
    const float L = l[u];
    if (col >= cols) continue;
    const int m = s.row0 + col / a.G, h = kh * a.G + col % a.G;
    if (ns == 1) {
      const float inv = L > 0.f ? 1.f / L : (L == L ? 0.f : L);
      uint16_t* o = a.o + (int64_t)m * a.ldo + (int64_t)h * D;
#pragma unroll
      for (int n = 0; n < NF; ++n) {
        uint16_t v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = f2h(acc[u][n][e] * inv);
        if (a.o_vec) {
          *reinterpret_cast<u32x2*>(o + 16 * n + 4 * g) =
              u32x2{(uint32_t)v[0] | ((uint32_t)v[1] << 16), (uint32_t)v[2] | ((uint32_t)v[3] << 16)};
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) o[16 * n + 4 * g + e] = v[e];
        }
      }
    } else {
      const int64_t at = ((int64_t)m * a.H + h) * a.splits + sp;
#pragma unroll
      for (int n = 0; n < NF; ++n) {
        *reinterpret_cast<f4*>(a.part + at * D + 16 * n + 4 * g) = acc[u][n];
      }
      if (g == 0) a.part_rl[at] = make_float2(R[u], L);
    }
  }
}

template <int D, int W, int PACK>
__global__ __launch_bounds__(W * 64) __attribute__((amdgpu_waves_per_eu(PACK == 2 ? 2 : 3))) void
attn_pages_few_k(AttnPages a) {
  __shared__ FewLds<D, W, PACK> lds;
  few_columns<D, W, PACK>(a, blockIdx.x, blockIdx.y, blockIdx.z, lds);
}

template <int D, int TEAMS>
__global__ __launch_bounds__(TEAMS * 256) __attribute__((amdgpu_waves_per_eu(2))) void
attn_pages_many_k(AttnPages a) {
  __shared__ ManyLds<D, TEAMS> lds;
  many_columns<D, TEAMS>(a, blockIdx.x, blockIdx.y, lds);
}

// Both, the many columns' workgroups first: these work for longer, and all of them
// leave half of a CU's LDS and registers to the others.
template <int D, int PACK>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void
attn_pages_both_k(AttnPages a, int many, int many_splits, int few_splits) {
  union Lds {
    ManyLds<D, 1> many;
    FewLds<D, 4, PACK> few;
  };
  __shared__ Lds lds;
  const int b = blockIdx.x;
  if (b < many * many_splits) {
    many_columns<D, 1>(a, b % many, b / many, lds.many);
  } else {
    const int i = b - many * many_splits, pairs = a.c.Hkv * a.c.n_seq;
    few_columns<D, 4, PACK>(a, i % pairs, i / pairs % few_splits, i / pairs / few_splits, lds.few);
  }
}

// sequence that holds row m (-1: none): the last i with q_start[i] <= m, 64
// candidates at a time
__device__ __forceinline__ int seq_of_row(const AttnPages& a, int m) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = a.c.n_seq + 1;
  while (n > 1) {
    const int step = (n + 63) / 64, i = lo + lane * step;
    const uint64_t below = __ballot(lane * step < n && a.q_start[min(i, a.c.n_seq)] <= m);
    const int k = __popcll(below) - 1;
    if (k < 0) return -1;
    lo += k * step;
    n = min(step, n - k * step);
  }
  return lo < a.c.n_seq ? lo : -1;
}

// Adds the splits of a row's head: threads on four dimensions each take the
// splits by turns, all their loads at once, and the groups of threads are added
// in order.  Up to kSmallMerge splits a wave does it alone, four heads to a
// workgroup (2036 rows of 32 heads in two parts: 58 -> 11 us); above, a workgroup.
// Sequences of few columns by (sequence, row of up to few_rows), the others by row.
constexpr int kSmallMerge = 8;
template <int D, int MAX, bool FEW>
__global__ __launch_bounds__(256) void attn_pages_merge_k(AttnPages a, int few_rows) {
  constexpr bool WAVE = MAX <= kSmallMerge;
  constexpr int LANES = D / 4, GROUPS = (WAVE ? 64 : 256) / LANES, EACH = (MAX + GROUPS - 1) / GROUPS;
  const int h = WAVE ? 4 * blockIdx.y + (threadIdx.x >> 6) : blockIdx.y;
  const int i = FEW ? blockIdx.x / few_rows : seq_of_row(a, blockIdx.x);
  if (i < 0 || h >= a.H) return;
  const Seq s = sequence(a, i);
  const int j = FEW ? blockIdx.x - i * few_rows : blockIdx.x - s.row0, m = s.row0 + j;
  const int chunk = FEW ? a.chunk_few : a.chunk_many;
  const int ns = max(1, (s.len + chunk - 1) / chunk);
  if (ns == 1 || j >= s.rows || FEW != (s.rows * a.G <= a.few_cols)) return;
  const int64_t at = ((int64_t)m * a.H + h) * a.splits;
  const int lane = threadIdx.x & 63, t = WAVE ? lane : threadIdx.x;
  const int grp = t / LANES, dim = 4 * (t % LANES);
  f4 x[EACH];
#pragma unroll
  for (int j = 0; j < EACH; ++j)
    if (grp + j * GROUPS < ns)
      x[j] = *reinterpret_cast<const f4*>(a.part + (at + grp + j * GROUPS) * D + dim);
  const float2 rl = lane < ns ? a.part_rl[at + lane] : make_float2(-INFINITY, 0.f);
  float R = rl.x, w = 0.f;
#pragma unroll
  for (int d = 32; d >= 1; d /= 2) R = fmaxf(R, wave_shfl_xor(R, d));
  if (R != -INFINITY) w = __builtin_amdgcn_exp2f(rl.x - R);
  float L = rl.y * w;
#pragma unroll
  for (int d = 32; d >= 1; d /= 2) L += wave_shfl_xor(L, d);
  f4 A = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int j = 0; j < EACH; ++j) {
    const float f = __shfl(w, min(grp + j * GROUPS, 63), 64);
    if (grp + j * GROUPS < ns)
#pragma unroll
      for (int e = 0; e < 4; ++e) A[e] = __builtin_fmaf(x[j][e], f, A[e]);
  }
  const auto result = [&](float v) { return f2h(L > 0.f ? v / L : (L == L ? 0.f : L)); };
  uint16_t* o = a.o + (int64_t)m * a.ldo + (int64_t)h * D;
  if constexpr (WAVE) {
#pragma unroll
    for (int d = LANES; d < 64; d *= 2)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float y = A[e];
        A[e] = y + wave_shfl_xor(y, d);
      }
    if (grp > 0) return;
    if (a.o_vec) {
      *reinterpret_cast<u32x2*>(o + dim) =
          u32x2{(uint32_t)result(A[0]) | ((uint32_t)result(A[1]) << 16),
                (uint32_t)result(A[2]) | ((uint32_t)result(A[3]) << 16)};
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) o[dim + e] = result(A[e]);
    }
  } else {
    __shared__ f4 sum[GROUPS][LANES];
    sum[grp][t % LANES] = A;
    __syncthreads();
    if (t >= D) return;
    float v = 0.f;
    for (int k = 0; k < GROUPS; ++k) v += sum[k][t / 4][t % 4];
    o[t] = result(v);
  }
}

static int64_t col_tiles(int64_t max_q, int G, int tile) { return (max_q * G + tile - 1) / tile; }

// keys of each of S parts, in whole multiples of `round`
static int chunk_of(int64_t max_len, int64_t S, int round) {
  S = std::max<int64_t>(1, std::min<int64_t>(S, kMaxSplits));
  return (int)std::max<int64_t>(round, ((max_len + S - 1) / S + round - 1) / round * round);
}

// Workgroups.  Few columns: eight waves, whose sums meet in LDS, up to a workgroup
// for each CU, four up to four, then two; below one a CU the keys are split as well,
// 256 at least each and from 768 on (a second kernel costs what 500 keys of a
// workgroup do).  us, 32/8 heads: 28 sequences of 2100 keys with eight waves 22,
// four 27; 64 of 544 20 and 16; 128 of 2048 with four 65, two 60; 16 of 500 unsplit
// 9.4, in two 11.0; 4 of 2000 20.1 and in eight 10.7; 1 of 8000 61.7 and in 32 11.0.
// 64 keys at a time from 1024 on (128 of 2048 67 -> 60, 64 of 2048 37.5 -> 33.8),
// below they leave waves without a block (64 of 544 15.9 -> 17.1).
// Many columns: two teams, one workgroup a CU, up to three workgroups for each, so
// that all SIMDs have two waves until the CU's last key; one team, two workgroups a
// CU, beyond (32/8 heads, 509 rows over 4099 keys: two sequences 128 us with two
// teams, 163 with one; eight 495 and 452; four over 509 to 4099 keys 141 and 171).
// Parts of 512 keys at least where there is not a workgroup for each CU.
// Both kinds in one launch hide the few columns' loads behind the many columns'
// matrix products, but leave these one team: worth it where sequences times key/value
// heads are more than half of the tiles of many columns (counting one row of each
// sequence out), or where one team is right anyway.  32/8 heads, one launch against
// two: 28 sequences of 520 to 2100 keys and two with 509 rows 52 us and 60, 15 and
// one of up to 4000 38 and 51, 94 and six 140 and 186; 12 and four 172 and 165, three
// and one of 16000 keys 439 and 268.
constexpr int kCUs = 256, kMinFew = 256, kSplitFew = 768, kPackKeys = 1024, kMinMany = 512;

struct Plan {
  bool few, many;  // sequences that may be of either kind
  bool both;       // in one launch
  int waves;       // of a workgroup for those of few columns
  bool pack;       // 64 keys at a time for them
  int teams;       // of a workgroup for the others
  int64_t tiles;   // of 128 columns they have at most
  int chunk_few, chunk_many, splits;
};
static Plan plan_attn(const pipo_kv_pages* c, int n_heads, int64_t M, int64_t max_q,
                      int64_t max_len) {
  const int G = n_heads / c->n_kv_heads;
  Plan p;
  p.many = max_q * G > kFewCols;
  p.few = !p.many || (G <= kFewCols && M < c->n_seq * max_q);
  const int64_t few_q = std::max<int64_t>(1, std::min<int64_t>(max_q, kFewCols / G));
  // (with many columns about, most of the others have one row)
  const int64_t q = p.many ? 1 : few_q, wgs = (int64_t)c->n_seq * c->n_kv_heads * col_tiles(q, G, 16);
  p.waves = wgs <= kCUs ? 8 : wgs < 4 * kCUs ? 4 : 2;
  p.chunk_few = chunk_of(max_len, max_len < kSplitFew ? 1 : std::min(kCUs / wgs, max_len / kMinFew),
                         32);
  p.pack = q * G <= kPackCols && p.chunk_few > kPackKeys;
  p.tiles = std::min(c->n_seq * col_tiles(max_q, G, kManyCols), M * G / kManyCols + c->n_seq);
  // (of n columns above 64, at most n / 64.5)
  static_assert(kManyCols == 2 * kFewCols, "the bound of a sequence's tiles");
  if (p.few) p.tiles = std::min(p.tiles, 2 * M * G / 129);
  const int64_t tiles = std::max<int64_t>(1, p.tiles * c->n_kv_heads);
  p.chunk_many = chunk_of(max_len, std::min((kCUs + tiles - 1) / tiles, max_len / kMinMany),
                          kManyKeys);
  if (M >= (1 << 23)) p.chunk_many = chunk_of(max_len, 1, kManyKeys);  // (a grid of M workgroups)
  p.teams = tiles > 3 * kCUs ? 1 : 2;
  const int64_t full = std::max<int64_t>(0, M - c->n_seq) * n_heads / kManyCols;
  p.both = p.few && p.tiles > 0 && (p.teams == 1 || 2 * (int64_t)c->n_seq * c->n_kv_heads > full) &&
           tiles + 8 * wgs < (1 << 23);  // (threads of a grid: 2^31)
  int chunk = p.chunk_few;
  if (p.many) chunk = p.few ? std::min(chunk, p.chunk_many) : p.chunk_many;
  p.splits = (int)std::max<int64_t>(1, (max_len + chunk - 1) / chunk);
  return p;
}

static int64_t partial_bytes(int64_t M, int n_heads, int head_dim, int64_t splits) {
  return splits > 1 ? M * n_heads * splits * (head_dim + 2) * 4 : 0;
}

static pipo_status check_attn(const char* what, const pipo_kv_pages* c, int32_t n_heads, int64_t M,
                              int32_t max_q, int32_t max_len) {
  if (n_heads < 1 || n_heads % c->n_kv_heads != 0 || M < 0 || max_q < 0 || max_len < 0 ||
      max_len > c->table_stride * c->page_size) {
    set_error("%s: %d query heads over %d, %lld rows, up to %d a sequence, %d keys of %lld", what,
              n_heads, c->n_kv_heads, (long long)M, max_q, max_len,
              (long long)(c->table_stride * c->page_size));
    return PIPO_ERR_ARG;
  }
  const int64_t cols = std::min<int64_t>(max_q, M) * (n_heads / c->n_kv_heads);
  if (M * n_heads >= ((int64_t)1 << 30) || n_heads > 65535 || c->n_seq > 65535 ||
      (int64_t)c->n_seq * c->n_kv_heads >= ((int64_t)1 << 22) || max_len > (1 << 30) ||
      (cols + kManyCols - 1) / kManyCols * c->n_kv_heads >= ((int64_t)1 << 22)) {
    set_error("%s: %lld rows of %d heads, %d sequences of %d keys", what, (long long)M, n_heads,
              c->n_seq, max_len);
    return PIPO_ERR_UNSUPPORTED;
  }
  return PIPO_OK;
}

template <int D>
static void launch_attn_pages(const AttnPages& a, const Plan& p, hipStream_t st) {
  const auto splits = [&](int chunk) {
    return (unsigned)std::max(1, (a.max_len + chunk - 1) / chunk);
  };
  const int64_t cols = std::min<int64_t>((int64_t)a.max_q * a.G, kFewCols);
  const int64_t tile = p.pack ? kPackCols : 16, col_tiles_few = (cols + tile - 1) / tile;
  // Few columns: sequences fastest, so that workgroups with nothing to do (columns and
  // splits that shorter ones lack) come in a row: workgroups go to the shader engines
  // by turns, and with the column tiles of a sequence side by side those with work all
  // went to one engine in four (28 sequences of 2100 keys among up to 16 rows: 63.8
  // us, 23 without)
  if (p.both) {
    const int many = (int)(a.c.Hkv * p.tiles);
    const dim3 g((unsigned)(many * splits(a.chunk_many) +
                            a.c.Hkv * a.c.n_seq * splits(a.chunk_few) * col_tiles_few));
    const auto go = [&](auto kernel) {
      launch(kernel, g, dim3(256), 0, st, a, many, (int)splits(a.chunk_many),
             (int)splits(a.chunk_few));
    };
    p.pack ? go(attn_pages_both_k<D, 2>) : go(attn_pages_both_k<D, 1>);
  } else if (p.few) {
    const dim3 g((unsigned)(a.c.Hkv * a.c.n_seq), splits(a.chunk_few), (unsigned)col_tiles_few);
    const auto go = [&](auto kernel) { launch(kernel, g, dim3(64 * p.waves), 0, st, a); };
    if (p.waves == 8)
      p.pack ? go(attn_pages_few_k<D, 8, 2>) : go(attn_pages_few_k<D, 8, 1>);
    else if (p.waves == 4)
      p.pack ? go(attn_pages_few_k<D, 4, 2>) : go(attn_pages_few_k<D, 4, 1>);
    else
      p.pack ? go(attn_pages_few_k<D, 2, 2>) : go(attn_pages_few_k<D, 2, 1>);
  }
  if (p.many && p.tiles > 0 && !p.both) {
    const dim3 g((unsigned)(a.c.Hkv * p.tiles), splits(a.chunk_many));
    if (p.teams == 2)
      launch(attn_pages_many_k<D, 2>, g, dim3(512), 0, st, a);
    else
      launch(attn_pages_many_k<D, 1>, g, dim3(256), 0, st, a);
  }
  const auto merge = [&](auto few_c, int chunk, int64_t rows, int few_rows) {
    constexpr bool FEW = decltype(few_c)::value;
    const unsigned n = splits(chunk);
    if (n > kSmallMerge)
      launch(attn_pages_merge_k<D, kMaxSplits, FEW>, dim3((unsigned)rows, (unsigned)a.H), dim3(256), 0,
             st, a, few_rows);
    else if (n > 1)
      launch(attn_pages_merge_k<D, kSmallMerge, FEW>, dim3((unsigned)rows, (unsigned)((a.H + 3) / 4)),
             dim3(256), 0, st, a, few_rows);
  };
  if (p.few) {
    const int few_rows = std::max(1, std::min(a.max_q, kFewCols / a.G));
    merge(std::true_type{}, a.chunk_few, (int64_t)a.c.n_seq * few_rows, few_rows);
  }
  if (p.many && p.tiles > 0) merge(std::false_type{}, a.chunk_many, a.M, 0);
}

}  // namespace pipo

using namespace pipo;

extern "C" {

int64_t pipo_op_attn_pages_workspace_bytes(const pipo_kv_pages* c, int32_t n_heads, int64_t M,
                                           int32_t max_q, int32_t max_len) {
  if (!c || pipo_kv_page_bytes(c->page_size, c->n_kv_heads, c->head_dim) == 0 || c->n_seq < 1 ||
      max_q < 1 || max_len < 1 || M < 1 ||
      check_attn("attn_pages", c, n_heads, M, max_q, max_len) != PIPO_OK)
    return 0;
  return partial_bytes(M, n_heads, c->head_dim,
                       plan_attn(c, n_heads, M, std::min<int64_t>(max_q, M), max_len).splits);
}

pipo_status pipo_op_attn_pages(const pipo_kv_pages* c, int32_t layer, const uint16_t* q, int64_t ldq,
                               const int32_t* q_start, const int32_t* kv_len, uint16_t* o,
                               int64_t ldo, int32_t n_heads, int64_t M, int32_t max_q,
                               int32_t max_len, void* workspace, int64_t workspace_bytes,
                               void* stream) {
  clear_error();
  AttnPages a;
  PIPO_TRY(check_pages("attn_pages", c, layer, &a.c));
  PIPO_TRY(check_attn("attn_pages", c, n_heads, M, max_q, max_len));
  const int64_t d = (int64_t)n_heads * c->head_dim;
  if (!q || !q_start || !kv_len || !o || ldq < d || ldo < d || workspace_bytes < 0) {
    set_error("attn_pages: NULL pointer, rows (%lld, %lld) shorter than %lld, or negative "
              "workspace size", (long long)ldq, (long long)ldo, (long long)d);
    return PIPO_ERR_ARG;
  }
  if (M == 0 || max_q == 0) return PIPO_OK;
  a.q = q;
  a.o = o;
  a.q_start = q_start;
  a.kv_len = kv_len;
  a.part = static_cast<float*>(workspace);
  a.ldq = ldq;
  a.ldo = ldo;
  a.M = M;
  a.H = n_heads;
  a.G = n_heads / c->n_kv_heads;
  a.max_q = (int)std::min<int64_t>(max_q, M);
  a.max_len = max_len;
  Plan p = plan_attn(c, n_heads, M, a.max_q, max_len);
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 16 != 0 ||
      workspace_bytes < partial_bytes(M, n_heads, c->head_dim, p.splits)) {
    p.chunk_few = p.chunk_many = std::max(128, (max_len + 127) / 128 * 128);
    p.splits = 1;
  }
  a.few_cols = p.few ? kFewCols : 0;
  a.chunk_few = p.chunk_few;
  a.chunk_many = p.chunk_many;
  a.splits = p.splits;
  a.part_rl = reinterpret_cast<float2*>(a.part + M * n_heads * a.splits * c->head_dim);
  a.q_vec = reinterpret_cast<uintptr_t>(q) % 16 == 0 && ldq % 8 == 0;
  a.o_vec = reinterpret_cast<uintptr_t>(o) % 8 == 0 && ldo % 4 == 0;
  const auto go = c->head_dim == 128 ? launch_attn_pages<128> : launch_attn_pages<64>;
  go(a, p, static_cast<hipStream_t>(stream));
  PIPO_HIP_TRY(hipGetLastError());
  return PIPO_OK;
}

}  // extern "C"
