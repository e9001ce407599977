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
  int chunk;                  // keys of a split
  int splits;                 // of a row's partials in `part`
  bool q_vec, o_vec;          // q rows 16-byte aligned, o rows 8-byte
};

constexpr int kBlockKeys = 32;
constexpr int kMaxSplits = 64;  // a wave's lanes, in attn_pages_merge_k
constexpr float kLog2e = 1.4426950408889634f;
// p is held times 2^15 / (a bound of the values' scales), so that p s fits a half
constexpr float kPBits = 15.f;

// a sequence's rows [row0, row0 + nq) and keys
struct Seq {
  int row0, nq, len;
};
__device__ __forceinline__ Seq sequence(const AttnPages& a, int i) {
  Seq s;
  const int64_t r0 = min(max((int64_t)a.q_start[i], (int64_t)0), a.M);
  const int64_t r1 = min(max((int64_t)a.q_start[i + 1], r0), a.M);
  s.row0 = (int)r0;
  s.nq = (int)(r1 - r0);
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
// a word of K codes -> eight dimensions in order, each 256 + c (dimensions 0,
// 1, 4, 5) or 16 + c
__device__ __forceinline__ h8 k_codes(uint32_t w, const Magic& g) {
  const uint32_t a = w << 2, b = w >> 6;
  u32x4 o;
  o[0] = (a & g.m256) | g.e256;
  o[1] = (a & g.m16) | g.e16;
  o[2] = (b & g.m256) | g.e256;
  o[3] = (b & g.m16) | g.e16;
  return __builtin_bit_cast(h8, o);
}
constexpr float kKBias(int j) { return (j / 2) % 2 ? 16.f : 256.f; }
// V words of two tiles -> the eight keys' codes of dimension 32 w + r (half 0:
// 256 + c) or 32 w + 16 + r (half 1: 16 + c); key order 0, 2, 1, 3 in each tile
constexpr float kVBias(int half) { return half ? 16.f : 256.f; }
template <int HALF>
__device__ __forceinline__ h8 v_codes(uint32_t w0, uint32_t w1, const Magic& g) {
  const uint32_t m = HALF ? g.m16 : g.m256, e = HALF ? g.e16 : g.e256;
  u32x4 o;
  o[0] = ((w0 << 2) & m) | e;
  o[1] = ((w0 >> 6) & m) | e;
  o[2] = ((w1 << 2) & m) | e;
  o[3] = ((w1 >> 6) & m) | e;
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

// A workgroup is W waves on (sequence, key/value head, 16 columns,
// split) that take the split's keys by turns, 32 at a time, from the cache into
// operand registers.
template <int D, int W>
__global__ __launch_bounds__(W * 64) __attribute__((amdgpu_waves_per_eu(3))) void
attn_pages_k(AttnPages a) {
  constexpr int KK = D / 32, NG = D / 64, NF = D / 16;
  const int kh = blockIdx.x % a.c.Hkv, ct = blockIdx.x / a.c.Hkv, sp = blockIdx.y;
  const int si = blockIdx.z;
  const Seq s = sequence(a, si);
  const int cols = s.nq * a.G;
  if (16 * ct >= cols) return;
  const int ns = max(1, (s.len + a.chunk - 1) / a.chunk);
  if (sp >= ns) return;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = lane & 15, g = lane >> 4;
  const Magic mg = magic();
  // two blocks a wave; the waves' sums at the end
  constexpr int BLK = 2 * kTileBytes<D>, ROW = D + 4;
  static_assert(16 * ROW * 4 <= 2 * BLK, "a wave's sums fit its blocks");
  __shared__ __attribute__((aligned(1024))) uint8_t lds[W * 2 * BLK];
  __shared__ float lR[W][16], ll[W][16];
  uint8_t* const ring = lds + wave * (2 * BLK);
  const uint32_t ring_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)ring;

  // this lane's column: keys [0, vis) are visible
  const int col = 16 * ct + r, qj = col / a.G, h = kh * a.G + col % a.G;
  const int vis = col < cols ? max(0, s.len - s.nq + qj + 1) : 0;
  const int jmin = 16 * ct / a.G, jmax = min(s.nq - 1, (16 * ct + 15) / a.G);
  const int all = max(0, s.len - s.nq + jmin + 1);      // visible to every column
  const int end = max(0, s.len - s.nq + jmax + 1);      // to any
  const int p0 = sp * a.chunk, p1 = min(end, p0 + a.chunk);

  f4 acc[NF];
#pragma unroll
  for (int n = 0; n < NF; ++n) acc[n] = f4{0.f, 0.f, 0.f, 0.f};
  float R = -INFINITY, l = 0.f, msum[NG] = {};  // sums of p and p m
  f4 psum[NG];                                  // of p s, in every element
#pragma unroll
  for (int n = 0; n < NG; ++n) psum[n] = f4{0.f, 0.f, 0.f, 0.f};
  const h8 ones = h8(1);

  // the wave's blocks are p0 + 32 (wave + W i); lane 2 i + j holds the page of
  // tile j of block i, 32 blocks at a time
  const int32_t* row = a.c.table + si * a.c.stride;
  const int step = W * kBlockKeys;
  int pages = -1, block = 32;
  uint32_t valid = 0;  // bit 2 s + j: tile j in slot s is a page's
  const auto issue = [&](int p, int slot) {
    if (block == 32) {
      block = 0;
      const int64_t pos = (int64_t)p + (lane >> 1) * step + 16 * (lane & 1);
      pages = pos < p1 ? row[pos >> a.c.ps_log2] : -1;
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int page = __builtin_amdgcn_readlane(pages, 2 * block + j);
      const bool ok = page >= 0 && page < a.c.n_pages;
      valid = (valid & ~(1u << (2 * slot + j))) | ((uint32_t)ok << (2 * slot + j));
      issue_tile<D>(tile_at<D>(a.c, ok ? page : 0, kh, p + 16 * j),
                    ring + slot * BLK + j * kTileBytes<D>, lane);
    }
    ++block;
  };

  int p = p0 + wave * kBlockKeys, slot = 0;
  if (p < p1) issue(p, 0);
  if (p + step < p1) issue(p + step, 1);

  h8 qf[KK];
  float qsum[NG], qbias[NG];  // of the column's q, and times the codes' bias
#pragma unroll
  for (int n = 0; n < NG; ++n) {
    float bias = 0.f, sum = 0.f;
#pragma unroll
    for (int kk = 2 * n; kk < 2 * n + 2; ++kk) {
      qf[kk] = col < cols ? load_q<D>(a, s.row0 + qj, h, 32 * kk + 8 * g) : zero_h8();
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        sum += (float)qf[kk][j];
        bias += kKBias(j) * (float)qf[kk][j];
      }
    }
    qsum[n] = cols_sum(sum);
    qbias[n] = cols_sum(bias);
  }

  const auto compute = [&](int p, int slot, auto edge_c) {
    constexpr bool EDGE = decltype(edge_c)::value;
    const uint32_t codes = ring_at + slot * BLK + lane * (D / 8), scales = ring_at + slot * BLK + g * (D / 4);
    // keys of the tiles that exist
    const int l0 = valid >> (2 * slot) & 1 ? p1 - p : 0;
    const int l1 = valid >> (2 * slot + 1) & 1 ? p1 - p - 16 : 0;
    float x[2][4], bm = -INFINITY;
    Part<D> t;
    read_part<D, 0, 16 * D>(t, codes, scales);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      f4 sc[NG];
#pragma unroll
      for (int n = 0; n < NG; ++n) {
        sc[n] = mfma16(k_codes(t.c[j][2 * n], mg), qf[2 * n], f4{0.f, 0.f, 0.f, 0.f});
        sc[n] = mfma16(k_codes(t.c[j][2 * n + 1], mg), qf[2 * n + 1], sc[n]);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float v = 0.f;
#pragma unroll
        for (int n = 0; n < NG; ++n) {
          const uint32_t w = t.pair[j][e * NG + n];
          v = n == 0 ? lo_half(w) * qsum[0] : __builtin_fmaf(lo_half(w), qsum[n], v);
          v = __builtin_fmaf(hi_half(w), sc[n][e] - qbias[n], v);
        }
        if constexpr (EDGE) {
          const int key = 4 * g + e;
          v = key < (j ? l1 : l0) && p + 16 * j + key < vis ? v : -INFINITY;
        }
        x[j][e] = v;
        bm = fmaxf(bm, v);
      }
    }
    uint32_t top = 0;
    read_part<D, 8 * D, 17 * D>(t, codes, scales);
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int n = 0; n < NG; ++n) {
          uint32_t& w = t.pair[j][e * NG + n];
          if constexpr (EDGE) w = 4 * g + e < (j ? l1 : l0) ? w : 0u;  // past the end: anything
          top = max(top, w);
        }
    bm = cols_max(bm);
    // scales are below 2^(exponent field - 14)
    const float es = cols_max((float)((int)(top >> 26) - 14));
    const float Rn = fmaxf(R, __builtin_fmaf(bm, kLog2e, es));
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
        const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(x[j][e], kLog2e, shift));
        l += y;
#pragma unroll
        for (int n = 0; n < NG; ++n) {
          const uint32_t w = t.pair[j][e * NG + n];
          // p s in two halves, 22 bits of it
          const float ys = y * hi_half(w);
          const _Float16 a16 = (_Float16)ys;
          hi[n][4 * j + kOrder[e]] = a16;
          lo[n][4 * j + kOrder[e]] = (_Float16)(ys - (float)a16);
          msum[n] = __builtin_fmaf(y, lo_half(w), msum[n]);
        }
      }
#pragma unroll
    for (int n = 0; n < NG; ++n) {
      psum[n] = mfma16(ones, hi[n], psum[n]);
      psum[n] = mfma16(ones, lo[n], psum[n]);
    }
#pragma unroll
    for (int w = 0; w < KK; ++w) {
      const int n = w / 2;
      const h8 v0 = v_codes<0>(t.c[0][w], t.c[1][w], mg),
               v1 = v_codes<1>(t.c[0][w], t.c[1][w], mg);
      acc[2 * w] = mfma16(v0, hi[n], acc[2 * w]);
      acc[2 * w] = mfma16(v0, lo[n], acc[2 * w]);
      acc[2 * w + 1] = mfma16(v1, hi[n], acc[2 * w + 1]);
      acc[2 * w + 1] = mfma16(v1, lo[n], acc[2 * w + 1]);
    }
  };

  // first the blocks that every column sees whole, up to one without a page
  const auto run = [&](auto edge_c) {
    constexpr bool EDGE = decltype(edge_c)::value;
    for (; p < p1; p += step, slot ^= 1) {
      if (!EDGE && (p + kBlockKeys > all || (valid >> (2 * slot) & 3) != 3)) return;
      if (p + step < p1)  // this block has landed, the next may still travel
        __builtin_amdgcn_s_waitcnt(waitcnt_imm(2 * kTileLoads<D>, false));
      else
        __builtin_amdgcn_s_waitcnt(waitcnt_imm(0, false));
      __builtin_amdgcn_sched_barrier(0);
      compute(p, slot, edge_c);
      __builtin_amdgcn_sched_barrier(0);  // (the slot is read)
      if (p + 2 * step < p1) issue(p + 2 * step, slot);
    }
  };
  run(std::false_type{});
  run(std::true_type{});

  // merge the waves: element e of acc[n] is dimension 16 n + 4 g + e of column r
  l = cols_sum(l);
#pragma unroll
  for (int n = 0; n < NG; ++n) msum[n] = cols_sum(msum[n]);
#pragma unroll
  for (int n = 0; n < NF; ++n) {
    f4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = acc[n][e] + (msum[n / 4] - kVBias(n % 2) * psum[n / 4][0]);
    *reinterpret_cast<f4*>(reinterpret_cast<float*>(ring) + r * ROW + 16 * n + 4 * g) = v;
  }
  if (g == 0) {
    lR[wave][r] = R;
    ll[wave][r] = l;
  }
  __syncthreads();
  for (int c = tid; c < 16 * D; c += W * 64) {
    const int cr = c / D, dim = c % D, cc = 16 * ct + cr;
    if (cc >= cols) break;
    float Rm = lR[0][cr];
#pragma unroll
    for (int w = 1; w < W; ++w) Rm = fmaxf(Rm, lR[w][cr]);
    const float Rs = Rm == -INFINITY ? 0.f : Rm;
    float A = 0.f, L = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float f = __builtin_amdgcn_exp2f(lR[w][cr] - Rs);
      A = __builtin_fmaf(reinterpret_cast<const float*>(lds + w * (2 * BLK))[cr * ROW + dim], f, A);
      L = __builtin_fmaf(ll[w][cr], f, L);
    }
    put<D>(a, s, kh * a.G + cc % a.G, s.row0 + cc / a.G, sp, ns, dim, A, Rm, L);
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
// in order.
template <int D>
__global__ __launch_bounds__(256) void attn_pages_merge_k(AttnPages a) {
  constexpr int LANES = D / 4, GROUPS = 256 / LANES, EACH = (kMaxSplits + GROUPS - 1) / GROUPS;
  const int m = blockIdx.x, h = blockIdx.y;
  const int i = seq_of_row(a, m);
  if (i < 0) return;
  const Seq s = sequence(a, i);
  const int ns = max(1, (s.len + a.chunk - 1) / a.chunk);
  if (ns == 1 || m - s.row0 >= a.max_q) return;
  const int64_t at = ((int64_t)m * a.H + h) * a.splits;
  const int tid = threadIdx.x, lane = tid & 63, grp = tid / LANES, dim = 4 * (tid % LANES);
  f4 x[EACH];
#pragma unroll
  for (int j = 0; j < EACH; ++j)
    if (grp + j * GROUPS < ns)
      x[j] = *reinterpret_cast<const f4*>(a.part + (at + grp + j * GROUPS) * D + dim);
  const float2 rl = lane < ns ? a.part_rl[at + lane] : make_float2(-INFINITY, 0.f);
  float R = rl.x, w = 0.f, L = 0.f;
#pragma unroll
  for (int d = 32; d >= 1; d /= 2) R = fmaxf(R, wave_shfl_xor(R, d));
  if (R != -INFINITY) w = __builtin_amdgcn_exp2f(rl.x - R);
  L = rl.y * w;
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
  __shared__ f4 sum[GROUPS][LANES];
  sum[grp][tid % LANES] = A;
  __syncthreads();
  if (tid >= D) return;
  float v = 0.f;
  for (int k = 0; k < GROUPS; ++k) v += sum[k][tid / 4][tid % 4];
  a.o[(int64_t)m * a.ldo + (int64_t)h * D + tid] = f2h(L > 0.f ? v / L : (L == L ? 0.f : L));
}

// Splits: workgroups for the whole chip where the sequences' columns alone are
// too few, at least 256 keys each.
constexpr int kWantWGs = 1024, kMinChunk = 256;

static int64_t col_tiles(int64_t max_q, int G) { return (max_q * G + 15) / 16; }

static int split_chunk(const pipo_kv_pages* c, int n_heads, int64_t max_q, int64_t max_len) {
  const int64_t wgs = (int64_t)c->n_seq * c->n_kv_heads * col_tiles(max_q, n_heads / c->n_kv_heads);
  int64_t S = std::min<int64_t>((kWantWGs + wgs - 1) / wgs, kMaxSplits);
  S = std::max<int64_t>(1, std::min(S, max_len / kMinChunk));
  return (int)(((max_len + S - 1) / S + 127) / 128 * 128);
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
  if (M * n_heads >= ((int64_t)1 << 31) || (int64_t)max_q * n_heads >= ((int64_t)1 << 31) ||
      n_heads > 65535 || c->n_seq > 65535 || max_len > (1 << 30)) {
    set_error("%s: %lld rows of %d heads, %d sequences of %d keys", what, (long long)M, n_heads,
              c->n_seq, max_len);
    return PIPO_ERR_UNSUPPORTED;
  }
  return PIPO_OK;
}

template <int D>
static void launch_attn_pages(const AttnPages& a, hipStream_t st) {
  const dim3 grid((unsigned)(a.c.Hkv * col_tiles(a.max_q, a.G)), (unsigned)a.splits,
                  (unsigned)a.c.n_seq);
  launch(attn_pages_k<D, 4>, grid, dim3(256), 0, st, a);
  if (a.splits > 1)
    launch(attn_pages_merge_k<D>, dim3((unsigned)a.M, (unsigned)a.H), dim3(256), 0, st, a);
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
  const int chunk = split_chunk(c, n_heads, std::min<int64_t>(max_q, M), max_len);
  return partial_bytes(M, n_heads, c->head_dim, (max_len + chunk - 1) / chunk);
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
  a.chunk = split_chunk(c, n_heads, a.max_q, max_len);
  a.splits = std::max(1, (max_len + a.chunk - 1) / a.chunk);
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 16 != 0 ||
      workspace_bytes < partial_bytes(M, n_heads, c->head_dim, a.splits)) {
    a.chunk = (max_len + 127) / 128 * 128;
    a.splits = 1;
  }
  a.chunk = std::max(a.chunk, 128);
  a.part_rl = reinterpret_cast<float2*>(a.part + M * n_heads * a.splits * c->head_dim);
  a.q_vec = reinterpret_cast<uintptr_t>(q) % 16 == 0 && ldq % 8 == 0;
  a.o_vec = reinterpret_cast<uintptr_t>(o) % 8 == 0 && ldo % 4 == 0;
  const auto go = c->head_dim == 128 ? launch_attn_pages<128> : launch_attn_pages<64>;
  go(a, static_cast<hipStream_t>(stream));
  PIPO_HIP_TRY(hipGetLastError());
  return PIPO_OK;
}

}  // extern "C"
