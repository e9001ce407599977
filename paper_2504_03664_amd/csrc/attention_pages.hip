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

#include "attention_common.h"
#include "kvpages.h"

namespace pipo {

struct AttnPages {
  PagesView c;
  const uint16_t* q;
  uint16_t* o;
  const int32_t *q_start, *kv_len;
  float* part;
  int64_t ldq, ldo, M;
  int H, G, max_q, max_len;
  int chunk;                  // keys of a split
  int splits;                 // of a row's partials in `part`
  bool q_vec, o_vec;          // q rows 16-byte aligned, o rows 8-byte
};

constexpr int kBlockKeys = 32;
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
constexpr float kVBias = 16.f;
// V words of two tiles -> the eight keys' codes, 16 + c, of dimension 32 w + r
// (half 0) or 32 w + 16 + r; key order 0, 2, 1, 3 in each tile
template <int HALF>
__device__ __forceinline__ h8 v_codes(uint32_t w0, uint32_t w1, const Magic& g) {
  u32x4 o;
  o[0] = ((HALF ? w0 << 2 : w0 << 6) & g.m16) | g.e16;
  o[1] = ((HALF ? w0 >> 6 : w0 >> 2) & g.m16) | g.e16;
  o[2] = ((HALF ? w1 << 2 : w1 << 6) & g.m16) | g.e16;
  o[3] = ((HALF ? w1 >> 6 : w1 >> 2) & g.m16) | g.e16;
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

// what a lane holds of a tile: K and V codes (operand words), the pairs of keys
// 4 g .. 4 g + 3
template <int D>
struct Tile {
  uint32_t k[D / 32], v[D / 32], kp[D / 16], vp[D / 16];
};
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
template <int D>
__device__ __forceinline__ void load_tile(Tile<D>& t, const uint8_t* p, int lane) {
  load_words(t.k, p + lane * (D / 8));
  load_words(t.v, p + 8 * D + lane * (D / 8));
  load_words(t.kp, p + 16 * D + (lane >> 4) * (D / 4));
  load_words(t.vp, p + 17 * D + (lane >> 4) * (D / 4));
}

// result of column r of a tile of 16 columns: straight to o, or a partial
template <int D>
__device__ __forceinline__ void put(const AttnPages& a, const Seq& s, int h, int row, int sp, int ns,
                                    int dim, float acc, float R, float l) {
  if (ns == 1) {
    a.o[(int64_t)row * a.ldo + (int64_t)h * D + dim] = f2h(l > 0.f ? acc / l : (l == l ? 0.f : l));
  } else {
    float* pp = a.part + (((int64_t)row * a.H + h) * a.splits + sp) * (D + 2);
    pp[dim] = acc;
    if (dim == 0) {
      pp[D] = R;
      pp[D + 1] = l;
    }
  }
}

// A workgroup is W waves on (sequence, key/value head, 16 columns,
// split) that take the split's keys by turns, 32 at a time, from the cache into
// operand registers.
template <int D, int W>
__global__ __launch_bounds__(W * 64) void attn_pages_k(AttnPages a) {
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

  // this lane's column: keys [0, vis) are visible
  const int col = 16 * ct + r, qj = col / a.G, h = kh * a.G + col % a.G;
  const int vis = col < cols ? max(0, s.len - s.nq + qj + 1) : 0;
  const int jmin = 16 * ct / a.G, jmax = min(s.nq - 1, (16 * ct + 15) / a.G);
  const int all = max(0, s.len - s.nq + jmin + 1);      // visible to every column
  const int end = max(0, s.len - s.nq + jmax + 1);      // to any
  const int p0 = sp * a.chunk, p1 = min(end, p0 + a.chunk);

  h8 qf[KK];
  f4 init[NG];
  float qsum[NG];
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
    bias = cols_sum(bias);
    init[n] = f4{-bias, -bias, -bias, -bias};
  }

  f4 acc[NF];
#pragma unroll
  for (int n = 0; n < NF; ++n) acc[n] = f4{0.f, 0.f, 0.f, 0.f};
  float R = -INFINITY, l = 0.f, corr[NG] = {};
  const int32_t* row = a.c.table + si * a.c.stride;

  for (int p = p0 + wave * kBlockKeys; p < p1; p += W * kBlockKeys) {
    Tile<D> t[2];
    int lim[2];  // keys of the tile that exist
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int pos = p + 16 * j;
      int page = pos < p1 ? row[pos >> a.c.ps_log2] : -1;
      const bool ok = page >= 0 && page < a.c.n_pages;
      lim[j] = ok ? p1 - pos : 0;
      load_tile<D>(t[j], tile_at<D>(a.c, ok ? page : 0, kh, pos), lane);
    }
    const bool edge = p + kBlockKeys > min(all, p1) || lim[0] < 16 || lim[1] < 16;
    if (edge) {  // what lies past the end may be anything
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (4 * g + e >= lim[j])
#pragma unroll
            for (int n = 0; n < NG; ++n) t[j].kp[e * NG + n] = t[j].vp[e * NG + n] = 0;
    }
    float x[2][4], bm = -INFINITY;
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      f4 sc[NG];
#pragma unroll
      for (int n = 0; n < NG; ++n) {
        sc[n] = init[n];
#pragma unroll
        for (int kk = 2 * n; kk < 2 * n + 2; ++kk)
          sc[n] = mfma16(k_codes(t[j].k[kk], mg), qf[kk], sc[n]);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float v = 0.f;
#pragma unroll
        for (int n = 0; n < NG; ++n) {
          const uint32_t w = t[j].kp[e * NG + n];
          v = __builtin_fmaf(lo_half(w), qsum[n], v);
          v = __builtin_fmaf(hi_half(w), sc[n][e], v);
          top = max(top, t[j].vp[e * NG + n]);
        }
        if (edge && (4 * g + e >= lim[j] || p + 16 * j + 4 * g + e >= vis)) v = -INFINITY;
        x[j][e] = v;
        bm = fmaxf(bm, v);
      }
    }
    bm = cols_max(bm);
    // scales are below 2^(exponent field - 14)
    const float es = cols_max((float)((int)(top >> 26) - 14));
    const float Rn = fmaxf(R, __builtin_fmaf(bm, kLog2e, es));
    const float Rs = Rn == -INFINITY ? 0.f : Rn;
    const float alpha = __builtin_amdgcn_exp2f(R - Rs);
    R = Rn;
    l *= alpha;
#pragma unroll
    for (int n = 0; n < NG; ++n) corr[n] *= alpha;
    if (__any(alpha != 1.f)) {
#pragma unroll
      for (int n = 0; n < NF; ++n) acc[n] *= alpha;
    }
    h8 hi[NG], lo[NG];
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        constexpr int kOrder[4] = {0, 2, 1, 3};  // of v_codes
        const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(x[j][e], kLog2e, kPBits - Rs));
        l += y;
#pragma unroll
        for (int n = 0; n < NG; ++n) {
          const uint32_t w = t[j].vp[e * NG + n];
          const float sv = hi_half(w);
          // p s in two halves: 22 bits of it
          const _Float16 a16 = (_Float16)(y * sv);
          hi[n][4 * j + kOrder[e]] = a16;
          lo[n][4 * j + kOrder[e]] = (_Float16)__builtin_fmaf(y, sv, -(float)a16);
          corr[n] = __builtin_fmaf(y, __builtin_fmaf(sv, -kVBias, lo_half(w)), corr[n]);
        }
      }
#pragma unroll
    for (int w = 0; w < KK; ++w) {
      const int n = w / 2;
      const h8 v0 = v_codes<0>(t[0].v[w], t[1].v[w], mg), v1 = v_codes<1>(t[0].v[w], t[1].v[w], mg);
      acc[2 * w] = mfma16(v0, hi[n], acc[2 * w]);
      acc[2 * w] = mfma16(v0, lo[n], acc[2 * w]);
      acc[2 * w + 1] = mfma16(v1, hi[n], acc[2 * w + 1]);
      acc[2 * w + 1] = mfma16(v1, lo[n], acc[2 * w + 1]);
    }
  }

  // merge the waves: element e of acc[n] is dimension 16 n + 4 g + e of column r
  __shared__ float lacc[W][16][D + 4], lR[W][16], ll[W][16];
  l = cols_sum(l);
#pragma unroll
  for (int n = 0; n < NG; ++n) corr[n] = cols_sum(corr[n]);
#pragma unroll
  for (int n = 0; n < NF; ++n) {
    f4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = acc[n][e] + corr[n / 4];
    *reinterpret_cast<f4*>(&lacc[wave][r][16 * n + 4 * g]) = v;
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
      A = __builtin_fmaf(lacc[w][cr][dim], f, A);
      L = __builtin_fmaf(ll[w][cr], f, L);
    }
    put<D>(a, s, kh * a.G + cc % a.G, s.row0 + cc / a.G, sp, ns, dim, A, Rm, L);
  }
}

// sequence that holds row m (-1: none)
__device__ __forceinline__ int seq_of_row(const AttnPages& a, int m) {
  int lo = 0, hi = a.c.n_seq;  // q_start[lo] <= m < q_start[hi]
  if (m < a.q_start[0] || m >= a.q_start[hi]) return -1;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (a.q_start[mid] <= m)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

// adds the splits of a row's head in order
template <int D>
__global__ __launch_bounds__(D) void attn_pages_merge_k(AttnPages a) {
  const int m = blockIdx.x, h = blockIdx.y;
  const int i = seq_of_row(a, m);
  if (i < 0) return;
  const Seq s = sequence(a, i);
  const int ns = max(1, (s.len + a.chunk - 1) / a.chunk);
  if (ns == 1 || m - s.row0 >= a.max_q) return;
  const float* part = a.part + ((int64_t)m * a.H + h) * a.splits * (D + 2);
  float R = -INFINITY;
  for (int k = 0; k < ns; ++k) R = fmaxf(R, part[k * (D + 2) + D]);
  const float Rs = R == -INFINITY ? 0.f : R;
  float A = 0.f, L = 0.f;
  for (int k = 0; k < ns; ++k) {
    const float* p = part + k * (D + 2);
    const float f = __builtin_amdgcn_exp2f(p[D] - Rs);
    A = __builtin_fmaf(p[threadIdx.x], f, A);
    L = __builtin_fmaf(p[D + 1], f, L);
  }
  a.o[(int64_t)m * a.ldo + (int64_t)h * D + threadIdx.x] =
      f2h(L > 0.f ? A / L : (L == L ? 0.f : L));
}

// Splits: workgroups for the whole chip where the sequences' columns alone are
// too few, at least 256 keys each.
constexpr int kWantWGs = 1024, kMinChunk = 256, kMaxSplits = 64;

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
    launch(attn_pages_merge_k<D>, dim3((unsigned)a.M, (unsigned)a.H), dim3(D), 0, st, a);
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
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 4 != 0 ||
      workspace_bytes < partial_bytes(M, n_heads, c->head_dim, a.splits)) {
    a.chunk = (max_len + 127) / 128 * 128;
    a.splits = 1;
  }
  a.chunk = std::max(a.chunk, 128);
  a.q_vec = reinterpret_cast<uintptr_t>(q) % 16 == 0 && ldq % 8 == 0;
  a.o_vec = reinterpret_cast<uintptr_t>(o) % 8 == 0 && ldo % 4 == 0;
  const auto go = c->head_dim == 128 ? launch_attn_pages<128> : launch_attn_pages<64>;
  go(a, static_cast<hipStream_t>(stream));
  PIPO_HIP_TRY(hipGetLastError());
  return PIPO_OK;
}

}  // extern "C"
