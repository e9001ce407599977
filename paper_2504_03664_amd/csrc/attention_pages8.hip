// Attention over the pages of an 8-bit KV cache (layout in kvpages8.h), with what
// pipo_attn_scores asks of the scores: a cap, a bias by distance, a window, a prefix.
//
// The G query heads of a key/value head times a sequence's queries are columns
// (column c: query c / G, head c % G), 16 to a matrix product.  A block's keys are
// operands in units of their scale, which multiplies the scores in fp32, and its values
// as they are: code * scale is a half exactly.
#include <algorithm>
#include <type_traits>

#include "attention_common.h"
#include "kvpages8.h"

namespace pipo {

struct Attn8 {
  Pages8 c;
  const uint16_t* q;
  uint16_t* o;
  const int32_t *q_start, *kv_len, *prefix;
  const float* slopes;
  float* part;      // [row][head][split][D] sums and, behind them, their (R, l)
  float2* part_rl;
  int64_t ldq, ldo, M;
  int H, G, max_q, max_len, window, max_prefix;
  float cap;
  int chunk;        // keys of a split
  int splits;       // of a row's partials in `part`
  bool q_vec, o_vec;
};

constexpr int kBlock = 32;      // keys that a wave takes at a time
constexpr int kMaxSplits = 64;  // a wave's lanes, where they are joined
constexpr float kLog2e = 1.4426950408889634f;
// p is held times 2^14: as a half it keeps 11 bits down to 2^-28
constexpr float kPBits = 14.f;

// a sequence's rows [row0, row0 + nq), how many of them count (up to max_q), its keys
// and the ones that every row sees
struct Seq8 {
  int row0, nq, rows, len, pre;
};
__device__ __forceinline__ Seq8 sequence(const Attn8& a, int i) {
  Seq8 s;
  const int64_t r0 = min(max((int64_t)a.q_start[i], (int64_t)0), a.M);
  const int64_t r1 = min(max((int64_t)a.q_start[i + 1], r0), a.M);
  s.row0 = (int)r0;
  s.nq = (int)(r1 - r0);
  s.rows = min(s.nq, a.max_q);
  s.len = min(max(a.kv_len[i], 0), a.max_len);
  s.pre = a.prefix ? min(min(max(a.prefix[i], 0), a.max_prefix), s.len) : 0;
  return s;
}
// keys [lo, hi) that row j sees, and [0, pre)
struct Seen {
  int lo, hi;
};
__device__ __forceinline__ Seen seen_by(const Attn8& a, const Seq8& s, int j) {
  const int64_t after = (int64_t)s.len - s.nq + j + 1;
  Seen w;
  w.hi = (int)min(max(after, (int64_t)0), (int64_t)s.len);
  w.lo = a.window > 0 ? (int)min(max(after - a.window, (int64_t)0), (int64_t)s.len) : 0;
  return w;
}
// blocks that rows j0 .. j1 see: [0, head) and [from, from + n - head), n in all
struct Blocks {
  int head, from, n;
};
__device__ __forceinline__ Blocks blocks_of(const Attn8& a, const Seq8& s, int j0, int j1) {
  Blocks b;
  const int pre = (s.pre + kBlock - 1) / kBlock;
  b.from = seen_by(a, s, j0).lo / kBlock;
  b.head = min(pre, b.from);
  b.n = b.head + max(max(pre, (seen_by(a, s, j1).hi + kBlock - 1) / kBlock) - b.from, 0);
  return b;
}
__device__ __forceinline__ int splits_of(const Attn8& a, const Seq8& s) {
  const int n = s.rows > 0 ? blocks_of(a, s, 0, s.rows - 1).n : 0;
  return min(max(1, (int)(((int64_t)n * kBlock + a.chunk - 1) / a.chunk)), a.splits);
}

template <int D>
__device__ __forceinline__ h8 load_q(const Attn8& a, int64_t row, int head, int dim) {
  const uint16_t* p = a.q + row * a.ldq + (int64_t)head * D + dim;
  if (a.q_vec) return load_h8(p);
  h8 v;
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = __builtin_bit_cast(_Float16, p[j]);
  return v;
}

__device__ __forceinline__ float cols_max(float x) {  // over the four lanes of a column
  x = pair_max(__builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false));
  return pair_max(__builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
}
__device__ __forceinline__ float cols_sum(float x) {
  x = pair_sum(__builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false));
  return pair_sum(__builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
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

// what becomes of scores, in units of log 2
struct Scores {
  float cap_in, cap_out;   // 2 log2(e) / cap, cap log2(e); 0: no cap
};
__device__ __forceinline__ Scores scores_of(const Attn8& a) {
  return Scores{a.cap > 0.f ? 2.f * kLog2e / a.cap : 0.f, a.cap * kLog2e};
}
// cap tanh(x / cap) = cap - 2 cap / (exp(2 x / cap) + 1): off by a few 2^-24 of the cap, in a
// number whose exponential is taken
__device__ __forceinline__ float score(const Scores& f, float x, float slope, float far) {
  float y = x * kLog2e;
  if (f.cap_in > 0.f)
    y = __builtin_fmaf(-2.f * f.cap_out,
                       __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(x * f.cap_in) + 1.f), f.cap_out);
  return __builtin_fmaf(-slope, far, y);
}

// result of a column: straight to o, or a partial
template <int D>
__device__ __forceinline__ void put(const Attn8& a, int h, int row, int sp, int ns, int dim, float acc,
                                    float R, float l) {
  if (ns == 1) {
    a.o[(int64_t)row * a.ldo + (int64_t)h * D + dim] = f2h(l > 0.f ? acc / l : (l == l ? 0.f : l));
  } else {
    const int64_t at = ((int64_t)row * a.H + h) * a.splits + sp;
    a.part[at * D + dim] = acc;
    if (dim == 0) a.part_rl[at] = make_float2(R, l);
  }
}

// Few columns: a workgroup is W waves on (sequence, key/value head, 16 columns, split)
// that take the split's blocks of 32 keys by turns, straight into registers in operand
// order, the next block's loads under way while one is worked on.  Weights go to
// the second product as a high and a low half, 22 bits.
template <int D>
struct Block8 {
  u32x4 k[2][D / 64], v[2][D / 64];
  float ks[2], vs[2];
  bool ok[2];
};
template <int D, int W>
struct Few8Lds {
  float sums[W][16][D + 4];
  float R[W][16], l[W][16];
};

template <int D, bool INT8, bool MOD, int W>
__global__ __launch_bounds__(W * 64) __attribute__((amdgpu_waves_per_eu(2))) void attn8_few_k(Attn8 a) {
  constexpr int KK = D / 32, NF = D / 16, C = D / 64;
  __shared__ Few8Lds<D, W> lds;
  const int kh = blockIdx.x % a.c.Hkv, si = blockIdx.x / a.c.Hkv, sp = blockIdx.y, ct = blockIdx.z;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Seq8 s = sequence(a, si);
  const int cols = s.rows * a.G;
  if (16 * ct >= cols) return;
  const int ns = splits_of(a, s);
  if (sp >= ns) return;
  const int r = lane & 15, g = lane >> 4;

  // this lane's column, the keys it sees, and those that all columns see
  const int col = 16 * ct + r, qj = col / a.G, h = kh * a.G + col % a.G;
  Seen mine = Seen{0, 0};
  if (col < cols) mine = seen_by(a, s, qj);
  const int pre = col < cols ? s.pre : 0;
  const int at = s.len - s.nq + qj;   // its position
  const int j0 = 16 * ct / a.G, j1 = min(s.rows - 1, (16 * ct + 15) / a.G);
  const int all_lo = seen_by(a, s, j1).lo, all_hi = seen_by(a, s, j0).hi;
  const Blocks blocks = blocks_of(a, s, j0, j1);
  const int per = a.chunk / kBlock, b1 = (int)min((int64_t)blocks.n, (int64_t)(sp + 1) * per);
  int b = sp * per + wave;
  const auto key_of = [&](int b) { return kBlock * (b < blocks.head ? b : b - blocks.head + blocks.from); };

  // lane 2 i + j holds the page and the scales of tile j of the wave's i-th block, 32
  // blocks at a time
  const int32_t* table = a.c.table + si * a.c.stride;
  int pages = -1, turn = 32;
  float2 scales = make_float2(1.f, 1.f);
  const auto load = [&](Block8<D>& x, int b) {
    if (turn == 32) {
      turn = 0;
      const int64_t mb = (int64_t)b + (lane >> 1) * W;
      pages = -1;
      scales = make_float2(1.f, 1.f);
      if (mb < b1) {
        const int pos = key_of((int)mb) + 16 * (lane & 1);
        if (pos < s.len) pages = table[pos >> a.c.ps_log2];
        if (pages < 0 || pages >= a.c.n_pages) pages = -1;
        if (pages >= 0) scales = *reinterpret_cast<const float2*>(scales8_at(a.c, pages, kh, pos));
      }
    }
    const int key = key_of(b);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int page = __builtin_amdgcn_readlane(pages, 2 * turn + j);
      x.ok[j] = page >= 0;
      x.ks[j] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(scales.x), 2 * turn + j));
      x.vs[j] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(scales.y), 2 * turn + j));
      const uint8_t* tile = tile8_at<D>(a.c, page >= 0 ? page : 0, kh, key + 16 * j) + 16 * lane;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        x.k[j][c] = load_u32x4_stream(tile + 1024 * c);
        x.v[j][c] = load_u32x4_stream(tile + 16 * D + 1024 * c);
      }
    }
    ++turn;
  };

  h8 qf[KK];
#pragma unroll
  for (int kk = 0; kk < KK; ++kk)
    qf[kk] = col < cols ? load_q<D>(a, s.row0 + qj, h, 32 * kk + 8 * g) : zero_h8();
  const Scores f = scores_of(a);
  const float slope = MOD && a.slopes && col < cols ? a.slopes[h] * kLog2e : 0.f;

  f4 acc[NF];
#pragma unroll
  for (int n = 0; n < NF; ++n) acc[n] = f4{0.f, 0.f, 0.f, 0.f};
  float R = -INFINITY, l = 0.f;

  const auto compute = [&](Block8<D>& x, int b) {
    const int key0 = key_of(b);
    const bool edge = !(x.ok[0] && x.ok[1] && ((key0 >= all_lo && key0 + kBlock <= all_hi) ||
                                               key0 + kBlock <= s.pre));
    float y[2][4], top = -INFINITY;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      f4 d = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        const u32x4 w = x.k[j][kk / 2];
        d = mfma16(halves8<INT8, true>(w[2 * (kk % 2)], w[2 * (kk % 2) + 1], 1.f, 1.f), qf[kk], d);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (MOD) {
          const int far = at - (key0 + 16 * j + 4 * g + e);
          y[j][e] = score(f, d[e] * x.ks[j], slope, (float)(far < 0 ? -far : far));
        } else {
          y[j][e] = d[e] * (x.ks[j] * kLog2e);
        }
      }
    }
    if (edge) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int first = key0 + 16 * j + 4 * g;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int key = first + e;
          const bool in = x.ok[j] && ((key >= mine.lo && key < mine.hi) || key < pre);
          y[j][e] = in ? y[j][e] : -INFINITY;
        }
        // codes of keys that do not exist may be anything
        const int n = x.ok[j] ? min(max(s.len - first, 0), 4) : 0;
        const uint32_t keep = n == 4 ? ~0u : (1u << (8 * n)) - 1;
#pragma unroll
        for (int c = 0; c < C; ++c) x.v[j][c] &= keep;
      }
    }
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) top = fmaxf(top, y[j][e]);
    const float Rn = fmaxf(R, cols_max(top));
    const float Rs = Rn == -INFINITY ? 0.f : Rn;
    const float alpha = __builtin_amdgcn_exp2f(R - Rs);
    R = Rn;
    if (__any(alpha != 1.f)) {  // the maxima rarely grow after the first blocks
      l *= alpha;
#pragma unroll
      for (int n = 0; n < NF; ++n) acc[n] *= alpha;
    }
    const float shift = kPBits - Rs;
    h8 hi, lo;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float p = __builtin_amdgcn_exp2f(y[j][e] + shift);
        l += p;
        hi[4 * j + e] = (_Float16)p;
        lo[4 * j + e] = (_Float16)(p - (float)hi[4 * j + e]);
      }
#pragma unroll
    for (int n = 0; n < NF; ++n) {
      const h8 v = halves8<INT8, false>(x.v[0][n / 4][n % 4], x.v[1][n / 4][n % 4], x.vs[0], x.vs[1]);
      acc[n] = mfma16(v, hi, acc[n]);
      acc[n] = mfma16(v, lo, acc[n]);
    }
  };

  Block8<D> x0, x1;
  if (b < b1) load(x0, b);
  while (b < b1) {
    if (b + W < b1) load(x1, b + W);
    compute(x0, b);
    b += W;
    if (b >= b1) break;
    if (b + W < b1) load(x0, b + W);
    compute(x1, b);
    b += W;
  }

  // join the waves: element e of acc[n] is dimension 16 n + 4 g + e of column r
  l = cols_sum(l);
#pragma unroll
  for (int n = 0; n < NF; ++n) *reinterpret_cast<f4*>(&lds.sums[wave][r][16 * n + 4 * g]) = acc[n];
  if (g == 0) {
    lds.R[wave][r] = R;
    lds.l[wave][r] = l;
  }
  __syncthreads();
  for (int i = tid; i < 16 * D; i += W * 64) {
    const int cr = i / D, dim = i % D, cc = 16 * ct + cr;
    if (cc >= cols) break;
    float Rm = -INFINITY;
#pragma unroll
    for (int w = 0; w < W; ++w) Rm = fmaxf(Rm, lds.R[w][cr]);
    const float Rs = Rm == -INFINITY ? 0.f : Rm;
    float A = 0.f, L = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float z = __builtin_amdgcn_exp2f(lds.R[w][cr] - Rs);
      A = __builtin_fmaf(lds.sums[w][cr][dim], z, A);
      L = __builtin_fmaf(lds.l[w][cr], z, L);
    }
    put<D>(a, kh * a.G + cc % a.G, s.row0 + cc / a.G, sp, ns, dim, A, Rm, L);
  }
}

// sequence that holds row m (-1: none): the last i with q_start[i] <= m, 64
// candidates at a time
__device__ __forceinline__ int seq_of_row(const Attn8& a, int m) {
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

// Adds the splits of a row's head, in order: a wave for each head, D / 64 dimensions a lane.
template <int D>
__global__ __launch_bounds__(256) void attn8_merge_k(Attn8 a) {
  constexpr int N = D / 64;
  const int m = blockIdx.x, h = 4 * blockIdx.y + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int i = seq_of_row(a, m);
  if (i < 0 || h >= a.H) return;
  const Seq8 s = sequence(a, i);
  const int ns = splits_of(a, s);
  if (ns == 1 || m - s.row0 >= s.rows) return;
  const int64_t at = ((int64_t)m * a.H + h) * a.splits;
  const float2 rl = lane < ns ? a.part_rl[at + lane] : make_float2(-INFINITY, 0.f);
  float R = rl.x, w = 0.f;
#pragma unroll
  for (int d = 32; d >= 1; d /= 2) R = fmaxf(R, wave_shfl_xor(R, d));
  if (R != -INFINITY) w = __builtin_amdgcn_exp2f(rl.x - R);
  float L = rl.y * w;
#pragma unroll
  for (int d = 32; d >= 1; d /= 2) L += wave_shfl_xor(L, d);
  float A[N] = {};
  for (int j = 0; j < ns; ++j) {
    const float z = __shfl(w, j, 64);
#pragma unroll
    for (int n = 0; n < N; ++n) A[n] = __builtin_fmaf(a.part[(at + j) * D + 64 * n + lane], z, A[n]);
  }
  uint16_t* o = a.o + (int64_t)m * a.ldo + (int64_t)h * D;
#pragma unroll
  for (int n = 0; n < N; ++n) o[64 * n + lane] = f2h(L > 0.f ? A[n] / L : (L == L ? 0.f : L));
}

// keys that a sequence's rows see at most, in whole blocks
static int64_t seen_keys(const pipo_attn_scores* f, int64_t max_q, int64_t max_len) {
  const auto up = [](int64_t n) { return (n + kBlock - 1) / kBlock * kBlock; };
  if (!f || f->window <= 0) return up(max_len);
  return std::min(up(max_len), up(f->prefix ? f->max_prefix : 0) + up(f->window + max_q) + kBlock);
}

constexpr int kCUs = 256, kMinKeys = 256, kSplitKeys = 768;
struct Plan8 {
  int waves, chunk, splits;
};
static Plan8 plan_attn8(const pipo_kv8_pages* c, const pipo_attn_scores* f, int n_heads, int64_t max_q,
                        int64_t max_len) {
  const int G = n_heads / c->n_kv_heads;
  const int64_t keys = seen_keys(f, max_q, max_len);
  const int64_t wgs = (int64_t)c->n_seq * c->n_kv_heads * ((max_q * G + 15) / 16);
  Plan8 p;
  p.waves = wgs <= kCUs ? 8 : 4;
  int64_t S = keys < kSplitKeys ? 1 : std::min(kCUs / wgs, keys / kMinKeys);
  S = std::max<int64_t>(1, std::min<int64_t>(S, kMaxSplits));
  p.chunk = (int)std::max<int64_t>(kBlock, ((keys + S - 1) / S + kBlock - 1) / kBlock * kBlock);
  p.splits = (int)std::max<int64_t>(1, (keys + p.chunk - 1) / p.chunk);
  return p;
}

static int64_t partial_bytes8(int64_t M, int n_heads, int head_dim, int64_t splits) {
  return splits > 1 ? M * n_heads * splits * (head_dim + 2) * 4 : 0;
}

static pipo_status check_attn8(const char* what, const pipo_kv8_pages* c, const pipo_attn_scores* f,
                               int32_t n_heads, int64_t M, int32_t max_q, int32_t max_len) {
  if (n_heads < 1 || n_heads % c->n_kv_heads != 0 || M < 0 || max_q < 0 || max_len < 0 ||
      max_len > c->table_stride * c->page_size) {
    set_error("%s: %d query heads over %d, %lld rows, up to %d a sequence, %d keys of %lld", what,
              n_heads, c->n_kv_heads, (long long)M, max_q, max_len,
              (long long)(c->table_stride * c->page_size));
    return PIPO_ERR_ARG;
  }
  if (f && (!(f->cap >= 0.f) || f->cap > 1e30f || f->window < 0 || f->max_prefix < 0)) {
    set_error("%s: scores capped at %g, window of %d, prefixes up to %d", what, (double)f->cap, f->window,
              f->max_prefix);
    return PIPO_ERR_ARG;
  }
  const int64_t cols = std::min<int64_t>(max_q, M) * (n_heads / c->n_kv_heads);
  if (M * n_heads >= ((int64_t)1 << 30) || n_heads > 65535 ||
      (int64_t)c->n_seq * c->n_kv_heads >= ((int64_t)1 << 22) || max_len > (1 << 30) ||
      (cols + 127) / 128 * c->n_kv_heads >= ((int64_t)1 << 22)) {
    set_error("%s: %lld rows of %d heads, %d sequences of %d keys", what, (long long)M, n_heads,
              c->n_seq, max_len);
    return PIPO_ERR_UNSUPPORTED;
  }
  return PIPO_OK;
}

template <int D, bool INT8, bool MOD>
static void launch_attn8(const Attn8& a, const Plan8& p, hipStream_t st) {
  const dim3 g((unsigned)(a.c.Hkv * a.c.n_seq), (unsigned)p.splits,
               (unsigned)(((int64_t)a.max_q * a.G + 15) / 16));
  if (p.waves == 8)
    launch(attn8_few_k<D, INT8, MOD, 8>, g, dim3(512), 0, st, a);
  else
    launch(attn8_few_k<D, INT8, MOD, 4>, g, dim3(256), 0, st, a);
  if (p.splits > 1)
    launch(attn8_merge_k<D>, dim3((unsigned)a.M, (unsigned)((a.H + 3) / 4)), dim3(256), 0, st, a);
}

}  // namespace pipo

using namespace pipo;

extern "C" {

int64_t pipo_op_attn_kv8_pages_workspace_bytes(const pipo_kv8_pages* c, const pipo_attn_scores* f,
                                               int32_t n_heads, int64_t M, int32_t max_q,
                                               int32_t max_len) {
  if (!c || pipo_kv8_page_bytes(c->page_size, c->n_kv_heads, c->head_dim) == 0 || c->n_seq < 1 ||
      c->n_seq > 65535 || max_q < 1 || max_len < 1 || M < 1 ||
      check_attn8("attn_kv8_pages", c, f, n_heads, M, max_q, max_len) != PIPO_OK)
    return 0;
  return partial_bytes8(M, n_heads, c->head_dim,
                        plan_attn8(c, f, n_heads, std::min<int64_t>(max_q, M), max_len).splits);
}

pipo_status pipo_op_attn_kv8_pages(const pipo_kv8_pages* c, int32_t layer, const pipo_attn_scores* f,
                                   const uint16_t* q, int64_t ldq, const int32_t* q_start,
                                   const int32_t* kv_len, uint16_t* o, int64_t ldo, int32_t n_heads,
                                   int64_t M, int32_t max_q, int32_t max_len, void* workspace,
                                   int64_t workspace_bytes, void* stream) {
  clear_error();
  Attn8 a;
  PIPO_TRY(check_pages8("attn_kv8_pages", c, layer, &a.c));
  PIPO_TRY(check_attn8("attn_kv8_pages", c, f, n_heads, M, max_q, max_len));
  const int64_t d = (int64_t)n_heads * c->head_dim;
  if (!q || !q_start || !kv_len || !o || ldq < d || ldo < d || workspace_bytes < 0) {
    set_error("attn_kv8_pages: NULL pointer, rows (%lld, %lld) shorter than %lld, or negative "
              "workspace size", (long long)ldq, (long long)ldo, (long long)d);
    return PIPO_ERR_ARG;
  }
  if (M == 0 || max_q == 0) return PIPO_OK;
  a.q = q;
  a.o = o;
  a.q_start = q_start;
  a.kv_len = kv_len;
  a.prefix = f ? f->prefix : nullptr;
  a.slopes = f ? f->slopes : nullptr;
  a.cap = f ? f->cap : 0.f;
  a.window = f ? f->window : 0;
  a.max_prefix = f ? f->max_prefix : 0;
  a.part = static_cast<float*>(workspace);
  a.ldq = ldq;
  a.ldo = ldo;
  a.M = M;
  a.H = n_heads;
  a.G = n_heads / c->n_kv_heads;
  a.max_q = (int)std::min<int64_t>(max_q, M);
  a.max_len = max_len;
  Plan8 p = plan_attn8(c, f, n_heads, a.max_q, max_len);
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 16 != 0 ||
      workspace_bytes < partial_bytes8(M, n_heads, c->head_dim, p.splits)) {
    p.chunk = std::max(kBlock, (max_len + kBlock - 1) / kBlock * kBlock);
    p.splits = 1;
  }
  a.chunk = p.chunk;
  a.splits = p.splits;
  a.part_rl = reinterpret_cast<float2*>(a.part + M * n_heads * a.splits * c->head_dim);
  a.q_vec = reinterpret_cast<uintptr_t>(q) % 16 == 0 && ldq % 8 == 0;
  a.o_vec = reinterpret_cast<uintptr_t>(o) % 8 == 0 && ldo % 4 == 0;
  const bool int8 = c->fmt == PIPO_KV8_INT8, mod = a.cap > 0.f || a.slopes;
  const auto pick = [&](auto dc) {
    constexpr int D = decltype(dc)::value;
    const auto go = int8 ? (mod ? launch_attn8<D, true, true> : launch_attn8<D, true, false>)
                         : (mod ? launch_attn8<D, false, true> : launch_attn8<D, false, false>);
    go(a, p, static_cast<hipStream_t>(stream));
  };
  c->head_dim == 128 ? pick(std::integral_constant<int, 128>{}) : pick(std::integral_constant<int, 64>{});
  PIPO_HIP_TRY(hipGetLastError());
  return PIPO_OK;
}

}  // extern "C"
