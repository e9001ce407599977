// Drawing tokens (pipo_op_sample): for each row of logits x the token at a given
// share u of the weights exp(x / T) of the kept tokens, in the order of falling
// logits (equal ones by index), which top-k, min-p and top-p each cut to a prefix.
//
// So everything asked of a row is a place in that order, by rank or by running
// weight.  With t = 8 x / T in 64 bits, a token is in bin floor(t), and its weight
// is exp((b + 1/2) / 8) of its bin times exp of what is left of t / 8, at most
// 1/16 away from 0, as a whole number of units 2^-36.  Bins are in order, the
// order inside a bin is found only for the bins that hold a place asked for, and
// sums of whole numbers do not depend on how a row is split or on atomics' order.
// Bins more than 255 below the largest logit's, under e^-31 of its weight, count
// as nothing.
#include <climits>
#include <cmath>

#include "common.h"
#include "device.h"

namespace pipo {

constexpr int kBins = 256;
constexpr int kUnitBits = 36;             // of a weight
constexpr int kCountShift = 50;           // of a bin's count above its weight, in a slice
constexpr int kSliceMax = 8192;           // logits of a slice, so that both fit 64 bits
constexpr int kListMax = 256;             // tokens of a slice's largest bins that it lists
constexpr int kSortMax = 512;             // tokens that are put in order at once
constexpr int64_t kMaxV = (int64_t)1 << 23;
typedef unsigned long long u64;

// what one slice of a row leaves for the row's workgroup: its largest logit (with
// its index, greedily), its bins from that logit's down (weight and count in
// one word), and the tokens of its first bins, as many whole bins as fit
struct Slice {
  float m;
  int32_t arg, n_list, list_bins;
  u64 bin[kBins];
  float2 list[kListMax];  // logit, index
};

struct SampleArgs {
  const float* logits;
  int64_t ld;
  const float *T, *p, *min_p, *u;
  const int32_t* k;
  int32_t* next;
  float* logprob;
  Slice* slices;   // [rows][n_slices]
  int V, n_slices, slice;
  bool vec;        // rows on 16 bytes
};

// 8 / T of a row, 0 where the largest logit is taken
__device__ __forceinline__ double row_rate(const SampleArgs& a, int64_t row) {
  const float T = a.T ? a.T[row] : 1.f;
  return T > 0.f ? 8.0 / (double)T : -1.0;
}

// a logit's place: bin below that of the largest logit m (t of m: tm, its bin bm)
// and weight.  m infinite: its equals alone count, one unit each.
struct Place {
  int r;       // kBins: none
  double f;    // t - floor(t)
};
__device__ __forceinline__ Place place_of(float x, float m, double rate, double bm) {
#pragma clang fp contract(off)  // (t - floor(t) of the rounded t: else it leaves 0 .. 1 for large t)
  Place p;
  const double t = (double)x * rate, b = __builtin_floor(t), d = bm - b;
  p.r = d < (double)kBins ? (int)d : kBins;
  p.f = t - b;
  if (__builtin_isinf(m)) {
    p.r = x == m ? 0 : kBins;
    p.f = 0.5;
  }
  if (x == -INFINITY) p.r = kBins;
  return p;
}
// exp((f - 1/2) / 8) 2^kUnitBits, rounded: the series to the sixth power, whose rest is
// below 2^-40 of it
__device__ __forceinline__ u64 units_of(double f) {
  const double d = (f - 0.5) * 0.125;
  constexpr double one = (double)(1ull << kUnitBits);
  double e = one / 720.0;
  e = __builtin_fma(e, d, one / 120.0);
  e = __builtin_fma(e, d, one / 24.0);
  e = __builtin_fma(e, d, one / 6.0);
  e = __builtin_fma(e, d, one / 2.0);
  e = __builtin_fma(e, d, one);
  e = __builtin_fma(e, d, one);
  return (u64)__builtin_bit_cast(uint64_t, e + 0x1p52) & ((1ull << 52) - 1);
}
__device__ __forceinline__ double bin_of(float m, double rate) {
  return __builtin_isinf(m) ? (double)m : __builtin_floor((double)m * rate);
}

// keys that rise as logits fall (-0 as 0)
__device__ __forceinline__ uint32_t falling(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? b : ~(b | 0x80000000u);
}

template <int W>
__device__ __forceinline__ float block_max(float v, float (&lds)[W]) {
#pragma unroll
  for (int d = 32; d >= 1; d /= 2) v = fmaxf(v, wave_shfl_xor(v, d));
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  v = lds[0];
#pragma unroll
  for (int w = 1; w < W; ++w) v = fmaxf(v, lds[w]);
  return v;
}
template <int W>
__device__ __forceinline__ int block_min(int v, int (&lds)[W]) {
#pragma unroll
  for (int d = 32; d >= 1; d /= 2) v = min(v, wave_shfl_xor(v, d));
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  v = lds[0];
#pragma unroll
  for (int w = 1; w < W; ++w) v = min(v, lds[w]);
  return v;
}

__device__ __forceinline__ float valid(float x) { return x == x ? x : -INFINITY; }

// four consecutive logits from i on (past the end: none)
__device__ __forceinline__ f4 load4(const SampleArgs& a, const float* row, int i, int end) {
  f4 x = f4{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
  if (a.vec && i + 4 <= end) {
    x = *reinterpret_cast<const f4*>(row + i);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (i + j < end) x[j] = row[i + j];
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] = valid(x[j]);
  return x;
}

// One slice of a row: the logits stay in registers.
template <int E>
__global__ __launch_bounds__(256) void sample_slices_k(SampleArgs a) {
  static_assert(256 * E <= kSliceMax, "a bin's count and weight fit a word");
  __shared__ u64 bins[4][kBins];
  __shared__ float red[4];
  __shared__ int redi[4], scan[4], n_list;
  const int tid = threadIdx.x, lane = tid & 63;
  const int64_t row = blockIdx.x / a.n_slices;
  const int s = blockIdx.x - (int)row * a.n_slices;
  const int lo = s * 256 * E, end = min(a.V, lo + 256 * E);
  Slice& out = a.slices[(int64_t)row * a.n_slices + s];
  const float* x = a.logits + row * a.ld;
  f4 v[E / 4];
#pragma unroll
  for (int i = 0; i < E / 4; ++i) v[i] = load4(a, x, lo + 4 * (256 * i + tid), end);
  for (int i = tid; i < 4 * kBins; i += 256) (&bins[0][0])[i] = 0;
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < E / 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) m = fmaxf(m, v[i][j]);
  m = block_max(m, red);
  const double rate = row_rate(a, row);
  if (rate < 0.0 || m == -INFINITY) {
    int arg = INT_MAX;
#pragma unroll
    for (int i = 0; i < E / 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (v[i][j] == m) arg = min(arg, lo + 4 * (256 * i + tid) + j);
    arg = block_min(arg, redi);
    if (tid == 0) {
      out.m = m;
      out.arg = arg;
    }
    return;
  }
  const double bm = bin_of(m, rate);
#pragma unroll
  for (int i = 0; i < E / 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const Place p = place_of(v[i][j], m, rate, bm);
      if (p.r < kBins) atomicAdd(&bins[lane & 3][p.r], units_of(p.f) + (1ull << kCountShift));
    }
  if (tid == 0) n_list = 0;
  __syncthreads();
  const u64 h = bins[0][tid] + bins[1][tid] + bins[2][tid] + bins[3][tid];
  out.bin[tid] = h;
  // whole bins, as many as the list takes
  int c = (int)(h >> kCountShift);
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int y = __shfl_up(c, d, 64);
    if (lane >= d) c += y;
  }
  if (lane == 63) scan[tid >> 6] = c;
  __syncthreads();
  for (int w = 0; w < tid >> 6; ++w) c += scan[w];
  const int fits = __popcll(__ballot(c <= kListMax));
  if (lane == 0) redi[tid >> 6] = fits;
  __syncthreads();
  const int list_bins = redi[0] + redi[1] + redi[2] + redi[3];
#pragma unroll
  for (int i = 0; i < E / 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (place_of(v[i][j], m, rate, bm).r < list_bins) {
        const int at = atomicAdd(&n_list, 1);  // (in any order)
        out.list[at] = make_float2(v[i][j], __int_as_float(lo + 4 * (256 * i + tid) + j));
      }
  __syncthreads();
  if (tid == 0) {
    out.m = m;
    out.arg = 0;
    out.n_list = n_list;
    out.list_bins = list_bins;
  }
}

constexpr int kRowThreads = 512, kRowWaves = kRowThreads / 64;

struct RowLds {
  double cum_w[kBins];             // weights of the bins up to each
  double factor[kBins];            // of a unit
  u64 w[kBins], cum_c[kBins];      // a bin's units; counts up to each
  u64 sub_w[kBins], sub_c[kBins];  // of parts of a bin
  u64 key[kSortMax], unit[kSortMax];
  u64 bins_c[kBins];
  u64 part[kRowWaves];
  double dpart[kRowWaves];
  float red[kRowWaves];
  int redi[kRowWaves];
  int n, pick;
  uint32_t lo, hi;
};

// inclusive sums over kBins values, one for each of the first kBins threads
template <typename T>
__device__ __forceinline__ T scan_bins(T v, T (&part)[kRowWaves]) {
  const int tid = threadIdx.x, lane = tid & 63;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const T y = __shfl_up(v, d, 64);
    if (lane >= d) v += y;
  }
  if (lane == 63) part[tid >> 6] = v;
  __syncthreads();
  for (int w = 0; w < tid >> 6 && w < kBins / 64; ++w) v += part[w];
  __syncthreads();
  return v;
}

// A row: SOLO without slices.
template <bool SOLO>
struct Row {
  const SampleArgs& a;
  RowLds& lds;
  const float* x;
  const Slice* slices;
  float m;
  double rate, bm, inv_T;

  // fn(logit, index) for every token of bin r
  template <typename F>
  __device__ __forceinline__ void each(int r, F fn) const {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const auto test = [&](float v, int i) {
      if (place_of(v, m, rate, bm).r == r) fn(v, i);
    };
    if constexpr (SOLO) {
      for (int i = 4 * tid; i < a.V; i += 4 * kRowThreads) {
        const f4 v = load4(a, x, i, a.V);
#pragma unroll
        for (int j = 0; j < 4; ++j) test(v[j], i + j);
      }
    } else {
      for (int s = wave; s < a.n_slices; s += kRowWaves) {
        const Slice& sl = slices[s];
        if (sl.m == -INFINITY) continue;
        const double off = sl.m == m ? 0.0 : bm - bin_of(sl.m, rate);
        if (!(off <= (double)r)) continue;
        const int at = r - (int)off;
        if (sl.bin[at] >> kCountShift == 0) continue;
        if (at < sl.list_bins) {
          for (int i = lane; i < sl.n_list; i += 64) {
            const float2 y = sl.list[i];
            test(y.x, __float_as_int(y.y));
          }
        } else {
          const int lo = s * a.slice, end = min(a.V, lo + a.slice);
          for (int i = lo + 4 * lane; i < end; i += 256) {
            const f4 v = load4(a, x, i, end);
#pragma unroll
            for (int j = 0; j < 4; ++j) test(v[j], i + j);
          }
        }
      }
    }
  }

  struct Pick {
    int64_t rank;   // in the bin, from 1
    double units;   // up to and with it
    float x;
    int index;      // (of a pick that asks for it)
  };
  // The token of bin r at a rank (by_rank: target, from 1), or the first one with which
  // the units so far are above the target, or reach it (reach); rank `most` at the
  // latest.
  __device__ Pick pick(int r, bool by_rank, bool reach, double target, int64_t most, bool index) {
    const int tid = threadIdx.x;
    int64_t n = lds.bins_c[r];
    u64 c0 = 0, w0 = 0;   // before the part [lo, hi] of keys
    uint32_t lo = 0, hi = 0xFFFFFFFFu;
    if (n > kSortMax) {
      if (tid == 0) {
        lds.lo = 0xFFFFFFFFu;
        lds.hi = 0;
      }
      __syncthreads();
      each(r, [&](float v, int) {
        atomicMin(&lds.lo, falling(v));
        atomicMax(&lds.hi, falling(v));
      });
      __syncthreads();
      lo = lds.lo;
      hi = lds.hi;
      while (n > kSortMax && lo != hi) {
        const int shift = max(0, 32 - __clz(hi - lo) - 8);
        if (tid < kBins) lds.sub_w[tid] = lds.sub_c[tid] = 0;
        __syncthreads();
        each(r, [&](float v, int) {
          const uint32_t d = falling(v);
          if (d < lo || d > hi) return;
          atomicAdd(&lds.sub_c[(d - lo) >> shift], 1ull);
          atomicAdd(&lds.sub_w[(d - lo) >> shift], units_of(place_of(v, m, rate, bm).f));
        });
        __syncthreads();
        const u64 c = tid < kBins ? lds.sub_c[tid] : 0, w = tid < kBins ? lds.sub_w[tid] : 0;
        const u64 cc = c0 + scan_bins(c, lds.part), cw = w0 + scan_bins(w, lds.part);
        if (tid == 0) lds.pick = kBins;
        __syncthreads();
        // the first part that holds the place, or the last allowed rank
        if (tid < kBins && c > 0 && passes(cc, cw, by_rank, reach, target, most)) atomicMin(&lds.pick, tid);
        __syncthreads();
        const int q = min(lds.pick, kBins - 1);   // (one passes: most is at most n)
        if (tid == q) {
          lds.part[0] = cc - c;
          lds.part[1] = cw - w;
          lds.part[2] = c;
        }
        __syncthreads();
        c0 = lds.part[0];
        w0 = lds.part[1];
        n = (int64_t)lds.part[2];
        __syncthreads();
        lo += (uint32_t)q << shift;
        hi = min(hi, lo + ((1u << shift) - 1));
      }
    }
    if (n > kSortMax) return pick_equal(r, lo, n, c0, w0, by_rank, reach, target, most, index);
    // in order: every token finds its place among the others
    if (tid == 0) {
      lds.n = 0;
      lds.pick = INT_MAX;
    }
    __syncthreads();
    each(r, [&](float v, int i) {
      const uint32_t d = falling(v);
      if (d < lo || d > hi) return;
      const int at = atomicAdd(&lds.n, 1);
      if (at >= kSortMax) return;
      lds.key[at] = (u64)d << 32 | (uint32_t)i;
      lds.unit[at] = units_of(place_of(v, m, rate, bm).f);
    });
    __syncthreads();
    n = min(lds.n, kSortMax);
    u64 mine = 0, c = c0, w = w0;
    if (tid < n) {
      mine = lds.key[tid];
      for (int j = 0; j < n; ++j) {
        const bool before = lds.key[j] <= mine;
        c += before;
        w += before ? lds.unit[j] : 0;
      }
      if (passes(c, w, by_rank, reach, target, most)) atomicMin(&lds.pick, (int)(c - c0));
    }
    __syncthreads();
    const int64_t rank = min((int64_t)lds.pick, n);
    if (tid < n && (int64_t)(c - c0) == rank) {
      lds.part[0] = c;
      lds.part[1] = w;
      lds.part[2] = mine;
    }
    __syncthreads();
    Pick p;
    p.rank = (int64_t)lds.part[0];
    p.units = (double)lds.part[1];
    p.x = logit((uint32_t)(lds.part[2] >> 32));
    p.index = (int)(uint32_t)lds.part[2];
    __syncthreads();
    return p;
  }
  static __device__ __forceinline__ bool passes(u64 c, u64 w, bool by_rank, bool reach, double target,
                                                int64_t most) {
    if ((int64_t)c >= most) return true;
    return by_rank ? (double)c >= target : reach ? (double)w >= target : (double)w > target;
  }
  static __device__ __forceinline__ float logit(uint32_t d) {  // of falling()
    return __uint_as_float(d & 0x80000000u ? d : ~d & 0x7FFFFFFFu);
  }
  // among more equal tokens than fit: their weights are equal, so the rank is a quotient,
  // and the index is found by counting
  __device__ Pick pick_equal(int r, uint32_t d, int64_t n, u64 c0, u64 w0, bool by_rank, bool reach,
                             double target, int64_t most, bool index) {
    const float v = logit(d);
    const u64 unit = units_of(place_of(v, m, rate, bm).f);
    // the least rank from 1 that passes, by halving
    int64_t lo = 1, hi = n;
    while (lo < hi) {
      const int64_t mid = (lo + hi) / 2;
      if (passes(c0 + mid, w0 + mid * unit, by_rank, reach, target, most))
        hi = mid;
      else
        lo = mid + 1;
    }
    Pick p;
    p.rank = (int64_t)c0 + lo;
    p.units = (double)(w0 + lo * unit);
    p.x = v;
    p.index = 0;
    if (!index) return p;
    const int tid = threadIdx.x, lane = tid & 63;
    int64_t before = 0;
    for (int i0 = 0; i0 < a.V; i0 += 4 * kRowThreads) {
      const f4 y = load4(a, x, i0 + 4 * tid, a.V);
      int c = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) c += y[j] == v;
      int run = c;
#pragma unroll
      for (int k = 1; k < 64; k *= 2) {
        const int z = __shfl_up(run, k, 64);
        if (lane >= k) run += z;
      }
      if (lane == 63) lds.redi[tid >> 6] = run;
      __syncthreads();
      int total = 0;
      for (int w = 0; w < kRowWaves; ++w) {
        if (w < tid >> 6) run += lds.redi[w];
        total += lds.redi[w];
      }
      if (before + total >= lo) {   // here: the thread that has it says which
        int64_t at = before + run - c;
        for (int j = 0; j < 4; ++j)
          if (y[j] == v && ++at == lo) lds.pick = i0 + 4 * tid + j;
        __syncthreads();
        p.index = lds.pick;
        __syncthreads();
        return p;
      }
      before += total;
      __syncthreads();
    }
    return p;
  }
};

template <bool SOLO>
__global__ __launch_bounds__(kRowThreads) void sample_rows_k(SampleArgs a) {
  __shared__ RowLds lds;
  const int64_t row = blockIdx.x;
  const int tid = threadIdx.x;
  Row<SOLO> R{a, lds, a.logits + row * a.ld, a.slices + row * a.n_slices, -INFINITY, 0.0, 0.0, 0.0};
  R.rate = row_rate(a, row);
  float m = -INFINITY;
  if constexpr (SOLO) {
    for (int i = 4 * tid; i < a.V; i += 4 * kRowThreads) {
      const f4 v = load4(a, R.x, i, a.V);
#pragma unroll
      for (int j = 0; j < 4; ++j) m = fmaxf(m, v[j]);
    }
  } else {
    for (int s = tid; s < a.n_slices; s += kRowThreads) m = fmaxf(m, R.slices[s].m);
  }
  m = block_max(m, lds.red);
  if (R.rate < 0.0 || m == -INFINITY) {   // the largest; nothing to draw from: 0
    int arg = INT_MAX;
    if (m != -INFINITY) {
      if constexpr (SOLO) {
        for (int i = 4 * tid; i < a.V; i += 4 * kRowThreads) {
          const f4 v = load4(a, R.x, i, a.V);
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (v[j] == m) arg = min(arg, i + j);
        }
      } else {
        for (int s = tid; s < a.n_slices; s += kRowThreads)
          if (R.slices[s].m == m) arg = min(arg, R.slices[s].arg);
      }
    }
    arg = block_min(arg, lds.redi);
    if (tid == 0) {
      a.next[row] = arg == INT_MAX ? 0 : arg;
      if (a.logprob) a.logprob[row] = m == -INFINITY ? -INFINITY : 0.f;
    }
    return;
  }
  R.m = m;
  R.bm = bin_of(m, R.rate);
  R.inv_T = R.rate * 0.125;

  // bins of the row
  if (tid < kBins) lds.w[tid] = lds.bins_c[tid] = 0;
  __syncthreads();
  if constexpr (SOLO) {
    for (int i = 4 * tid; i < a.V; i += 4 * kRowThreads) {
      const f4 v = load4(a, R.x, i, a.V);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const Place p = place_of(v[j], m, R.rate, R.bm);
        if (p.r < kBins) {
          atomicAdd(&lds.w[p.r], units_of(p.f));
          atomicAdd(&lds.bins_c[p.r], 1ull);
        }
      }
    }
  } else {
    const int r = tid & (kBins - 1);
    u64 w = 0, c = 0;
    for (int s = tid / kBins; s < a.n_slices; s += kRowThreads / kBins) {
      const float ms = R.slices[s].m;
      if (ms == -INFINITY) continue;
      const double off = ms == m ? 0.0 : R.bm - bin_of(ms, R.rate);
      if (!(off <= (double)r)) continue;
      const u64 h = R.slices[s].bin[r - (int)off];
      w += h & ((1ull << kCountShift) - 1);
      c += h >> kCountShift;
    }
    atomicAdd(&lds.w[r], w);
    atomicAdd(&lds.bins_c[r], c);
  }
  __syncthreads();
  double f = 0.0;
  u64 w = 0, c = 0;
  if (tid < kBins) {
    w = lds.w[tid];
    c = lds.bins_c[tid];
    // over the first bin's middle: equal logits there are summed and divided exactly
    f = exp(-0.125 * tid) * (1.0 / (double)(1ull << kUnitBits));
    lds.factor[tid] = f;
  }
  const double cum_w = scan_bins((double)w * f, lds.dpart);
  const u64 cum_c = scan_bins(c, lds.part);
  if (tid < kBins) {
    lds.cum_w[tid] = cum_w;
    lds.cum_c[tid] = cum_c;
  }
  __syncthreads();

  // The kept prefix: bins below `bin` and the first `n` of it, with weight `total`.
  int bin = kBins - 1;
  int64_t n = (int64_t)lds.bins_c[bin];
  double total = lds.cum_w[kBins - 1];
  const auto below_w = [&](int r) { return r > 0 ? lds.cum_w[r - 1] : 0.0; };
  const auto below_c = [&](int r) { return r > 0 ? (int64_t)lds.cum_c[r - 1] : 0; };
  // the first bin with fn
  const auto first = [&](auto fn) {
    if (tid == 0) lds.pick = kBins - 1;
    __syncthreads();
    if (tid < kBins && fn(tid)) atomicMin(&lds.pick, tid);
    __syncthreads();
    const int r = lds.pick;
    __syncthreads();
    return r;
  };
  const auto cut = [&](int r, int64_t rank, double units) {
    bin = r;
    n = rank;
    total = below_w(r) + units * lds.factor[r];
  };
  const auto cut_at = [&](int r, int64_t rank) {
    if (rank == (int64_t)lds.bins_c[r]) {
      cut(r, rank, (double)lds.w[r]);
    } else if (rank > 0) {
      const auto p = R.pick(r, true, false, (double)rank, rank, false);
      cut(r, p.rank, p.units);
    } else {
      cut(r, 0, 0.0);
    }
  };

  const int64_t k = a.k ? a.k[row] : 0;
  if (k > 0 && k < (int64_t)lds.cum_c[kBins - 1]) {
    const int r = first([&](int i) { return (int64_t)lds.cum_c[i] >= k; });
    cut_at(r, k - below_c(r));
  }
  const float min_p = a.min_p ? a.min_p[row] : 0.f;
  if (min_p > 0.f && !__builtin_isinf(m)) {
    // the bin where weights fall below min_p, and how many of it do not
    const double low = (double)fminf(min_p, 1.f);
    const double d = R.bm - __builtin_floor(((double)m * R.inv_T + log(low)) * 8.0);
    const int r = d < (double)kBins ? max(0, (int)d) : kBins;
    if (r <= bin) {
      if (tid == 0) lds.n = 0;
      __syncthreads();
      R.each(r, [&](float v, int) {
        if (exp(((double)v - (double)m) * R.inv_T) >= low) atomicAdd(&lds.n, 1);
      });
      __syncthreads();
      const int64_t keep = lds.n;
      __syncthreads();
      if (r < bin || keep < n) cut_at(r, keep);
    }
  }
  const float top_p = a.p ? a.p[row] : 1.f;
  if (top_p < 1.f) {
    const double target = (double)fmaxf(top_p, 0.f) * total;
    const int r = min(bin, first([&](int i) { return lds.bins_c[i] > 0 && lds.cum_w[i] >= target; }));
    const int64_t most = r == bin ? n : (int64_t)lds.bins_c[r];
    if (most > 0) {
      const auto p = R.pick(r, false, true, (target - below_w(r)) / lds.factor[r], most, false);
      cut(r, p.rank, p.units);
    }
  }
  const float u = fminf(fmaxf(a.u[row], 0.f), 1.f);   // (NaN: 0)
  const double target = (double)u * total;
  int r = min(bin, first([&](int i) { return lds.cum_w[i] > target; }));
  int64_t most = r == bin ? n : (int64_t)lds.bins_c[r];
  while (most == 0 && r > 0) most = (int64_t)lds.bins_c[--r];   // (a cut at the head of a bin)
  const auto p = R.pick(r, false, false, (target - below_w(r)) / lds.factor[r], most, true);
  if (tid == 0) {
    a.next[row] = p.index;
    if (a.logprob) {
      // (the first bin's middle over the largest logit)
      const double top = (0.5 - place_of(m, m, R.rate, R.bm).f) * 0.125;
      const double z = p.x == m ? 0.0 : ((double)p.x - (double)m) * R.inv_T;
      a.logprob[row] = (float)(z - top - log(total));
    }
  }
}

static int slice_elements(int64_t rows, int64_t V) {
  (void)rows;
  (void)V;
  return 32;
}
static int64_t slices_of(int64_t rows, int64_t V) {
  const int64_t slice = 256 * slice_elements(rows, V);
  return (V + slice - 1) / slice;
}

}  // namespace pipo

using namespace pipo;

extern "C" {

int64_t pipo_op_sample_workspace_bytes(int64_t rows, int64_t V) {
  if (rows < 1 || V < 1 || V > kMaxV || rows * slices_of(rows, V) >= ((int64_t)1 << 23)) return 0;
  return rows * slices_of(rows, V) * (int64_t)sizeof(Slice);
}

pipo_status pipo_op_sample(const float* logits, int64_t ld, const float* temperature,
                           const int32_t* top_k, const float* top_p, const float* min_p,
                           const float* u, int32_t* next, float* logprob, int64_t rows, int64_t V,
                           void* workspace, int64_t workspace_bytes, void* stream) {
  clear_error();
  if (!logits || !u || !next || rows < 0 || V < 1 || ld < V || workspace_bytes < 0) {
    set_error("sample: NULL pointer, %lld rows of %lld logits every %lld, or negative workspace size",
              (long long)rows, (long long)V, (long long)ld);
    return PIPO_ERR_ARG;
  }
  if (V > kMaxV || rows >= ((int64_t)1 << 22)) {
    set_error("sample: %lld rows of %lld logits", (long long)rows, (long long)V);
    return PIPO_ERR_UNSUPPORTED;
  }
  if (rows == 0) return PIPO_OK;
  SampleArgs a;
  a.logits = logits;
  a.ld = ld;
  a.T = temperature;
  a.k = top_k;
  a.p = top_p;
  a.min_p = min_p;
  a.u = u;
  a.next = next;
  a.logprob = logprob;
  a.slices = static_cast<Slice*>(workspace);
  a.V = (int)V;
  a.n_slices = (int)slices_of(rows, V);
  a.slice = 256 * slice_elements(rows, V);
  a.vec = reinterpret_cast<uintptr_t>(logits) % 16 == 0 && ld % 4 == 0;
  const int64_t need = pipo_op_sample_workspace_bytes(rows, V);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 16 != 0 || need == 0 ||
      workspace_bytes < need) {
    launch(sample_rows_k<true>, dim3((unsigned)rows), dim3(kRowThreads), 0, st, a);
  } else {
    launch(sample_slices_k<32>, dim3((unsigned)(rows * a.n_slices)), dim3(256), 0, st, a);
    launch(sample_rows_k<false>, dim3((unsigned)rows), dim3(kRowThreads), 0, st, a);
  }
  PIPO_HIP_TRY(hipGetLastError());
  return PIPO_OK;
}

}  // extern "C"
