// Page tables of a 4-bit KV cache: growing, trimming and freeing sequences,
// continuing sequences from others (forks) and moving the pages in use to the
// front (pipo_op_kv_pages_resize, _fork, _compact in pipo_ops.h).
//
// The state is the table and the lengths alone: a row's first ceil(len /
// page_size) entries are the sequence's pages, and a page is in use if a row
// says so.  Each call finds the pages in use anew, as a bitmap in LDS, so there
// are no reference counts or free lists that could disagree with the table,
// and everything is decided in one workgroup, in order: the lowest free pages
// go to the lowest sequences.  Bound by the latency of a few passes over the
// table by one CU.
#include <algorithm>

#include "common.h"
#include "device.h"

namespace pipo {

constexpr int kMaxTablePages = 1 << 20, kMaxTableSeqs = 2048;
constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kMaxWords = kMaxTablePages / 32;

struct TableArgs {
  const int32_t *table, *len;
  int32_t *table_out, *len_out;
  int64_t stride;
  int n_seq, n_pages, ps;
};

// pages of n positions, at most a row's
__device__ __forceinline__ int pages_of(const TableArgs& a, int n) {
  if (n <= 0) return 0;
  return (int)min((int64_t)((n - 1) / a.ps + 1), a.stride);
}

// exclusive prefix of v over the workgroup, and the total
__device__ __forceinline__ int block_scan(int v, int* sums, int& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int x = v;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int y = __shfl_up(x, d, 64);
    if (lane >= d) x += y;
  }
  __syncthreads();  // sums is free
  if (lane == 63) sums[wave] = x;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const int s = sums[w];
    if (w < wave) before += s;
    total += s;
  }
  return before + x - v;
}

// A set of pages as bits, the members of each thread's share of the words
// counted in thread order: rank and select over it.
struct Ranks {
  const uint32_t* bits;
  const int* before;  // members in the shares of the threads before t
  int share, words;   // words per thread, in all
  __device__ __forceinline__ int nth(int r) const {  // the r-th member
    int lo = 0, hi = kThreads - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if (before[mid] <= r)
        lo = mid;
      else
        hi = mid - 1;
    }
    r -= before[lo];
    int w = lo * share;
    for (;; ++w) {
      const int n = __popc(bits[w]);
      if (r < n) break;
      r -= n;
    }
    const uint32_t x = bits[w];
    int at = 0;
#pragma unroll
    for (int n = 16; n >= 1; n /= 2) {
      const int c = __popc((x >> at) & ((1u << n) - 1));
      if (r >= c) {
        r -= c;
        at += n;
      }
    }
    return 32 * w + at;
  }
  __device__ __forceinline__ int rank(int page) const {  // members below page
    const int w = page >> 5;
    int t = w / share, n = before[t];
    for (int i = t * share; i < w; ++i) n += __popc(bits[i]);
    return n + __popc(bits[w] & ((1u << (page & 31)) - 1));
  }
};

__device__ __forceinline__ void mark(uint32_t* bits, int page, int n_pages) {
  if (page >= 0 && page < n_pages) atomicOr(&bits[page >> 5], 1u << (page & 31));
}

// f(j, entry) for the entries j < n of a row, by 16 lanes with four loads under
// way: a row for each 16 lanes of the workgroup at a time
constexpr int kRowLanes = 16, kRows = kThreads / kRowLanes;
template <typename F>
__device__ __forceinline__ void row_entries(const int32_t* row, int n, F&& f) {
  const int lane = threadIdx.x % kRowLanes;
  for (int j = lane; j < n; j += 4 * kRowLanes) {
    int x[4];
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (j + u * kRowLanes < n) x[u] = row[j + u * kRowLanes];
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (j + u * kRowLanes < n) f(j + u * kRowLanes, x[u]);
  }
}

// bits -> their complement among n_pages pages, with its ranks; returns the
// number of members
__device__ __forceinline__ int free_ranks(uint32_t* bits, int* before, int* sums, int n_pages,
                                          Ranks& r) {
  const int words = (n_pages + 31) / 32, share = (words + kThreads - 1) / kThreads;
  int n = 0, total;
  __syncthreads();
  for (int w = threadIdx.x * share; w < min((int)(threadIdx.x + 1) * share, words); ++w) {
    uint32_t x = ~bits[w];
    if (w == words - 1 && n_pages % 32) x &= (1u << (n_pages % 32)) - 1;
    bits[w] = x;
    n += __popc(x);
  }
  before[threadIdx.x] = block_scan(n, sums, total);
  __syncthreads();
  r = Ranks{bits, before, share, words};
  return total;
}

// The lengths first; then the pages that stay are marked and what sequences grow
// by is summed; then the rows are written, grown entries by their rank.
__global__ __launch_bounds__(kThreads) void pages_resize_k(TableArgs a, const int32_t* want,
                                                           int32_t* missing) {
  __shared__ uint32_t bits[kMaxWords];
  __shared__ int before[kThreads], sums[kWaves], grown[kMaxTableSeqs], held[kMaxTableSeqs],
      need[kMaxTableSeqs];
  __shared__ unsigned long long excess;  // pages wanted past the rows' ends
  const int tid = threadIdx.x, row0 = tid / kRowLanes;
  for (int w = tid; w < (a.n_pages + 31) / 32; w += kThreads) bits[w] = 0;
  if (tid == 0) excess = 0;
  int total = 0;
  for (int i0 = 0; i0 < a.n_seq; i0 += kThreads) {
    const int i = i0 + tid;
    int g = 0, n;
    int64_t over = 0;
    if (i < a.n_seq) {
      const int to = want[i], h = pages_of(a, a.len[i]), k = to < 0 ? h : pages_of(a, to);
      held[i] = h;
      need[i] = k;
      g = max(0, k - h);
      if (to > 0) over = (to - 1) / a.ps + 1 - a.stride;
    }
    const int at = block_scan(g, sums, n);
    if (i < a.n_seq) grown[i] = total + at;
    total += n;
    if (over > 0) atomicAdd(&excess, (unsigned long long)over);
  }
  __syncthreads();
  for (int i = row0; i < a.n_seq; i += kRows)
    row_entries(a.table + i * a.stride, min(held[i], need[i]),
                [&](int, int page) { mark(bits, page, a.n_pages); });
  Ranks free;
  const int n_free = free_ranks(bits, before, sums, a.n_pages, free);
  const int short_by = (int)min((int64_t)max(0, total - n_free) + (int64_t)excess, (int64_t)INT32_MAX);
  if (tid == 0) *missing = short_by;
  const bool copy = a.table_out != a.table;
  for (int i = row0; i < a.n_seq; i += kRows) {
    const int h = held[i], k = short_by ? h : need[i];
    int32_t* out = a.table_out + i * a.stride;
    if (copy) row_entries(a.table + i * a.stride, min(h, k), [&](int j, int page) { out[j] = page; });
    for (int64_t j = min(h, k) + tid % kRowLanes; j < a.stride; j += kRowLanes)
      out[j] = j < k ? free.nth(grown[i] + (int)(j - h)) : -1;
  }
  for (int i = tid; i < a.n_seq; i += kThreads) {
    const int to = want[i];
    a.len_out[i] = to < 0 || short_by ? a.len[i] : to;
  }
}

// Sequence i of the output continues parent[i].  The pages that stay are the
// parents' with a child; a parent's last page, if it is not full, goes to its
// first child, the others get copies.
__global__ __launch_bounds__(kThreads) void pages_fork_k(TableArgs a, int n_out,
                                                         const int32_t* parent, int32_t* pairs,
                                                         int32_t* n_pairs, int32_t* missing) {
  __shared__ uint32_t bits[kMaxWords];
  __shared__ int before[kThreads], sums[kWaves], first[kMaxTableSeqs], copy[kMaxTableSeqs],
      length[kMaxTableSeqs];
  const int tid = threadIdx.x, row0 = tid / kRowLanes, lane = tid % kRowLanes;
  for (int w = tid; w < (a.n_pages + 31) / 32; w += kThreads) bits[w] = 0;
  for (int i = tid; i < a.n_seq; i += kThreads) {
    first[i] = n_out;
    length[i] = max(a.len[i], 0);
  }
  __syncthreads();
  for (int i = tid; i < n_out; i += kThreads) {
    const int p = parent[i];
    if (p >= 0 && p < a.n_seq) atomicMin(&first[p], i);
  }
  __syncthreads();
  for (int i = row0; i < a.n_seq; i += kRows)
    if (first[i] < n_out)
      row_entries(a.table + i * a.stride, pages_of(a, length[i]),
                  [&](int, int page) { mark(bits, page, a.n_pages); });
  int total = 0;
  for (int i0 = 0; i0 < n_out; i0 += kThreads) {
    const int i = i0 + tid;
    int c = 0, n;
    if (i < n_out) {
      const int p = parent[i];
      c = p >= 0 && p < a.n_seq && length[p] % a.ps != 0 && first[p] != i;
    }
    const int at = block_scan(c, sums, n);
    if (i < n_out) copy[i] = c ? total + at : -1;
    total += n;
  }
  Ranks free;
  const int n_free = free_ranks(bits, before, sums, a.n_pages, free);
  const int short_by = max(0, total - n_free);
  if (tid == 0) {
    *missing = short_by;
    *n_pairs = short_by ? 0 : total;
  }
  if (short_by) return;
  for (int i = row0; i < n_out; i += kRows) {
    const int p = parent[i];
    const bool ok = p >= 0 && p < a.n_seq;
    const int len = ok ? length[p] : 0, held = pages_of(a, len), c = copy[i];
    int32_t* out = a.table_out + i * a.stride;
    if (ok)
      row_entries(a.table + p * a.stride, held, [&](int j, int page) {
        if (c >= 0 && j == held - 1) {
          const int to = free.nth(c);
          pairs[2 * c] = page;
          pairs[2 * c + 1] = to;
          page = to;
        }
        out[j] = page;
      });
    for (int64_t j = held + lane; j < a.stride; j += kRowLanes) out[j] = -1;
    if (lane == 0) a.len_out[i] = len;
  }
}

// With U pages in use, the i-th of them at U or above moves to the i-th page
// below U that is not.
__global__ __launch_bounds__(kThreads) void pages_compact_k(TableArgs a, int32_t* pairs,
                                                            int32_t* n_pairs) {
  __shared__ uint32_t bits[kMaxWords];
  __shared__ int before[kThreads], sums[kWaves], held[kMaxTableSeqs];
  const int tid = threadIdx.x, row0 = tid / kRowLanes;
  for (int w = tid; w < (a.n_pages + 31) / 32; w += kThreads) bits[w] = 0;
  for (int i = tid; i < a.n_seq; i += kThreads) held[i] = pages_of(a, a.len[i]);
  __syncthreads();
  for (int i = row0; i < a.n_seq; i += kRows)
    row_entries(a.table + i * a.stride, held[i],
                [&](int, int page) { mark(bits, page, a.n_pages); });
  Ranks free;
  const int U = a.n_pages - free_ranks(bits, before, sums, a.n_pages, free);
  // free pages below U take the pages in use from U on
  const int moves = U < a.n_pages ? free.rank(U) : 0;
  if (tid == 0) *n_pairs = moves;
  // a page in use from U on is the p - U less the free ones between-th of those
  const auto place = [&](int p) { return p - U - (free.rank(p) - moves); };
  // the free pages below U as a list behind the bits, where there is room (up to
  // 61680 pages always; 4900 pages: 9.9 us, 20 without)
  const bool listed = moves <= kMaxWords - free.words;
  uint32_t* const list = bits + free.words;
  if (listed)
    for (int p = tid; p < U; p += kThreads)
      if (bits[p >> 5] >> (p & 31) & 1) list[free.rank(p)] = p;
  __syncthreads();
  const auto target = [&](int i) { return listed ? (int)list[i] : free.nth(i); };
  for (int p = U + tid; p < a.n_pages; p += kThreads) {
    if (bits[p >> 5] >> (p & 31) & 1) continue;
    const int i = place(p);
    pairs[2 * i] = p;
    pairs[2 * i + 1] = target(i);
  }
  for (int i = row0; i < a.n_seq; i += kRows) {
    int32_t* out = a.table_out + i * a.stride;
    row_entries(a.table + i * a.stride, held[i], [&](int j, int p) {
      out[j] = p >= U && p < a.n_pages ? target(place(p)) : p;
    });
    for (int64_t j = held[i] + tid % kRowLanes; j < a.stride; j += kRowLanes) out[j] = -1;
  }
}

static pipo_status check_table(const char* what, const TableArgs& a) {
  if (!a.table || !a.len || !a.table_out || a.stride < 1 || a.n_seq < 1 || a.n_pages < 1 ||
      a.ps < 16 || a.ps > 256 || (a.ps & (a.ps - 1)) != 0) {
    set_error("%s: NULL pointer, or table %d x %lld, %d pages of %d positions", what, a.n_seq,
              (long long)a.stride, a.n_pages, a.ps);
    return PIPO_ERR_ARG;
  }
  if (a.n_pages > kMaxTablePages || a.n_seq > kMaxTableSeqs ||
      a.n_seq * a.stride >= ((int64_t)1 << 31)) {
    set_error("%s: %d sequences of %lld and %d pages, above %d, 2^31 in all, and %d", what, a.n_seq,
              (long long)a.stride, a.n_pages, kMaxTableSeqs, kMaxTablePages);
    return PIPO_ERR_UNSUPPORTED;
  }
  return PIPO_OK;
}

// whether [a, a + na) and [b, b + nb) share an element
static bool overlap(const int32_t* a, int64_t na, const int32_t* b, int64_t nb) {
  return a < b + nb && b < a + na;
}

static pipo_status check_apart(const char* what, bool apart) {
  if (apart) return PIPO_OK;
  set_error("%s: outputs overlap the inputs or each other", what);
  return PIPO_ERR_ARG;
}

}  // namespace pipo

using namespace pipo;

extern "C" {

pipo_status pipo_op_kv_pages_resize(const int32_t* table, const int32_t* len, const int32_t* want,
                                    int32_t* table_out, int32_t* len_out, int64_t table_stride,
                                    int32_t n_seq, int32_t n_pages, int32_t page_size,
                                    int32_t* missing, void* stream) {
  clear_error();
  const TableArgs a{table, len, table_out, len_out, table_stride, n_seq, n_pages, page_size};
  if (!want || !len_out || !missing) {
    set_error("kv_pages_resize: NULL pointer");
    return PIPO_ERR_ARG;
  }
  PIPO_TRY(check_table("kv_pages_resize", a));
  const int64_t n = n_seq * table_stride;
  PIPO_TRY(check_apart(
      "kv_pages_resize",
      (table == table_out || !overlap(table, n, table_out, n)) &&
          (len == len_out || !overlap(len, n_seq, len_out, n_seq)) &&
          !overlap(table_out, n, len, n_seq) && !overlap(table_out, n, want, n_seq) &&
          !overlap(table_out, n, len_out, n_seq) && !overlap(len_out, n_seq, table, n) &&
          !overlap(len_out, n_seq, want, n_seq) && !overlap(missing, 1, table, n) &&
          !overlap(missing, 1, table_out, n) && !overlap(missing, 1, len, n_seq) &&
          !overlap(missing, 1, len_out, n_seq) && !overlap(missing, 1, want, n_seq)));
  launch(pages_resize_k, dim3(1), dim3(kThreads), 0, static_cast<hipStream_t>(stream), a, want,
         missing);
  PIPO_HIP_TRY(hipGetLastError());
  return PIPO_OK;
}

pipo_status pipo_op_kv_pages_fork(const int32_t* table, const int32_t* len, int32_t n_seq,
                                  const int32_t* parent, int32_t* table_out, int32_t* len_out,
                                  int32_t n_out, int64_t table_stride, int32_t n_pages,
                                  int32_t page_size, int32_t* pairs, int32_t* n_pairs,
                                  int32_t* missing, void* stream) {
  clear_error();
  const TableArgs a{table, len, table_out, len_out, table_stride, n_seq, n_pages, page_size};
  if (!parent || !len_out || !pairs || !n_pairs || !missing || n_out < 1) {
    set_error("kv_pages_fork: NULL pointer or %d sequences", n_out);
    return PIPO_ERR_ARG;
  }
  PIPO_TRY(check_table("kv_pages_fork", a));
  if (n_out > kMaxTableSeqs || n_out * table_stride >= ((int64_t)1 << 31)) {
    set_error("kv_pages_fork: %d sequences of %lld pages, above %d or 2^31 in all", n_out,
              (long long)table_stride, kMaxTableSeqs);
    return PIPO_ERR_UNSUPPORTED;
  }
  const int64_t n = n_seq * table_stride;
  const struct { const int32_t* p; int64_t n; bool out; } r[] = {
      {table, n, false}, {len, n_seq, false}, {parent, n_out, false},
      {table_out, n_out * table_stride, true}, {len_out, n_out, true}, {pairs, 2 * (int64_t)n_out, true},
      {n_pairs, 1, true}, {missing, 1, true}};
  bool apart = true;
  for (const auto& x : r)
    for (const auto& y : r)
      if (&x != &y && (x.out || y.out)) apart = apart && !overlap(x.p, x.n, y.p, y.n);
  PIPO_TRY(check_apart("kv_pages_fork", apart));
  launch(pages_fork_k, dim3(1), dim3(kThreads), 0, static_cast<hipStream_t>(stream), a, n_out,
         parent, pairs, n_pairs, missing);
  PIPO_HIP_TRY(hipGetLastError());
  return PIPO_OK;
}

pipo_status pipo_op_kv_pages_compact(const int32_t* table, const int32_t* len, int32_t* table_out,
                                     int64_t table_stride, int32_t n_seq, int32_t n_pages,
                                     int32_t page_size, int32_t* pairs, int32_t* n_pairs,
                                     void* stream) {
  clear_error();
  const TableArgs a{table, len, table_out, nullptr, table_stride, n_seq, n_pages, page_size};
  if (!pairs || !n_pairs) {
    set_error("kv_pages_compact: NULL pointer");
    return PIPO_ERR_ARG;
  }
  PIPO_TRY(check_table("kv_pages_compact", a));
  const int64_t n = n_seq * table_stride, np = n_pages / 2 * 2;
  PIPO_TRY(check_apart(
      "kv_pages_compact",
      (table == table_out || !overlap(table, n, table_out, n)) &&
          !overlap(table_out, n, len, n_seq) && !overlap(pairs, np, table, n) &&
          !overlap(pairs, np, table_out, n) && !overlap(pairs, np, len, n_seq) &&
          !overlap(pairs, np, n_pairs, 1) && !overlap(n_pairs, 1, table, n) &&
          !overlap(n_pairs, 1, table_out, n) && !overlap(n_pairs, 1, len, n_seq)));
  launch(pages_compact_k, dim3(1), dim3(kThreads), 0, static_cast<hipStream_t>(stream), a, pairs,
         n_pairs);
  PIPO_HIP_TRY(hipGetLastError());
  return PIPO_OK;
}

}  // extern "C"
