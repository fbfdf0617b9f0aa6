// Shared pieces of the kernels around a paged KV cache (internal).
#pragma once

#include "spts_common.cuh"

namespace spts {
namespace paged {

// A cache as the kernels see it.  Row j of sequence b lies in page table[b, j >> shift] at j & (page - 1); an entry of the table
// outside [0, n_pages) names no page: its rows read as zeros and are not written.
struct Cache {
  const char* k; const char* v;
  int32_t* pos; float* weight;
  const int32_t* table; int32_t* len;
  int n_pages, max_pages, n_seq, shift;
};

inline Cache make_cache(const spts_paged_kv* c) {
  Cache d;
  d.k = (const char*)c->k; d.v = (const char*)c->v; d.pos = c->pos; d.weight = c->weight; d.table = c->table; d.len = c->len;
  d.n_pages = c->n_pages; d.max_pages = c->max_pages; d.n_seq = c->n_seq;
  d.shift = 0;
  while ((1 << d.shift) < c->page_size) ++d.shift;
  return d;
}

// Rows that sequence b holds: len beyond the table counts as the table's rows.
__device__ __forceinline__ int held_rows(const Cache& c, int b) {
  return max(0, min(c.len[b], c.max_pages << c.shift));
}

// The rows [first, first + n) of a call that belong to sequence b.  Starts are held within [0, n_rows].
__device__ __forceinline__ void call_rows(const int32_t* __restrict__ row_start, int n_rows, int b, int& first, int& n) {
  if (row_start == nullptr) { first = b; n = 1; return; }
  first = max(0, min(__ldg(&row_start[b]), n_rows));
  n = max(first, min(__ldg(&row_start[b + 1]), n_rows)) - first;
}

// SPTS_ERR_INDEX for starts that descend or leave [0, n_rows]
__device__ __forceinline__ void check_starts(const int32_t* __restrict__ row_start, int n_rows, int b, int* status) {
  if (row_start == nullptr) return;
  const int r0 = __ldg(&row_start[b]), r1 = __ldg(&row_start[b + 1]);
  if (r0 < 0 || r1 < r0 || r1 > n_rows) set_status(status, SPTS_ERR_INDEX);
}

// Place of row j of sequence b among all rows of the pages; -1: the table names no page there.
__device__ __forceinline__ int64_t slot_of(const Cache& c, int b, int j) {
  const int p = __ldg(&c.table[(int64_t)b * c.max_pages + (j >> c.shift)]);
  if (p < 0 || p >= c.n_pages) return -1;
  return ((int64_t)p << c.shift) + (j & ((1 << c.shift) - 1));
}

// Exclusive prefix sums of up to PREFIX_MAX values by a block of NT threads; value(b) is evaluated once for each b.  pre [n + 1] in
// shared memory; all threads get the total.  `warp_sums`: 32 entries of shared memory.  Up to 32 values are summed by the first warp alone,
// and only its threads get the total then (others: pre[n] behind the block's next barrier).
static const int PREFIX_MAX = SPTS_PAGED_MAX_SEQ;
template <int NT, typename F>
__device__ __forceinline__ long long block_prefix(int n, long long* pre, long long* warp_sums, F value) {
  constexpr int PER = (PREFIX_MAX + NT - 1) / NT;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (n <= 32) {
    if (warp > 0) return 0;
    const long long mine = lane < n ? value(lane) : 0;
    long long inc = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long other = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += other;
    }
    if (lane < n) pre[lane] = inc - mine;
    if (lane == 31) pre[n] = inc;
    __syncwarp();
    return __shfl_sync(0xffffffffu, inc, 31);
  }
  long long v[PER], sum = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int b = tid * PER + i;
    v[i] = b < n ? value(b) : 0;
    sum += v[i];
  }
  long long inc = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long other = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += other;
  }
  if (lane == 31) warp_sums[warp] = inc;
  __syncthreads();
  long long before = 0, total = 0;
  for (int w = 0; w < NT / 32; ++w) {
    if (w < warp) before += warp_sums[w];
    total += warp_sums[w];
  }
  long long at = before + inc - sum;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int b = tid * PER + i;
    if (b < n) pre[b] = at;
    at += v[i];
  }
  if (tid == 0) pre[n] = total;
  __syncthreads();
  return total;
}

// The last b with pre[b] <= x among those with a share of their own (pre[b + 1] > x).
__device__ __forceinline__ int find_share(const long long* pre, int n, long long x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (pre[mid] <= x) lo = mid; else hi = mid;
  }
  return lo;
}

}  // namespace paged
}  // namespace spts
