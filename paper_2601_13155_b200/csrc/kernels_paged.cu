// The paged KV cache on CUDA cores: rows are appended to it (paged_append_kernel), attention and the weights that its rows gather in
// either storage type (paged_attn_plain_kernel, paged_weights_plain_kernel: fp32 storage, SPTS_REFERENCE_KERNELS, more than 128 query
// heads to a KV head), and sequences are cut down to a budget (evict_rank_kernel, evict_move_kernel).
#include <climits>

#include <cooperative_groups.h>

#include "paged_common.cuh"

namespace spts {

namespace {

using namespace paged;
namespace cg = cooperative_groups;

// ------------------------------------------------------------------------------------------------ append
constexpr int APPEND_WARPS = 8;

// One warp copies a row's K, another its V, in 16-byte pieces.  Lengths grow only once no block reads the old ones any more: the
// block that is done last sets them (one launch).
__global__ void __launch_bounds__(APPEND_WARPS * 32)
paged_append_kernel(Cache c, const char* __restrict__ K, int64_t ldk, const char* __restrict__ V, int64_t ldv, int row_bytes,
                    const int32_t* __restrict__ pos, const int32_t* __restrict__ row_start, const int32_t* __restrict__ at, int n_rows,
                    int* arrived, int* status) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int capacity = c.max_pages << c.shift;
  dep_wait();
  for (int64_t unit = (int64_t)blockIdx.x * APPEND_WARPS + warp; unit < 2 * (int64_t)n_rows; unit += (int64_t)gridDim.x * APPEND_WARPS) {
    const int row = (int)(unit >> 1);
    const bool is_v = unit & 1;
    int b = row, first = row;
    if (row_start != nullptr) {
      // the last b with row_start[b] <= row
      int lo = 0, hi = c.n_seq;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (__ldg(&row_start[mid]) <= row) lo = mid; else hi = mid;
      }
      b = lo;
      first = max(0, __ldg(&row_start[b]));
      if (row < first || row >= __ldg(&row_start[b + 1])) continue;
    }
    const int64_t j = (int64_t)(at != nullptr ? __ldg(&at[b]) : c.len[b]) + (row - first);
    if (j < 0 || j >= capacity) {
      if (lane == 0) set_status(status, SPTS_ERR_WORKSPACE);
      continue;
    }
    const int64_t slot = slot_of(c, b, (int)j);
    if (slot < 0) {
      if (lane == 0) set_status(status, SPTS_ERR_INDEX);
      continue;
    }
    const uint4* src = reinterpret_cast<const uint4*>((is_v ? V + row * ldv : K + row * ldk));
    uint4* dst = reinterpret_cast<uint4*>(const_cast<char*>(is_v ? c.v : c.k) + slot * row_bytes);
    const int pieces = row_bytes >> 4;
    for (int i = lane; i < pieces; i += 128) {
      uint4 x[4];
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (i + 32 * u < pieces) x[u] = __ldg(src + i + 32 * u);
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (i + 32 * u < pieces) dst[i + 32 * u] = x[u];
    }
    if (lane == 0 && !is_v) {
      if (pos != nullptr && c.pos != nullptr) c.pos[slot] = __ldg(&pos[row]);
      if (c.weight != nullptr) c.weight[slot] = 0.f;
    }
  }
  __shared__ bool last;
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();
    last = atomicAdd(arrived, 1) == (int)gridDim.x - 1;
  }
  __syncthreads();
  if (!last) return;
  if (threadIdx.x == 0) *arrived = 0;
  for (int b = threadIdx.x; b < c.n_seq; b += APPEND_WARPS * 32) {
    int first, n;
    call_rows(row_start, n_rows, b, first, n);
    check_starts(row_start, n_rows, b, status);
    const int64_t v = (int64_t)(at != nullptr ? at[b] : c.len[b]) + n;
    c.len[b] = (int32_t)(v < 0 ? 0 : v > capacity ? capacity : v);
  }
}

// ------------------------------------------------------------------------------------------------ attention, plain
constexpr int PL_THREADS = 256;
constexpr int PL_ROWS = 32;                    // queries of a tile: token x head of a KV head's group, heads inside
constexpr int PL_KEYS = 64;                    // rows of the cache in shared memory at a time
constexpr int PL_SPLIT = 8;                    // CTAs that share a tile's rows of the cache at most (a portable cluster)

template <typename T> __device__ __forceinline__ float4 load4(const T* p);
template <> __device__ __forceinline__ float4 load4<float>(const float* p) { return *reinterpret_cast<const float4*>(p); }
template <> __device__ __forceinline__ float4 load4<bf16>(const bf16* p) {
  const uint2 u = *reinterpret_cast<const uint2*>(p);
  return make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xFFFF0000u), __uint_as_float(u.y << 16), __uint_as_float(u.y & 0xFFFF0000u));
}
template <typename T> __device__ __forceinline__ void store4(T* p, float4 v);
template <> __device__ __forceinline__ void store4<float>(float* p, float4 v) { *reinterpret_cast<float4*>(p) = v; }
template <> __device__ __forceinline__ void store4<bf16>(bf16* p, float4 v) {
  __nv_bfloat162 a = __floats2bfloat162_rn(v.x, v.y), b = __floats2bfloat162_rn(v.z, v.w);
  *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<uint32_t*>(&a), *reinterpret_cast<uint32_t*>(&b));
}

// Rows [j0, j0 + PL_KEYS) of K or V of one KV head into shared memory, zeros from row `end` on and where the table names no page.
template <typename T, int D, int LD>
__device__ __forceinline__ void load_rows(const Cache& c, const T* __restrict__ x, int b, int kvh, int Hkv, int j0, int end, float* to, int* status) {
  constexpr int PER = D / 4;
  for (int i = threadIdx.x; i < PL_KEYS * PER; i += PL_THREADS) {
    const int r = i / PER, e = (i % PER) * 4, j = j0 + r;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (j < end) {
      const int64_t slot = slot_of(c, b, j);
      if (slot >= 0) v = load4(x + (slot * Hkv + kvh) * D + e);
      else set_status(status, SPTS_ERR_INDEX);
    }
    *reinterpret_cast<float4*>(to + r * LD + e) = v;
  }
}

// Queries [r0, r0 + PL_ROWS) of a sequence's rows x heads, zeros behind the last.
template <typename T, int D>
__device__ __forceinline__ void load_queries(const T* __restrict__ Q, int64_t ldq, int64_t first, int r0, int64_t rows, int kvh, int G, float* to) {
  constexpr int PER = D / 4;
  for (int i = threadIdx.x; i < PL_ROWS * PER; i += PL_THREADS) {
    const int r = i / PER, e = (i % PER) * 4;
    const int64_t q = (int64_t)r0 + r;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (q < rows) v = load4(Q + (first + q / G) * ldq + (int64_t)(kvh * G + q % G) * D + e);
    *reinterpret_cast<float4*>(to + r * D + e) = v;
  }
}

// Scores of queries tr and tr + 16 with keys tk, tk + 16, tk + 32, tk + 48 of the tiles in shared memory.
template <int D, int LD>
__device__ __forceinline__ void tile_scores(const float* sq, const float* sk, int tr, int tk, float (&s)[2][4]) {
#pragma unroll
  for (int a = 0; a < 2; ++a)
#pragma unroll
    for (int k = 0; k < 4; ++k) s[a][k] = 0.f;
#pragma unroll 4
  for (int e = 0; e < D; e += 4) {
    const float4 q0 = *reinterpret_cast<const float4*>(sq + tr * D + e), q1 = *reinterpret_cast<const float4*>(sq + (tr + 16) * D + e);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float4 x = *reinterpret_cast<const float4*>(sk + (tk + 16 * k) * LD + e);
      s[0][k] += q0.x * x.x + q0.y * x.y + q0.z * x.z + q0.w * x.w;
      s[1][k] += q1.x * x.x + q1.y * x.y + q1.z * x.z + q1.w * x.w;
    }
  }
}

template <int D> constexpr int plain_attn_smem() { return (PL_ROWS * D + PL_KEYS * (D + 4) + PL_KEYS * D + PL_ROWS * (PL_KEYS + 1)) * 4; }

// A cluster of CTAs per (tile of 32 queries, KV head): each takes a share of the rows that the tile sees, 64 at a time, online
// softmax, and the shares are joined in their order through distributed shared memory.  Fewer tiles than SMs are shared by up to
// eight CTAs (three ragged chunks of up to 37 tokens over up to 1000 rows, 4 heads of 64 dims in fp32).
template <typename T, int D>
__global__ void __launch_bounds__(PL_THREADS)
paged_attn_plain_kernel(Cache c, const T* __restrict__ Q, int64_t ldq, const int32_t* __restrict__ row_start, int n_rows, int H, int Hkv,
                        T* __restrict__ O, int64_t ldo, float* __restrict__ lse, int* status) {
  constexpr int LD = D + 4, PIECES = D / 64;
  extern __shared__ __align__(16) float smem_f[];
  float* sq = smem_f;
  float* sk = sq + PL_ROWS * D;
  float* sv = sk + PL_KEYS * LD;
  float* sp = sv + PL_KEYS * D;
  __shared__ float sm[PL_ROWS], sl[PL_ROWS], salpha[PL_ROWS];
  __shared__ long long pre[PREFIX_MAX + 1], sums[32];
  cg::cluster_group cluster = cg::this_cluster();
  const int split = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int G = H / Hkv, kvh = blockIdx.y, tid = threadIdx.x;
  const int64_t tile = blockIdx.x / split;
  block_prefix<PL_THREADS>(c.n_seq, pre, sums, [&](int b) {
    int f, n;
    call_rows(row_start, n_rows, b, f, n);
    if (kvh == 0 && tile == 0) check_starts(row_start, n_rows, b, status);
    return ((long long)n * G + PL_ROWS - 1) / PL_ROWS;
  });
  __syncthreads();
  if (tile >= pre[c.n_seq]) return;                   // (all CTAs of a cluster have the same tile)
  const int b = find_share(pre, c.n_seq, tile);
  int first, n;
  call_rows(row_start, n_rows, b, first, n);
  const int held = held_rows(c, b), off = held - n;
  const int r0 = (int)(tile - pre[b]) * PL_ROWS;
  const int64_t rows = (int64_t)n * G;
  const int seen = max(0, off + (int)min((int64_t)n, ((int64_t)r0 + PL_ROWS - 1) / G + 1));   // rows that the tile's last query sees
  load_queries<T, D>(Q, ldq, first, r0, rows, kvh, G, sq);
  if (tid < PL_ROWS) { sm[tid] = -INFINITY; sl[tid] = 0.f; }
  const float scale = rsqrtf((float)D);
  const int tr = tid >> 4, tk = tid & 15;
  // limit of a query: the rows that it sees
  int limit[2];
#pragma unroll
  for (int a = 0; a < 2; ++a) limit[a] = r0 + tr + 16 * a < rows ? off + (r0 + tr + 16 * a) / G + 1 : 0;
  float4 acc[2][PIECES];
#pragma unroll
  for (int a = 0; a < 2; ++a)
#pragma unroll
    for (int p = 0; p < PIECES; ++p) acc[a][p] = make_float4(0.f, 0.f, 0.f, 0.f);
  const int chunks = (seen + PL_KEYS - 1) / PL_KEYS;
  for (int ch = (int)((int64_t)chunks * rank / split); ch < (int)((int64_t)chunks * (rank + 1) / split); ++ch) {
    const int j0 = ch * PL_KEYS;
    __syncthreads();
    load_rows<T, D, LD>(c, (const T*)c.k, b, kvh, Hkv, j0, seen, sk, status);
    load_rows<T, D, D>(c, (const T*)c.v, b, kvh, Hkv, j0, seen, sv, status);
    __syncthreads();
    float s[2][4];
    tile_scores<D, LD>(sq, sk, tr, tk, s);
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
      for (int k = 0; k < 4; ++k) sp[(tr + 16 * a) * (PL_KEYS + 1) + tk + 16 * k] = j0 + tk + 16 * k < limit[a] ? s[a][k] * scale : -INFINITY;
    __syncthreads();
    // eight lanes to a query
    {
      const int r = tid >> 3, l8 = tid & 7;
      float* row = sp + r * (PL_KEYS + 1);
      float m = -INFINITY;
#pragma unroll
      for (int k = 0; k < PL_KEYS / 8; ++k) m = fmaxf(m, row[l8 + 8 * k]);
#pragma unroll
      for (int o = 4; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
      const float was = sm[r], now = fmaxf(was, m), base = now == -INFINITY ? 0.f : now;
      float sum = 0.f;
#pragma unroll
      for (int k = 0; k < PL_KEYS / 8; ++k) {
        const float p = expf(row[l8 + 8 * k] - base);
        row[l8 + 8 * k] = p;
        sum += p;
      }
#pragma unroll
      for (int o = 4; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      __syncwarp();
      if (l8 == 0) {
        const float alpha = was == -INFINITY ? 0.f : expf(was - base);
        salpha[r] = alpha;
        sm[r] = now;
        sl[r] = sl[r] * alpha + sum;
      }
    }
    __syncthreads();
    // O = alpha O + P V; a row that a query does not see has p = 0 and is passed over, whatever V holds
#pragma unroll
    for (int a = 0; a < 2; ++a) {
      const float alpha = salpha[tr + 16 * a];
#pragma unroll
      for (int p = 0; p < PIECES; ++p) { acc[a][p].x *= alpha; acc[a][p].y *= alpha; acc[a][p].z *= alpha; acc[a][p].w *= alpha; }
    }
    for (int k = 0; k < PL_KEYS; ++k) {
      const float w[2] = {sp[tr * (PL_KEYS + 1) + k], sp[(tr + 16) * (PL_KEYS + 1) + k]};
#pragma unroll
      for (int p = 0; p < PIECES; ++p) {
        const float4 v = *reinterpret_cast<const float4*>(sv + k * D + 64 * p + 4 * tk);
#pragma unroll
        for (int a = 0; a < 2; ++a) {
          if (w[a] != 0.f) {
            acc[a][p].x = fmaf(w[a], v.x, acc[a][p].x); acc[a][p].y = fmaf(w[a], v.y, acc[a][p].y);
            acc[a][p].z = fmaf(w[a], v.z, acc[a][p].z); acc[a][p].w = fmaf(w[a], v.w, acc[a][p].w);
          }
        }
      }
    }
  }
  // every CTA leaves its share in its own shared memory; query r is joined by CTA r % split
  __syncthreads();
#pragma unroll
  for (int a = 0; a < 2; ++a)
#pragma unroll
    for (int p = 0; p < PIECES; ++p) *reinterpret_cast<float4*>(sk + (tr + 16 * a) * D + 64 * p + 4 * tk) = acc[a][p];
  cluster.sync();
  for (int r = rank + split * (tid / (D / 4)); r < PL_ROWS; r += split * (PL_THREADS / (D / 4))) {
    const int e = (tid % (D / 4)) * 4;
    if (r0 + r >= rows) continue;
    float m = -INFINITY;
    for (int s = 0; s < split; ++s) m = fmaxf(m, *cluster.map_shared_rank(&sm[r], s));
    float l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s = 0; s < split; ++s) {
      const float ms = *cluster.map_shared_rank(&sm[r], s), ls = *cluster.map_shared_rank(&sl[r], s);
      if (ms == -INFINITY) continue;                    // saw none of its rows
      const float f = expf(ms - m);
      const float4 x = *reinterpret_cast<const float4*>(cluster.map_shared_rank(sk, s) + r * D + e);
      l += ls * f;
      o.x += x.x * f; o.y += x.y * f; o.z += x.z * f; o.w += x.w * f;
    }
    if (m == -INFINITY) { l = 1.f; o = make_float4(0.f, 0.f, 0.f, 0.f); }
    const int64_t token = first + (int64_t)(r0 + r) / G;
    const int head = kvh * G + (int)((r0 + r) % G);
    store4(O + token * ldo + (int64_t)head * D + e, make_float4(o.x / l, o.y / l, o.z / l, o.w / l));
    if (e == 0 && lse != nullptr) lse[token * H + head] = m + logf(l);
  }
  cluster.sync();
}

template <int D> constexpr int plain_weights_smem() { return (PL_ROWS * D + PL_KEYS * (D + 4) + 16 * PL_KEYS) * 4; }

// Persistent CTAs over (sequence, 64 rows of it); for every KV head its K in shared memory and the queries that see any of the rows
// passing by.  A thread sums its queries' weights of four rows; the sixteen threads of a row meet at the end, in their order.
template <typename T, int D>
__global__ void __launch_bounds__(PL_THREADS)
paged_weights_plain_kernel(Cache c, const T* __restrict__ Q, int64_t ldq, const int32_t* __restrict__ row_start, int n_rows, int H, int Hkv,
                           const float* __restrict__ lse, float decay, int* status) {
  constexpr int LD = D + 4;
  extern __shared__ __align__(16) float smem_f[];
  float* sq = smem_f;
  float* sk = sq + PL_ROWS * D;
  float* part = sk + PL_KEYS * LD;
  __shared__ long long pre[PREFIX_MAX + 1], sums[32];
  const int G = H / Hkv, tid = threadIdx.x, tr = tid >> 4, tk = tid & 15;
  const float scale = rsqrtf((float)D);
  block_prefix<PL_THREADS>(c.n_seq, pre, sums, [&](int b) {
    if (blockIdx.x == 0) check_starts(row_start, n_rows, b, status);
    return (long long)(held_rows(c, b) + PL_KEYS - 1) / PL_KEYS;
  });
  __syncthreads();
  const long long items = pre[c.n_seq];
  for (long long item = blockIdx.x; item < items; item += gridDim.x) {
    const int b = find_share(pre, c.n_seq, item);
    int first, n;
    call_rows(row_start, n_rows, b, first, n);
    const int held = held_rows(c, b), off = held - n, j0 = (int)(item - pre[b]) * PL_KEYS;
    const int64_t rows = (int64_t)n * G;
    // query i sees the first of these rows if off + i >= j0
    const int64_t from = (int64_t)max(0, j0 - off) * G / PL_ROWS * PL_ROWS;
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    for (int kvh = 0; kvh < Hkv && from < rows; ++kvh) {
      __syncthreads();
      load_rows<T, D, LD>(c, (const T*)c.k, b, kvh, Hkv, j0, held, sk, status);
      for (int64_t r0 = from; r0 < rows; r0 += PL_ROWS) {
        __syncthreads();
        load_queries<T, D>(Q, ldq, first, (int)r0, rows, kvh, G, sq);
        __syncthreads();
        float s[2][4];
        tile_scores<D, LD>(sq, sk, tr, tk, s);
#pragma unroll
        for (int a = 0; a < 2; ++a) {
          const int64_t r = r0 + tr + 16 * a;
          if (r >= rows) continue;
          const int limit = off + (int)(r / G) + 1;
          const float e = lse[(first + r / G) * H + kvh * G + (int)(r % G)];
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (j0 + tk + 16 * k < limit) sum[k] += expf(s[a][k] * scale - e);
        }
      }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; ++k) part[tr * PL_KEYS + tk + 16 * k] = sum[k];
    __syncthreads();
    if (tid < PL_KEYS && j0 + tid < held) {
      float w = 0.f;
      for (int i = 0; i < 16; ++i) w += part[i * PL_KEYS + tid];
      const int64_t slot = slot_of(c, b, j0 + tid);
      if (slot >= 0) c.weight[slot] = (decay == 0.f ? 0.f : decay * c.weight[slot]) + w / (float)H;
      else set_status(status, SPTS_ERR_INDEX);
    }
  }
}

// ------------------------------------------------------------------------------------------------ eviction
constexpr int RANK_THREADS = 1024;
constexpr int RANK_KEYS = 24576;               // rows of a CTA whose keys and positions fit shared memory
constexpr int MOVE_THREADS = 512;

// Order of the rows of a sequence: the larger key stays.  Rows that stay before all others have the largest one, NaN the smallest.
__device__ __forceinline__ uint32_t weight_key(float w) {
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w == 0.f ? 0.f : w);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

struct EvictArgs {
  Cache c;
  const int32_t* keep;
  int n_sink, n_recent;
  int first_seq;                               // of this launch
  int words;                                   // of evict_bits for each sequence
  uint32_t* bits; int2* before; int2* total;
  int* arrived;                                // blocks of the moves that are done, zero between calls
  int* status;
};

// A cluster of CTAs ranks one sequence's rows: each holds the keys of a contiguous part in shared memory; the smallest key that stays is
// found by a radix select of three digits (of eleven, eleven and ten bits), whose histograms meet in distributed shared memory (a thread for
// two bins, the CTAs' bins all on their way at once); of the rows that have just this key the first ones stay.  What comes out is a bit for each row, and the numbers of
// holes (rows among the first keep that go) and movers (rows behind them that stay) before each chunk of 256 rows, from which
// evict_move_kernel finds its copies.  Parts too long for shared memory (capacities beyond 196,608 rows) read their weights again for every
// digit.  Bound by the chain of barriers and round trips.
constexpr int BINS = 2 * RANK_THREADS;
static_assert(BINS == 2048, "two bins of a digit of eleven bits to a thread");

// Rows of a CTA's part of a sequence: whole words for each of its warps, whole chunks.
__host__ __device__ __forceinline__ int part_rows(int held, int split) {
  return (int)((((int64_t)held + split - 1) / split + RANK_THREADS - 1) / RANK_THREADS) * RANK_THREADS;
}
// Sum of v over the threads before this one.
__device__ __forceinline__ int block_above(int v, int (*warp_n)[3]) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int inc = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int other = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += other;
  }
  if (lane == 31) warp_n[warp][0] = inc;
  __syncthreads();
  const int w = warp_n[lane][0];
  return inc - v + __reduce_add_sync(0xffffffffu, lane < warp ? w : 0);
}

template <bool SMEM>
__global__ void __launch_bounds__(RANK_THREADS)
evict_rank_kernel(EvictArgs a) {
  extern __shared__ __align__(16) uint32_t keys[];                       // [part], then positions [part]
  __shared__ __align__(16) uint32_t hist[3][BINS];
  __shared__ long long newest_here, newest_all;
  __shared__ int ties_here, warp_n[RANK_THREADS / 32][3], s_need;
  __shared__ uint32_t s_digit;
  cg::cluster_group cluster = cg::this_cluster();
  const int split = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const Cache& c = a.c;
  const int local = blockIdx.x / split, b = a.first_seq + local, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  for (int i = tid; i < 3 * BINS; i += RANK_THREADS) (&hist[0][0])[i] = 0;
  dep_launch();
  dep_wait();
  const int held = held_rows(c, b), keep = a.keep[b];
  if (keep < 0 || held <= keep) return;        // (the same for all CTAs of a cluster)
  const int part = part_rows(held, split);
  const int j0 = (int)min((int64_t)held, (int64_t)rank * part), n = min(part, held - j0);
  uint32_t* spos = keys + part;
  if (tid == 0) { newest_here = LLONG_MIN; ties_here = 0; }
  __syncthreads();
  const bool by_pos = a.n_sink > 0 || a.n_recent > 0;
  // the rows' weights and positions, and the largest position that the sequence holds
  long long newest = LLONG_MIN;
  bool bad = false, none = false;
  if (SMEM || by_pos) {
#pragma unroll 4
    for (int i = tid; i < n; i += RANK_THREADS) {
      const int64_t slot = slot_of(c, b, j0 + i);
      if (SMEM) {
        const float w = slot >= 0 ? c.weight[slot] : 0.f;
        bad |= w != w;
        keys[i] = slot >= 0 ? weight_key(w) : 0u;
      }
      none |= slot < 0;
      if (by_pos && slot >= 0) {
        const int p = c.pos[slot];
        newest = max(newest, (long long)p);
        if (SMEM) spos[i] = (uint32_t)p;
      }
    }
  }
  if (bad) set_status(a.status, SPTS_ERR_NONFINITE);
  if (none) set_status(a.status, SPTS_ERR_INDEX);
  if (a.n_recent > 0) {
    for (int o = 16; o > 0; o >>= 1) newest = max(newest, __shfl_xor_sync(0xffffffffu, newest, o));
    if (lane == 0) atomicMax(&newest_here, newest);
    cluster.sync();
    if (warp == 0) {
      newest = lane < split ? *cluster.map_shared_rank(&newest_here, lane) : LLONG_MIN;
      for (int o = 16; o > 0; o >>= 1) newest = max(newest, __shfl_xor_sync(0xffffffffu, newest, o));
      if (lane == 0) newest_all = newest;
    }
    __syncthreads();
    newest = newest_all;
  }
  const auto stays_first = [&](int p) { return p < a.n_sink || (a.n_recent > 0 && (long long)p > newest - a.n_recent); };
  const auto key_at = [&](int i) -> uint32_t {
    if (SMEM) return keys[i];
    const int64_t slot = slot_of(c, b, j0 + i);
    if (slot < 0) { set_status(a.status, SPTS_ERR_INDEX); return 0u; }
    if (by_pos && stays_first(c.pos[slot])) return 0xFFFFFFFFu;
    const float w = c.weight[slot];
    if (w != w) set_status(a.status, SPTS_ERR_NONFINITE);
    return weight_key(w);
  };
  if (SMEM && by_pos)
    for (int i = tid; i < n; i += RANK_THREADS)
      if (stays_first((int)spos[i]) && slot_of(c, b, j0 + i) >= 0) keys[i] = 0xFFFFFFFFu;      // (a thread's own entries)
  // ---- the smallest key that stays
  uint32_t prefix = 0;
  int need = keep;                             // rows still to be taken among those with the digits found so far
  for (int d = 0; d < 3 && keep > 0; ++d) {
    const int shift = d == 0 ? 21 : d == 1 ? 10 : 0, known = d == 1 ? 21 : 10;
    const uint32_t mask = d == 2 ? 1023u : 2047u;
    for (int i = tid; i < n; i += RANK_THREADS) {
      const uint32_t k = key_at(i);
      if (d == 0 || (k >> known) == prefix) atomicAdd(&hist[d][(k >> shift) & mask], 1u);
    }
    cluster.sync();
    // thread t has bins BINS - 1 - 2 t and BINS - 2 - 2 t; sums run from the largest digit down
    uint2 bin = make_uint2(0u, 0u);            // (x: the lower one)
    {
      uint2 from[EVICT_SPLIT];
#pragma unroll
      for (int r = 0; r < EVICT_SPLIT; ++r)
        from[r] = r < split ? *reinterpret_cast<const uint2*>(cluster.map_shared_rank(&hist[d][0], r) + BINS - 2 - 2 * tid) : make_uint2(0u, 0u);
#pragma unroll
      for (int r = 0; r < EVICT_SPLIT; ++r) { bin.x += from[r].x; bin.y += from[r].y; }
    }
    const int above = block_above((int)(bin.x + bin.y), warp_n);
    if (above < need && above + (int)bin.y >= need) { s_digit = BINS - 1 - 2 * tid; s_need = need - above; }
    else if (above + (int)bin.y < need && above + (int)(bin.x + bin.y) >= need) { s_digit = BINS - 2 - 2 * tid; s_need = need - above - (int)bin.y; }
    __syncthreads();
    prefix = (prefix << (d == 2 ? 10 : 11)) | s_digit;
    need = s_need;
    __syncthreads();
  }
  // ---- a warp has part / 32 neighbouring rows from here on
  const bool cut = keep > 0;                   // (keep == 0: no row stays)
  const int per_warp = part / (RANK_THREADS / 32), w0 = warp * per_warp, w1 = min(n, w0 + per_warp);
  // rows that have just this key: how many lie in the parts and warps before
  int ties = 0;
  {
    int mine = 0;
    for (int i = w0 + lane; i < w1; i += 32) mine += cut && key_at(i) == prefix;
    mine = __reduce_add_sync(0xffffffffu, mine);
    if (lane == 0 && mine) atomicAdd(&ties_here, mine);
    if (lane == 0) warp_n[warp][0] = mine;
    cluster.sync();
    ties = __reduce_add_sync(0xffffffffu, (lane < rank ? *cluster.map_shared_rank(&ties_here, lane) : 0) + (lane < warp ? warp_n[lane][0] : 0));
  }
  // a bit for every row
  int holes = 0, movers = 0;
  const int64_t word0 = (int64_t)local * a.words;
  for (int i0 = w0; i0 < w1; i0 += 32) {
    const int i = i0 + lane, j = j0 + i;
    const uint32_t k = i < w1 ? key_at(i) : 0u;
    const bool tie = i < w1 && cut && k == prefix;
    const uint32_t tie_mask = __ballot_sync(0xffffffffu, tie);
    const bool stays = i < w1 && cut && (k > prefix || (tie && ties + __popc(tie_mask & ((1u << lane) - 1)) < need));
    ties += __popc(tie_mask);
    const uint32_t bits = __ballot_sync(0xffffffffu, stays);
    holes += __popc(__ballot_sync(0xffffffffu, i < w1 && !stays && j < keep));
    movers += __popc(__ballot_sync(0xffffffffu, stays && j >= keep));
    if (lane == 0) a.bits[word0 + (j >> 5)] = bits;      // (parts begin on a chunk, warps on a word)
    if (SMEM) {
      __syncwarp();
      if (lane == 0) keys[w0 + (i0 - w0) / 32] = bits;   // in the place of a row that is done with
    }
  }
  // holes and movers before each chunk
  if (lane == 0) { warp_n[warp][1] = holes; warp_n[warp][2] = movers; }
  __syncthreads();
  const int warp_holes = warp_n[lane][1], warp_movers = warp_n[lane][2];
  holes = __reduce_add_sync(0xffffffffu, lane < warp ? warp_holes : 0);
  movers = __reduce_add_sync(0xffffffffu, lane < warp ? warp_movers : 0);
  __syncwarp();
  for (int i0 = w0; i0 < w1; i0 += 32) {
    const int j = j0 + i0;
    const uint32_t bits = SMEM ? keys[w0 + (i0 - w0) / 32] : a.bits[word0 + (j >> 5)], there = w1 - i0 >= 32 ? 0xFFFFFFFFu : (1u << (w1 - i0)) - 1;
    const uint32_t front = j + 32 <= keep ? 0xFFFFFFFFu : j >= keep ? 0u : (1u << (keep - j)) - 1;       // rows below keep
    if (lane == 0 && j % EVICT_CHUNK == 0) a.before[(word0 >> 3) + j / EVICT_CHUNK] = make_int2(holes, movers);
    holes += __popc(~bits & there & front);
    movers += __popc(bits & ~front);
  }
  holes = __reduce_add_sync(0xffffffffu, warp_holes);
  movers = __reduce_add_sync(0xffffffffu, warp_movers);
  if (tid == 0) a.total[local * EVICT_SPLIT + rank] = make_int2(holes, movers);
  cluster.sync();                              // the histograms are read by other CTAs of the cluster until here
}

// Persistent CTAs over groups of sixteen movers: mover r of a sequence and its hole r are found by the numbers of movers and holes before
// each chunk (in shared memory), and all pieces of their rows are copied side by side.  Movers lie behind the rows that stay in place and
// holes among them, so no row is both read and written.  The block that is done last sets the lengths, which the others read.  Launched as a
// dependent of the ranking.
constexpr int MOVE_ROWS = 16;                  // movers of a group
constexpr int MOVE_AT_ONCE = 8;                // pieces of a thread in flight
constexpr int MOVE_CHUNKS = 4096;              // chunks of a sequence whose numbers fit shared memory (beyond 1,048,576 rows they are read where they lie)

// The row of `bits` (words of chunk `chunk`, those outside [from, to) left out) that is set for the (r + 1)-th time; -1: there is none.
__device__ __forceinline__ int nth_row(const uint32_t* bits, bool set, int chunk, int r, int from, int to) {
  const uint4* words = reinterpret_cast<const uint4*>(bits + (int64_t)chunk * (EVICT_CHUNK / 32));
  const uint4 w0 = __ldcg(words), w1 = __ldcg(words + 1);
  const uint32_t word[8] = {w0.x, w0.y, w0.z, w0.w, w1.x, w1.y, w1.z, w1.w};
  int found = -1;
#pragma unroll
  for (int w = 0; w < 8; ++w) {
    const int j = chunk * EVICT_CHUNK + 32 * w;
    uint32_t x = set ? word[w] : ~word[w];
    if (j < from) x &= from - j >= 32 ? 0u : ~0u << (from - j);
    if (j + 32 > to) x &= j >= to ? 0u : (1u << (to - j)) - 1;
    const int m = __popc(x);
    if (found < 0 && r < m) found = j + __fns(x, 0, r + 1);
    if (found < 0) r -= m;
  }
  return found;
}

__global__ void __launch_bounds__(MOVE_THREADS, 2)
evict_move_kernel(EvictArgs a, int n_seq, int split, int row_bytes) {
  __shared__ long long pre[PREFIX_MAX + 1], sums[32];
  __shared__ int64_t src[MOVE_ROWS], dst[MOVE_ROWS];       // places of the rows
  __shared__ int2 before[MOVE_CHUNKS];
  __shared__ bool last;
  const Cache& c = a.c;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  dep_wait();
  block_prefix<MOVE_THREADS>(n_seq, pre, sums, [&](int l) {
    const int held = held_rows(c, a.first_seq + l), keep = a.keep[a.first_seq + l];
    if (keep < 0 || held <= keep) return 0LL;
    int movers = 0;
#pragma unroll
    for (int s = 0; s < EVICT_SPLIT; ++s) movers += s < split ? __ldcg(&a.total[l * EVICT_SPLIT + s].y) : 0;
    return (long long)(movers + MOVE_ROWS - 1) / MOVE_ROWS;
  });
  __syncthreads();
  const long long items = pre[n_seq];
  int noted = -1;                              // the sequence whose numbers are in shared memory
  for (long long item = blockIdx.x; item < items; item += gridDim.x) {
    const int l = find_share(pre, n_seq, item), b = a.first_seq + l;
    const int held = held_rows(c, b), keep = a.keep[b];
    const int chunks = (held + EVICT_CHUNK - 1) / EVICT_CHUNK, per = part_rows(held, split) / EVICT_CHUNK;
    const int64_t word0 = (int64_t)l * a.words, chunk0 = word0 >> 3;
    const bool near = chunks <= MOVE_CHUNKS;
    if (near && noted != l) {
      for (int i = tid; i < chunks; i += MOVE_THREADS) before[i] = __ldcg(&a.before[chunk0 + i]);
      noted = l;
    }
    // holes and movers of the parts, one to a lane
    const int2 whole = lane < split ? __ldcg(&a.total[l * EVICT_SPLIT + lane]) : make_int2(0, 0);
    const int movers = __reduce_add_sync(0xffffffffu, whole.y);
    const int r0 = (int)(item - pre[l]) * MOVE_ROWS, n = min(MOVE_ROWS, movers - r0);
    __syncthreads();
    if (warp < 2) {
      // warp 0 finds the movers, warp 1 their holes
      const bool hole = warp == 1;
      int r = r0 + lane, s = 0;
#pragma unroll
      for (int u = 0; u < EVICT_SPLIT - 1; ++u) {
        const int here = __shfl_sync(0xffffffffu, hole ? whole.x : whole.y, u);
        if (s == u && u < split - 1 && r >= here) { r -= here; ++s; }
      }
      if (lane < n) {
        // the last chunk of part s with no more than r before it
        const auto number = [&](int chunk) {
          const int2 x = near ? before[chunk] : __ldcg(&a.before[chunk0 + chunk]);
          return hole ? x.x : x.y;
        };
        int lo = s * per, hi = min((s + 1) * per, chunks);
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if (number(mid) <= r) lo = mid; else hi = mid;
        }
        const int j = nth_row(a.bits + word0, !hole, lo, r - number(lo), hole ? 0 : keep, hole ? keep : held);
        (hole ? dst : src)[lane] = j < 0 ? -1 : slot_of(c, b, j);
      }
    }
    __syncthreads();
    // all rows' pieces of 16 bytes one after the other, K and V of a row in turn
    const int pieces = row_bytes >> 4, total = 2 * n * pieces;
    for (int u0 = tid; u0 < total; u0 += MOVE_AT_ONCE * MOVE_THREADS) {
      uint4 x[MOVE_AT_ONCE];
#pragma unroll
      for (int v = 0; v < MOVE_AT_ONCE; ++v) {
        const int u = u0 + v * MOVE_THREADS, r = u / pieces;
        if (u < total && src[r >> 1] >= 0)
          x[v] = reinterpret_cast<const uint4*>(((r & 1) ? c.v : c.k) + src[r >> 1] * row_bytes)[u - r * pieces];
      }
#pragma unroll
      for (int v = 0; v < MOVE_AT_ONCE; ++v) {
        const int u = u0 + v * MOVE_THREADS, r = u / pieces;
        if (u < total && src[r >> 1] >= 0 && dst[r >> 1] >= 0)
          reinterpret_cast<uint4*>(const_cast<char*>((r & 1) ? c.v : c.k) + dst[r >> 1] * row_bytes)[u - r * pieces] = x[v];
      }
    }
    if (tid < n && src[tid] >= 0 && dst[tid] >= 0) {
      c.weight[dst[tid]] = c.weight[src[tid]];
      if (c.pos != nullptr) c.pos[dst[tid]] = c.pos[src[tid]];
    }
    __syncthreads();
  }
  if (tid == 0) {
    __threadfence();
    last = atomicAdd(a.arrived, 1) == (int)gridDim.x - 1;
  }
  __syncthreads();
  if (!last) return;
  if (tid == 0) *a.arrived = 0;
  for (int l = tid; l < n_seq; l += MOVE_THREADS) {
    const int keep = a.keep[a.first_seq + l];
    if (keep >= 0 && held_rows(c, a.first_seq + l) > keep) c.len[a.first_seq + l] = keep;
  }
}

template <typename T, int D>
spts_status attn_plain_t(spts_ctx* ctx, const spts_paged_kv* cache, const void* Q, int64_t ldq, const int32_t* row_start, int n_rows,
                         void* O, int64_t ldo, float* lse) {
  const int H = ctx->desc.n_q_heads, Hkv = ctx->desc.n_kv_heads, G = H / Hkv;
  const int64_t tiles = (int64_t)n_rows * G / PL_ROWS + cache->n_seq;          // no fewer than there are
  const int split = tiles * Hkv <= ctx->sm_count / 2 ? PL_SPLIT : 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(tiles * split), Hkv);
  cfg.blockDim = dim3(PL_THREADS);
  cfg.dynamicSmemBytes = plain_attn_smem<D>();
  cfg.stream = ctx->stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = split; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, paged_attn_plain_kernel<T, D>, make_cache(cache), (const T*)Q, ldq, row_start, n_rows, H, Hkv, (T*)O, ldo, lse,
                         ctx->ws.status) != cudaSuccess)
    return SPTS_ERR_CUDA;
  ctx->launches++;
  return SPTS_OK;
}

template <typename T, int D>
spts_status weights_plain_t(spts_ctx* ctx, const spts_paged_kv* cache, const void* Q, int64_t ldq, const int32_t* row_start, int n_rows,
                            const float* lse, float decay) {
  const int64_t items = (int64_t)cache->n_seq * ceil_div(cache->max_pages * cache->page_size, PL_KEYS);
  const int grid = (int)(items < 3 * ctx->sm_count ? items : 3 * ctx->sm_count);
  paged_weights_plain_kernel<T, D><<<grid, PL_THREADS, plain_weights_smem<D>(), ctx->stream>>>(
      make_cache(cache), (const T*)Q, ldq, row_start, n_rows, ctx->desc.n_q_heads, ctx->desc.n_kv_heads, lse, decay, ctx->ws.status);
  SPTS_CUDA_OK(ctx);
  return SPTS_OK;
}

template <typename T, int D>
bool plain_attr() {
  return cudaFuncSetAttribute(paged_attn_plain_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, plain_attn_smem<D>()) == cudaSuccess &&
         cudaFuncSetAttribute(paged_weights_plain_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, plain_weights_smem<D>()) == cudaSuccess;
}

}  // namespace

spts_status paged_init(spts_ctx* ctx) {
  const bool ok = plain_attr<float, 64>() && plain_attr<float, 128>() && plain_attr<bf16, 64>() && plain_attr<bf16, 128>() &&
                  cudaFuncSetAttribute(evict_rank_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, RANK_KEYS * 8) == cudaSuccess;
  if (!ok) return SPTS_ERR_CUDA;
  return ctx->desc.dtype == SPTS_BF16 ? paged_tc_init(ctx) : SPTS_OK;
}

spts_status launch_paged_append(spts_ctx* ctx, const spts_paged_kv* cache, const void* K, int64_t ldk, const void* V, int64_t ldv,
                                const int32_t* pos, const int32_t* row_start, const int32_t* at, int n_rows) {
  const int es = ctx->desc.dtype == SPTS_BF16 ? 2 : 4, row_bytes = ctx->desc.n_kv_heads * ctx->desc.head_dim * es;
  const int64_t blocks = (2 * (int64_t)n_rows + APPEND_WARPS - 1) / APPEND_WARPS;
  const int grid = (int)(blocks < 1 ? 1 : blocks < 8 * ctx->sm_count ? blocks : 8 * ctx->sm_count);
  if (launch_dependent(paged_append_kernel, dim3(grid), dim3(APPEND_WARPS * 32), ctx->stream, make_cache(cache), (const char*)K, ldk * es,
                       (const char*)V, ldv * es, row_bytes, pos, row_start, at, n_rows, ctx->ws.paged_arrived, ctx->ws.status) != cudaSuccess)
    return SPTS_ERR_CUDA;
  ctx->launches++;
  return SPTS_OK;
}

spts_status launch_paged_attention(spts_ctx* ctx, const spts_paged_kv* cache, const void* Q, int64_t ldq, const int32_t* row_start,
                                   int n_rows, void* O, int64_t ldo, float* lse) {
  if (n_rows == 1) { ldq = 0; ldo = 0; }      // one row has no stride
  if (paged_tc(ctx)) return launch_paged_attention_tc(ctx, cache, Q, ldq, row_start, n_rows, O, ldo, lse);
  const bool d64 = ctx->desc.head_dim == 64;
  if (ctx->desc.dtype == SPTS_BF16)
    return d64 ? attn_plain_t<bf16, 64>(ctx, cache, Q, ldq, row_start, n_rows, O, ldo, lse)
               : attn_plain_t<bf16, 128>(ctx, cache, Q, ldq, row_start, n_rows, O, ldo, lse);
  return d64 ? attn_plain_t<float, 64>(ctx, cache, Q, ldq, row_start, n_rows, O, ldo, lse)
             : attn_plain_t<float, 128>(ctx, cache, Q, ldq, row_start, n_rows, O, ldo, lse);
}

spts_status launch_paged_weights(spts_ctx* ctx, const spts_paged_kv* cache, const void* Q, int64_t ldq, const int32_t* row_start,
                                 int n_rows, const float* lse, float decay) {
  if (n_rows == 1) ldq = 0;
  if (paged_tc(ctx)) return launch_paged_weights_tc(ctx, cache, Q, ldq, row_start, n_rows, lse, decay);
  const bool d64 = ctx->desc.head_dim == 64;
  if (ctx->desc.dtype == SPTS_BF16)
    return d64 ? weights_plain_t<bf16, 64>(ctx, cache, Q, ldq, row_start, n_rows, lse, decay)
               : weights_plain_t<bf16, 128>(ctx, cache, Q, ldq, row_start, n_rows, lse, decay);
  return d64 ? weights_plain_t<float, 64>(ctx, cache, Q, ldq, row_start, n_rows, lse, decay)
             : weights_plain_t<float, 128>(ctx, cache, Q, ldq, row_start, n_rows, lse, decay);
}

spts_status launch_paged_evict(spts_ctx* ctx, const spts_paged_kv* cache, const int32_t* keep, int n_sink, int n_recent) {
  const int es = ctx->desc.dtype == SPTS_BF16 ? 2 : 4, row_bytes = ctx->desc.n_kv_heads * ctx->desc.head_dim * es;
  const int capacity = cache->max_pages * cache->page_size;
  EvictArgs a;
  a.c = make_cache(cache); a.keep = keep; a.n_sink = n_sink; a.n_recent = n_recent;
  a.words = (int)align_up((size_t)capacity, EVICT_CHUNK) / 32;
  a.bits = ctx->ws.evict_bits; a.before = ctx->ws.evict_before; a.total = ctx->ws.evict_total; a.status = ctx->ws.status;
  a.arrived = ctx->ws.paged_arrived + 1;
  // one CTA ranks what it holds in a few rounds of its threads; longer sequences are shared by a cluster, whose barriers cost more
  const int split = capacity <= 8 * RANK_THREADS ? 1 : EVICT_SPLIT;
  const int part = part_rows(capacity, split);
  const bool smem = part <= RANK_KEYS;
  const int round = SPTS_PAGED_MAX_ROWS / (a.words * 32);             // sequences whose rows have a bit each in the workspace
  for (a.first_seq = 0; a.first_seq < cache->n_seq; a.first_seq += round) {
    const int n = cache->n_seq - a.first_seq < round ? cache->n_seq - a.first_seq : round;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(n * split));
    cfg.blockDim = dim3(RANK_THREADS);
    cfg.dynamicSmemBytes = smem ? part * 8 : 0;
    cfg.stream = ctx->stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = split; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    if (cudaLaunchKernelEx(&cfg, smem ? evict_rank_kernel<true> : evict_rank_kernel<false>, a) != cudaSuccess) return SPTS_ERR_CUDA;
    ctx->launches++;
    const int64_t items = (int64_t)n * a.words * 32 / (2 * MOVE_ROWS);         // no fewer than there are: at most half of the rows move
    const int move = (int)(items < 2 * ctx->sm_count ? items : 2 * ctx->sm_count);
    if (launch_dependent(evict_move_kernel, dim3(move), dim3(MOVE_THREADS), ctx->stream, a, n, split, row_bytes) != cudaSuccess) return SPTS_ERR_CUDA;
    ctx->launches++;
  }
  return SPTS_OK;
}

}  // namespace spts
