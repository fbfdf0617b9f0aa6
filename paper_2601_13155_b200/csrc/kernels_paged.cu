// The paged KV cache on CUDA cores: rows are appended to it (paged_append_kernel), attention and the weights that its rows gather in
// either storage type (paged_attn_*_kernel, paged_weights_*_kernel: fp32 storage, SPTS_REFERENCE_KERNELS, more than 128 query
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

// One warp copies a row's K, another its V, in 16-byte pieces, four in flight to a lane.  Lengths grow only once no block reads the old ones
// any more: the block that is done last sets them (one launch).  Bound by memory where rows are many (eight chunks of up to 4099 tokens,
// 118 MB: 22 us, 5.4 TB/s), else by the launch (one row of 64 sequences: 3.3 us).
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
    const int64_t j = (int64_t)(at != nullptr ? __ldg(&at[b]) : held_rows(c, b)) + (row - first);
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
  if (threadIdx.x == 0) last = count_arrival(arrived) == (int)gridDim.x - 1;
  __syncthreads();
  if (!last) return;
  if (threadIdx.x == 0) *arrived = 0;
  for (int b = threadIdx.x; b < c.n_seq; b += APPEND_WARPS * 32) {
    int first, n;
    call_rows(row_start, n_rows, b, first, n);
    check_starts(row_start, n_rows, b, status);
    const int64_t v = (int64_t)(at != nullptr ? at[b] : held_rows(c, b)) + n;
    c.len[b] = (int32_t)(v < 0 ? 0 : v > capacity ? capacity : v);
  }
}

// ------------------------------------------------------------------------------------------------ attention and weights, plain
// CUDA cores, fp32 arithmetic in either storage type.  Rows of queries are token x head of a KV head's group, heads inside.  Chunks of more
// than eight such rows to a sequence on average go 64 rows at a time against 64 rows of the cache in shared memory (tile kernels: bound by
// the multiply-adds and the shared memory that feeds them), shorter ones four at a time, straight from global memory (row kernels: bound by
// memory where there is enough to do).  Where that makes too few blocks, a cluster of up to eight shares a block's rows of the cache, or
// its heads and queries, and joins what it found in the order of its blocks.
constexpr int PL_THREADS = 256, PL_WARPS = PL_THREADS / 32;
constexpr int PL_SPLIT = 8;                    // CTAs that share a block's work at most (a portable cluster)
constexpr int TILE = 64;                       // tile kernels: rows of queries, rows of the cache
constexpr int FEW = 4, STEP = 8;               // row kernels: rows of queries, rows of the cache that a warp takes at a time
constexpr int FEW_MOST = 8;                    // rows of queries to a sequence up to which the row kernels are taken
constexpr int WARP_KEYS = 32;                  // row kernel of the weights: rows of the cache that belong to a warp
constexpr float SLACK = 8.0f;                  // log2 units the running maximum may lag behind
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

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
// the D / 32 dims of a row that belong to a lane
template <typename T, int PER> __device__ __forceinline__ void load_lane(const T* p, float (&x)[PER]) {
  if (PER == 4) {
    const float4 v = load4(p);
    x[0] = v.x; x[1] = v.y; x[PER - 2] = v.z; x[PER - 1] = v.w;
  } else {
#pragma unroll
    for (int e = 0; e < PER; ++e) x[e] = to_f32(p[e]);
  }
}

struct PlainArgs {
  Cache c;
  const int32_t* row_start; int n_rows, H, Hkv;
  const void* Q; int64_t ldq;
  void* O; int64_t ldo;
  float* lse;                                  // of the attention: written; of the weights: read
  float decay;
  int* status;
};

// The tile of queries that a block works on; all threads of a block, whose clusters have one tile.
struct QueryTile {
  int b, first, n, held, off;                  // sequence, its first query, how many, its rows, rows before the first query
  int64_t r0, rows;                            // first row of queries of the tile; of the sequence
  int seen;                                    // rows of the cache that the tile's last query sees
};
template <int ROWS>
__device__ __forceinline__ bool find_tile(const PlainArgs& a, int64_t tile, bool check, long long* pre, long long* sums, QueryTile& t) {
  const int G = a.H / a.Hkv;
  block_prefix<PL_THREADS>(a.c.n_seq, pre, sums, [&](int b) {
    int f, n;
    call_rows(a.row_start, a.n_rows, b, f, n);
    if (check) check_starts(a.row_start, a.n_rows, b, a.status);
    return ((long long)n * G + ROWS - 1) / ROWS;
  });
  __syncthreads();
  if (tile >= pre[a.c.n_seq]) return false;
  t.b = find_share(pre, a.c.n_seq, tile);
  call_rows(a.row_start, a.n_rows, t.b, t.first, t.n);
  t.held = held_rows(a.c, t.b);
  t.off = t.held - t.n;
  t.r0 = (tile - pre[t.b]) * ROWS;
  t.rows = (int64_t)t.n * G;
  t.seen = max(0, t.off + (int)min((int64_t)t.n, (t.r0 + ROWS - 1) / G + 1));
  return true;
}

// Shares of the CTAs of a cluster, of `rows` rows: maxima (log2 units) and sums in m and l, O [rows][D] in o, all in shared memory.  Row r is
// joined and written by CTA r % split.
template <typename T, int D>
__device__ __forceinline__ void join_cluster(cg::cluster_group& cluster, const PlainArgs& a, const QueryTile& t, int rows, int kvh, float* m, float* l, float* o) {
  const int split = (int)cluster.num_blocks(), rank = (int)cluster.block_rank(), G = a.H / a.Hkv, tid = threadIdx.x;
  cluster.sync();
  for (int r = rank + split * (tid / (D / 4)); r < rows; r += split * (PL_THREADS / (D / 4))) {
    const int e = (tid % (D / 4)) * 4;
    if (t.r0 + r >= t.rows) continue;
    float ms[PL_SPLIT], ls[PL_SPLIT], top = -INFINITY, sum = 0.f;
    float4 y[PL_SPLIT], x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int s = 0; s < PL_SPLIT; ++s) {                 // all on their way at once
      ms[s] = -INFINITY;
      ls[s] = 0.f;
      if (s >= split) continue;
      ms[s] = *cluster.map_shared_rank(&m[r], s);
      ls[s] = *cluster.map_shared_rank(&l[r], s);
      y[s] = *reinterpret_cast<const float4*>(cluster.map_shared_rank(o, s) + r * D + e);
    }
#pragma unroll
    for (int s = 0; s < PL_SPLIT; ++s) top = fmaxf(top, ms[s]);
#pragma unroll
    for (int s = 0; s < PL_SPLIT; ++s) {
      if (ms[s] == -INFINITY && ls[s] == 0.f) continue;  // saw none of its rows
      const float f = ms[s] == -INFINITY ? 1.f : exp2f(ms[s] - top);
      sum += ls[s] * f;
      x.x += y[s].x * f; x.y += y[s].y * f; x.z += y[s].z * f; x.w += y[s].w * f;
    }
    const bool none = sum == 0.f;
    const float inv = none ? 0.f : 1.0f / sum;
    const int64_t token = t.first + (t.r0 + r) / G;
    const int head = kvh * G + (int)((t.r0 + r) % G);
    store4((T*)a.O + token * a.ldo + (int64_t)head * D + e, none ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(x.x * inv, x.y * inv, x.z * inv, x.w * inv));
    if (e == 0 && a.lse != nullptr) a.lse[token * a.H + head] = none ? -INFINITY : (top + log2f(sum)) * LN2;
  }
  cluster.sync();
}

// ---- tile kernels
constexpr int PAD = 4;                         // floats between rows in shared memory: neighbouring rows in neighbouring banks
template <int D> constexpr int tile_floats() { return TILE * (D + PAD); }

// Rows [j0, j0 + TILE) of K (and V) of one KV head into shared memory, zeros from row `end` on and where the table names no page.
template <typename T, int D, bool BOTH>
__device__ __forceinline__ void load_rows(const PlainArgs& a, int b, int kvh, int j0, int end, float* to_k, float* to_v) {
  constexpr int PER = D / 4;
#pragma unroll 4
  for (int i = threadIdx.x; i < TILE * PER; i += PL_THREADS) {
    const int r = i / PER, e = (i % PER) * 4, j = j0 + r;
    float4 k = make_float4(0.f, 0.f, 0.f, 0.f), v = k;
    if (j < end) {
      const int64_t slot = slot_of(a.c, b, j);
      if (slot >= 0) {
        k = load4((const T*)a.c.k + (slot * a.Hkv + kvh) * D + e);
        if (BOTH) v = load4((const T*)a.c.v + (slot * a.Hkv + kvh) * D + e);
      } else {
        set_status(a.status, SPTS_ERR_INDEX);
      }
    }
    *reinterpret_cast<float4*>(to_k + r * (D + PAD) + e) = k;
    if (BOTH) *reinterpret_cast<float4*>(to_v + r * (D + PAD) + e) = v;
  }
}
// Rows of queries [r0, r0 + TILE), zeros behind the last: into registers, and from there, times `scale`, into shared memory.
template <int D> constexpr int query_pieces() { return TILE * D / 4 / PL_THREADS; }
template <typename T, int D>
__device__ __forceinline__ void fetch_queries(const PlainArgs& a, int64_t first, int64_t r0, int64_t rows, int kvh, float4 (&v)[query_pieces<D>()]) {
  constexpr int PER = D / 4;
  const int G = a.H / a.Hkv;
#pragma unroll
  for (int u = 0; u < query_pieces<D>(); ++u) {
    const int i = threadIdx.x + u * PL_THREADS, e = (i % PER) * 4;
    const int64_t q = r0 + i / PER;
    v[u] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (q < rows) v[u] = load4((const T*)a.Q + (first + q / G) * a.ldq + (int64_t)(kvh * G + q % G) * D + e);
  }
}
template <int D>
__device__ __forceinline__ void store_queries(const float4 (&v)[query_pieces<D>()], float scale, float* to) {
  constexpr int PER = D / 4;
#pragma unroll
  for (int u = 0; u < query_pieces<D>(); ++u) {
    const int i = threadIdx.x + u * PL_THREADS;
    *reinterpret_cast<float4*>(to + i / PER * (D + PAD) + (i % PER) * 4) = make_float4(v[u].x * scale, v[u].y * scale, v[u].z * scale, v[u].w * scale);
  }
}
// Products of rows 4 tq .. + 3 of queries and rows tk + 16 k of the cache.
template <int D>
__device__ __forceinline__ void tile_scores(const float* sq, const float* sk, int tq, int tk, float (&s)[4][4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int k = 0; k < 4; ++k) s[i][k] = 0.f;
#pragma unroll 4
  for (int e = 0; e < D; e += 4) {
    float4 q[4], x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = *reinterpret_cast<const float4*>(sq + (4 * tq + i) * (D + PAD) + e);
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = *reinterpret_cast<const float4*>(sk + (tk + 16 * k) * (D + PAD) + e);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) s[i][k] = fmaf(q[i].x, x[k].x, fmaf(q[i].y, x[k].y, fmaf(q[i].z, x[k].z, fmaf(q[i].w, x[k].w, s[i][k]))));
  }
}

// Adds the weights [TILE][TILE + PAD] of rows 4 tq .. + 3 times V to their dims 64 p + 4 tk .. + 3.
template <int D, bool PASS_ZEROS>
__device__ __forceinline__ void tile_pv(const float* sp, const float* sv, int tq, int tk, float4 (&acc)[4][D / 64]) {
#pragma unroll 2
  for (int k = 0; k < TILE; k += 4) {
    float4 w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = *reinterpret_cast<const float4*>(sp + (4 * tq + i) * (TILE + PAD) + k);
#pragma unroll
    for (int p = 0; p < D / 64; ++p) {
      float4 v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) v[u] = *reinterpret_cast<const float4*>(sv + (k + u) * (D + PAD) + 64 * p + 4 * tk);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float ws[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (!PASS_ZEROS || ws[u] != 0.f) {
            acc[i][p].x = fmaf(ws[u], v[u].x, acc[i][p].x); acc[i][p].y = fmaf(ws[u], v[u].y, acc[i][p].y);
            acc[i][p].z = fmaf(ws[u], v[u].z, acc[i][p].z); acc[i][p].w = fmaf(ws[u], v[u].w, acc[i][p].w);
          }
      }
    }
  }
}

template <int D> constexpr int attn_tile_smem() { return 3 * tile_floats<D>() * 4; }

// A cluster to (tile of 64 rows of queries, KV head).  A thread has 4 x 4 scores, then 4 rows x D / 16 dims of O; sixteen neighbouring threads
// share the rows, whose maxima and sums stay in registers.  The weights take K's place in shared memory.  fp32 storage, 32 heads of 128 dims:
// 1024 tokens over 4096 rows 1.9 ms (32 TFLOP/s; with 32 x 64 to a block and 8 scores to a thread 3.7), four chunks of 64 tokens 180 us.
template <typename T, int D>
__global__ void __launch_bounds__(PL_THREADS, 2)
paged_attn_tile_kernel(const __grid_constant__ PlainArgs a) {
  constexpr int PIECES = D / 64, LP = TILE + PAD;
  extern __shared__ __align__(16) float smem_f[];
  float* sq = smem_f;
  float* sk = sq + tile_floats<D>();
  float* sv = sk + tile_floats<D>();
  float* sp = sk;                              // [TILE][LP]
  __shared__ float sm[TILE], sl[TILE];
  __shared__ long long pre[PREFIX_MAX + 1], sums[32];
  cg::cluster_group cluster = cg::this_cluster();
  const int split = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int G = a.H / a.Hkv, kvh = blockIdx.y, tid = threadIdx.x, tq = tid >> 4, tk = tid & 15;
  QueryTile t;
  if (!find_tile<TILE>(a, blockIdx.x / split, kvh == 0 && blockIdx.x == 0, pre, sums, t)) return;
  {
    float4 q[query_pieces<D>()];
    fetch_queries<T, D>(a, t.first, t.r0, t.rows, kvh, q);
    store_queries<D>(q, LOG2E * rsqrtf((float)D), sq);
  }
  // rows of the cache that a query sees; those that all of the tile's see
  int limit[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t r = t.r0 + 4 * tq + i;
    limit[i] = r < t.rows ? t.off + (int)(r / G) + 1 : 0;
  }
  const int all = t.r0 + TILE <= t.rows ? t.off + (int)(t.r0 / G) + 1 : 0;
  float m[4], l[4];
  float4 acc[4][PIECES];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    m[i] = -INFINITY;
    l[i] = 0.f;
#pragma unroll
    for (int p = 0; p < PIECES; ++p) acc[i][p] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  const int chunks = (t.seen + TILE - 1) / TILE;
  for (int ch = (int)((int64_t)chunks * rank / split); ch < (int)((int64_t)chunks * (rank + 1) / split); ++ch) {
    const int j0 = ch * TILE;
    const bool whole = j0 + TILE <= all;
    __syncthreads();
    load_rows<T, D, true>(a, t.b, kvh, j0, t.seen, sk, sv);
    __syncthreads();
    float s[4][4];
    tile_scores<D>(sq, sk, tq, tk, s);
    __syncthreads();                           // K is done with
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (!whole) {
#pragma unroll
        for (int k = 0; k < 4; ++k) s[i][k] = j0 + tk + 16 * k < limit[i] ? s[i][k] : -INFINITY;
      }
      float top = fmaxf(fmaxf(s[i][0], s[i][1]), fmaxf(s[i][2], s[i][3]));
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      if (top > m[i] + SLACK || m[i] == -INFINITY) {
        const float alpha = m[i] == -INFINITY ? 0.f : exp2f(m[i] - top);
        m[i] = top;
        l[i] *= alpha;
#pragma unroll
        for (int p = 0; p < PIECES; ++p) { acc[i][p].x *= alpha; acc[i][p].y *= alpha; acc[i][p].z *= alpha; acc[i][p].w *= alpha; }
      }
      const float base = m[i] == -INFINITY ? 0.f : m[i];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float p = exp2f(s[i][k] - base);
        l[i] += p;
        sp[(4 * tq + i) * LP + tk + 16 * k] = p;
      }
    }
    __syncthreads();
    // O += P V; where a query does not see all of the rows, those of weight zero are passed over, whatever V holds
    if (whole) tile_pv<D, false>(sp, sv, tq, tk, acc);
    else tile_pv<D, true>(sp, sv, tq, tk, acc);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], o);
    if (tk == 0) { sm[4 * tq + i] = m[i]; sl[4 * tq + i] = l[i]; }
#pragma unroll
    for (int p = 0; p < PIECES; ++p) *reinterpret_cast<float4*>(sv + (4 * tq + i) * D + 64 * p + 4 * tk) = acc[i][p];
  }
  join_cluster<T, D>(cluster, a, t, TILE, kvh, sm, sl, sv);
}

// Blocks of the cache for the weights: (sequence, ROWS rows of it); all threads.
template <int ROWS>
__device__ __forceinline__ long long blocks_of_rows(const PlainArgs& a, bool check, long long* pre, long long* sums) {
  block_prefix<PL_THREADS>(a.c.n_seq, pre, sums, [&](int b) {
    if (check) check_starts(a.row_start, a.n_rows, b, a.status);
    return (long long)(held_rows(a.c, b) + ROWS - 1) / ROWS;
  });
  __syncthreads();
  return pre[a.c.n_seq];
}
// The sums [rows] of the CTAs of a cluster, which had different heads or queries, are added in their order and become weights.
__device__ __forceinline__ void write_weights(cg::cluster_group& cluster, const PlainArgs& a, int b, int held, int j0, int rows, float* sum) {
  const int split = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  cluster.sync();
  for (int i = rank * PL_THREADS + threadIdx.x; i < rows; i += split * PL_THREADS) {
    if (j0 + i >= held) continue;
    float w = 0.f;
#pragma unroll
    for (int s = 0; s < PL_SPLIT; ++s)
      if (s < split) w += *cluster.map_shared_rank(&sum[i], s);
    const int64_t slot = slot_of(a.c, b, j0 + i);
    if (slot >= 0) a.c.weight[slot] = (a.decay == 0.f ? 0.f : a.decay * a.c.weight[slot]) + w / (float)a.H;
    else set_status(a.status, SPTS_ERR_INDEX);
  }
  cluster.sync();
}

template <int D> constexpr int weights_tile_smem() { return (2 * tile_floats<D>() + 16 * TILE) * 4; }

// Persistent clusters over (sequence, 64 rows of it); a CTA has a part of the KV heads and tiles of queries that see any of the rows: a head's K in
// shared memory, the queries passing by.  A thread sums its queries' weights of four rows; the sixteen threads of a row meet at the end, in their order.
// 1024 tokens over 4096 rows, 32 heads, fp32: 1.28 ms (23 TFLOP/s; with queries fetched as they are needed 1.36, with one CTA to 64 rows and 8
// scores to a thread 5.2).
template <typename T, int D>
__global__ void __launch_bounds__(PL_THREADS, 2)
paged_weights_tile_kernel(const __grid_constant__ PlainArgs a) {
  extern __shared__ __align__(16) float smem_f[];
  float* sq = smem_f;
  float* sk = sq + tile_floats<D>();
  float* part = sk + tile_floats<D>();         // [16][TILE]
  __shared__ float sum_all[TILE], slse[TILE];
  __shared__ long long pre[PREFIX_MAX + 1], sums[32];
  cg::cluster_group cluster = cg::this_cluster();
  const int split = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int G = a.H / a.Hkv, tid = threadIdx.x, tq = tid >> 4, tk = tid & 15;
  const long long items = blocks_of_rows<TILE>(a, blockIdx.x == 0, pre, sums);
  for (long long item = blockIdx.x / split; item < items; item += gridDim.x / split) {
    const int b = find_share(pre, a.c.n_seq, item);
    int first, n;
    call_rows(a.row_start, a.n_rows, b, first, n);
    const int held = held_rows(a.c, b), off = held - n, j0 = (int)(item - pre[b]) * TILE;
    const int64_t rows = (int64_t)n * G;
    // query i sees the first of these rows if off + i >= j0
    const int64_t from = (int64_t)max(0, j0 - off) * G / TILE * TILE;
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    // this CTA's part of the pairs (KV head, tile of queries), head by head
    const int64_t tiles = rows > from ? (rows - from + TILE - 1) / TILE : 0, p1 = tiles * a.Hkv * (rank + 1) / split;
    int64_t pair = tiles * a.Hkv * rank / split;
    float4 q[query_pieces<D>()];               // the next tile of queries, on its way
    float e = 0.f;
    const auto fetch = [&](int64_t pair) {
      const int kvh = (int)(pair / tiles);
      const int64_t r0 = from + pair % tiles * TILE, r = r0 + tid;
      fetch_queries<T, D>(a, first, r0, rows, kvh, q);
      if (tid < TILE) e = r < rows ? a.lse[(first + r / G) * a.H + kvh * G + (int)(r % G)] * LOG2E : 0.f;
    };
    if (pair < p1) fetch(pair);
    int in_k = -1;                             // the head whose K is in shared memory
    for (; pair < p1; ++pair) {
      const int kvh = (int)(pair / tiles);
      const int64_t r0 = from + pair % tiles * TILE;
      __syncthreads();
      if (kvh != in_k) load_rows<T, D, false>(a, b, kvh, j0, held, sk, nullptr);
      in_k = kvh;
      store_queries<D>(q, LOG2E * rsqrtf((float)D), sq);
      if (tid < TILE) slse[tid] = e == -INFINITY ? 0.f : e;        // (such a query sees nothing)
      __syncthreads();
      if (pair + 1 < p1) fetch(pair + 1);
      float s[4][4];
      tile_scores<D>(sq, sk, tq, tk, s);
      const bool whole = r0 + TILE <= rows && j0 + TILE <= off + (int)(r0 / G) + 1;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t r = r0 + 4 * tq + i;
        const int limit = whole ? INT_MAX : r < rows ? off + (int)(r / G) + 1 : 0;
        const float base = slse[4 * tq + i];
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (j0 + tk + 16 * k < limit) sum[k] += exp2f(s[i][k] - base);
      }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; ++k) part[tq * TILE + tk + 16 * k] = sum[k];
    __syncthreads();
    if (tid < TILE) {
      float w = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) w += part[i * TILE + tid];
      sum_all[tid] = w;
    }
    write_weights(cluster, a, b, held, j0, TILE, sum_all);
  }
}

// ---- row kernels
// Totals over the lanes of v[32]: lane i gets that of v[i].
__device__ __forceinline__ float lane_totals(float (&v)[32]) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const bool high = lane & o;
#pragma unroll
    for (int i = 0; i < o; ++i) {
      const float keep = high ? v[i + o] : v[i], give = high ? v[i] : v[i + o];
      v[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
    }
  }
  return v[0];
}
// Scores of four rows of queries and eight of the cache: lane 8 r + k gets that of row r and k.
template <int PER>
__device__ __forceinline__ float few_scores(const float (&q)[FEW][PER], const float (&k)[STEP][PER]) {
  float v[32];
#pragma unroll
  for (int r = 0; r < FEW; ++r)
#pragma unroll
    for (int u = 0; u < STEP; ++u) {
      float x = 0.f;
#pragma unroll
      for (int e = 0; e < PER; ++e) x = fmaf(q[r][e], k[u][e], x);
      v[STEP * r + u] = x;
    }
  return lane_totals(v);
}
template <typename T, int D>
__device__ __forceinline__ void load_few(const PlainArgs& a, int64_t first, int64_t r0, int64_t rows, int kvh, float (&q)[FEW][D / 32]) {
  const int G = a.H / a.Hkv, lane = threadIdx.x & 31;
  const float scale = LOG2E * rsqrtf((float)D);
#pragma unroll
  for (int r = 0; r < FEW; ++r) {
#pragma unroll
    for (int e = 0; e < D / 32; ++e) q[r][e] = 0.f;
    const int64_t x = r0 + r;
    if (x < rows) load_lane<T, D / 32>((const T*)a.Q + (first + x / G) * a.ldq + (int64_t)(kvh * G + x % G) * D + lane * (D / 32), q[r]);
#pragma unroll
    for (int e = 0; e < D / 32; ++e) q[r][e] *= scale;
  }
}

// A cluster to (four rows of queries, KV head); each warp takes every eighth step of eight rows of the cache of the CTA's share, the lanes
// hold D / 32 dims of everything; the warps' results meet in shared memory.  Where a step's rows lie is looked up a step ahead.  32 single
// tokens over up to 4096 rows, 32 heads, fp32: 118 us, 3.7 TB/s (eight rows of queries against four of the cache, looked up in place: 298).
template <typename T, int D>
__global__ void __launch_bounds__(PL_THREADS, 2)
paged_attn_row_kernel(const __grid_constant__ PlainArgs a) {
  constexpr int PER = D / 32;
  __shared__ __align__(16) float so[PL_WARPS][FEW * D];
  __shared__ __align__(16) float sp[PL_WARPS][32];
  __shared__ float sm[PL_WARPS][FEW], sl[PL_WARPS][FEW], tm[FEW], tl[FEW];
  __shared__ long long pre[PREFIX_MAX + 1], sums[32];
  cg::cluster_group cluster = cg::this_cluster();
  const int split = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int G = a.H / a.Hkv, kvh = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  QueryTile t;
  if (!find_tile<FEW>(a, blockIdx.x / split, kvh == 0 && blockIdx.x == 0, pre, sums, t)) return;
  float q[FEW][PER], acc[FEW][PER];
  load_few<T, D>(a, t.first, t.r0, t.rows, kvh, q);
#pragma unroll
  for (int r = 0; r < FEW; ++r)
#pragma unroll
    for (int e = 0; e < PER; ++e) acc[r][e] = 0.f;
  // this lane's row of queries and its place in a step
  const int64_t mine = t.r0 + lane / STEP;
  const int limit = mine < t.rows ? t.off + (int)(mine / G) + 1 : 0, at = lane % STEP;
  const int all = t.r0 + FEW <= t.rows ? t.off + (int)(t.r0 / G) + 1 : 0;      // rows that all of the tile's queries see
  float m = -INFINITY, l = 0.f;
  const int steps = (t.seen + STEP - 1) / STEP, s1 = (int)((int64_t)steps * (rank + 1) / split);
  const auto look_up = [&](int st) -> int64_t {          // where row `at` of a step is
    const int j = st * STEP + at;
    if (st >= s1 || j >= t.seen) return -1;
    const int64_t slot = slot_of(a.c, t.b, j);
    if (slot < 0) set_status(a.status, SPTS_ERR_INDEX);
    return slot;
  };
  int st = (int)((int64_t)steps * rank / split) + warp;
  int64_t next = look_up(st);
  for (; st < s1; st += PL_WARPS) {
    const int j0 = st * STEP;
    const int64_t slot = next;
    float k[STEP][PER], v[STEP][PER];
#pragma unroll
    for (int u = 0; u < STEP; ++u) {
#pragma unroll
      for (int e = 0; e < PER; ++e) { k[u][e] = 0.f; v[u][e] = 0.f; }
      const int64_t x = __shfl_sync(0xffffffffu, slot, u);
      if (x < 0) continue;
      load_lane<T, PER>((const T*)a.c.k + (x * a.Hkv + kvh) * D + lane * PER, k[u]);
      load_lane<T, PER>((const T*)a.c.v + (x * a.Hkv + kvh) * D + lane * PER, v[u]);
    }
    next = look_up(st + PL_WARPS);
    float s = few_scores<PER>(q, k);
    const bool whole = j0 + STEP <= all;
    if (!whole && j0 + at >= limit) s = -INFINITY;
    float top = s;
#pragma unroll
    for (int o = 1; o < STEP; o *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    float alpha = 1.f;
    if (top > m + SLACK || m == -INFINITY) {
      alpha = m == -INFINITY ? 0.f : exp2f(m - top);
      m = top;
    }
    const float p = exp2f(s - (m == -INFINITY ? 0.f : m));
    l = l * alpha + p;
    sp[warp][lane] = p;
    if (__any_sync(0xffffffffu, alpha != 1.f)) {
#pragma unroll
      for (int r = 0; r < FEW; ++r) {
        const float f = __shfl_sync(0xffffffffu, alpha, STEP * r);
#pragma unroll
        for (int e = 0; e < PER; ++e) acc[r][e] *= f;
      }
    }
    __syncwarp();
#pragma unroll
    for (int r = 0; r < FEW; ++r) {
      const float4 w0 = *reinterpret_cast<const float4*>(&sp[warp][STEP * r]), w1 = *reinterpret_cast<const float4*>(&sp[warp][STEP * r + 4]);
      const float w[STEP] = {w0.x, w0.y, w0.z, w0.w, w1.x, w1.y, w1.z, w1.w};
#pragma unroll
      for (int u = 0; u < STEP; ++u)
        if (whole || w[u] != 0.f) {
#pragma unroll
          for (int e = 0; e < PER; ++e) acc[r][e] = fmaf(w[u], v[u][e], acc[r][e]);
        }
    }
    __syncwarp();
  }
#pragma unroll
  for (int o = 1; o < STEP; o *= 2) l += __shfl_xor_sync(0xffffffffu, l, o);
  if (at == 0) { sm[warp][lane / STEP] = m; sl[warp][lane / STEP] = l; }
#pragma unroll
  for (int r = 0; r < FEW; ++r)
#pragma unroll
    for (int e = 0; e < PER; ++e) so[warp][r * D + lane * PER + e] = acc[r][e];
  __syncthreads();
  // warp r joins row r of the CTA's warps
  if (warp < FEW) {
    const int r = warp;
    float top = -INFINITY, sum = 0.f, o[PER];
#pragma unroll
    for (int w = 0; w < PL_WARPS; ++w) top = fmaxf(top, sm[w][r]);
#pragma unroll
    for (int e = 0; e < PER; ++e) o[e] = 0.f;
#pragma unroll
    for (int w = 0; w < PL_WARPS; ++w) {
      if (sm[w][r] == -INFINITY && sl[w][r] == 0.f) continue;
      const float f = sm[w][r] == -INFINITY ? 1.f : exp2f(sm[w][r] - top);
      sum += sl[w][r] * f;
#pragma unroll
      for (int e = 0; e < PER; ++e) o[e] += so[w][r * D + lane * PER + e] * f;
    }
#pragma unroll
    for (int e = 0; e < PER; ++e) so[0][r * D + lane * PER + e] = o[e];      // (no other warp reads row r)
    if (lane == 0) { tm[r] = top; tl[r] = sum; }
  }
  join_cluster<T, D>(cluster, a, t, FEW, kvh, tm, tl, so[0]);
}

// Persistent clusters over (sequence, 256 rows of it), 32 to a warp; a CTA has every split-th KV head, whose queries stay in registers while
// the warp's rows pass.  32 single tokens over up to 4096 rows, 32 heads, fp32: 104 us, 2.1 TB/s.
template <typename T, int D>
__global__ void __launch_bounds__(PL_THREADS, 2)
paged_weights_row_kernel(const __grid_constant__ PlainArgs a) {
  constexpr int PER = D / 32, ROWS = PL_WARPS * WARP_KEYS, STEPS = WARP_KEYS / STEP;
  __shared__ float sum_all[ROWS];
  __shared__ long long pre[PREFIX_MAX + 1], sums[32];
  cg::cluster_group cluster = cg::this_cluster();
  const int split = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int G = a.H / a.Hkv, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, at = lane % STEP;
  const long long items = blocks_of_rows<ROWS>(a, blockIdx.x == 0, pre, sums);
  for (long long item = blockIdx.x / split; item < items; item += gridDim.x / split) {
    const int b = find_share(pre, a.c.n_seq, item);
    int first, n;
    call_rows(a.row_start, a.n_rows, b, first, n);
    const int held = held_rows(a.c, b), off = held - n, block0 = (int)(item - pre[b]) * ROWS, j0 = block0 + warp * WARP_KEYS;
    const int64_t rows = (int64_t)n * G, from = (int64_t)max(0, j0 - off) * G / FEW * FEW;
    float sum[STEPS];
#pragma unroll
    for (int st = 0; st < STEPS; ++st) sum[st] = 0.f;
    const int64_t slot = j0 + lane < held ? slot_of(a.c, b, j0 + lane) : -1;       // (lane i: of row j0 + i)
    for (int kvh = rank; kvh < a.Hkv && j0 < held; kvh += split) {
      for (int64_t r0 = from; r0 < rows; r0 += FEW) {
        float q[FEW][PER];
        load_few<T, D>(a, first, r0, rows, kvh, q);
        const int64_t mine = r0 + lane / STEP;
        const int limit = mine < rows ? off + (int)(mine / G) + 1 : 0;
        float e = mine < rows ? a.lse[(first + mine / G) * a.H + kvh * G + (int)(mine % G)] * LOG2E : 0.f;
        if (e == -INFINITY) e = 0.f;                                   // (such a query sees nothing)
#pragma unroll
        for (int st = 0; st < STEPS; ++st) {
          float k[STEP][PER];
#pragma unroll
          for (int u = 0; u < STEP; ++u) {
            const int64_t x = __shfl_sync(0xffffffffu, slot, st * STEP + u);
#pragma unroll
            for (int i = 0; i < PER; ++i) k[u][i] = 0.f;
            if (x >= 0) load_lane<T, PER>((const T*)a.c.k + (x * a.Hkv + kvh) * D + lane * PER, k[u]);
          }
          const float s = few_scores<PER>(q, k);
          if (j0 + st * STEP + at < limit) sum[st] += exp2f(s - e);
        }
      }
    }
#pragma unroll
    for (int st = 0; st < STEPS; ++st) {
      float w = sum[st];
#pragma unroll
      for (int o = STEP; o < 32; o *= 2) w += __shfl_xor_sync(0xffffffffu, w, o);
      if (lane < STEP) sum_all[warp * WARP_KEYS + st * STEP + lane] = w;
    }
    __syncthreads();
    write_weights(cluster, a, b, held, block0, ROWS, sum_all);
  }
}

// ------------------------------------------------------------------------------------------------ eviction
constexpr int RANK_THREADS = 1024;
constexpr int RANK_KEYS = 24576;               // rows of a CTA whose keys and positions fit shared memory
// Rows that go up to which the ranking kernel moves those that stay.  (48 sequences of 4096 rows and n more, ranked and moved by the second
// kernel 29.6 us, by the first for n = 1, 16, 32: 22.2, 22.8, 23.6; one of 32768: 29.5 and 23.7, 25.8, 27.7.)
constexpr int RANK_MOVES = 32;
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
  int row_bytes;                               // of K, of V
  uint32_t* bits; int2* before; int2* total;
  int* arrived;                                // blocks of the moves that are done, zero between calls
  int* status;
};

// A cluster of CTAs ranks one sequence's rows: each holds the keys of a contiguous part in shared memory; the smallest key that stays is
// found by a radix select of three digits (of eleven, eleven and ten bits), whose histograms meet in distributed shared memory (a thread for
// two bins, the CTAs' bins all on their way at once); of the rows that have just this key the first ones stay.  What comes out is a bit for
// each row, and the numbers of holes (rows among the first keep that go) and movers (rows behind them that stay) before each chunk of 256
// rows, from which evict_move_kernel finds its copies.  Parts too long for shared memory (capacities beyond 196,608 rows) read their weights again for every
// digit.  Where no more than RANK_MOVES rows go, as of a sequence that is held at its budget, no more move, and the first CTA moves them.
// Bound by the chain of barriers and round trips (with the moves 28 us for 32768 rows of which 4096 stay, 20 for 48 sequences of 4111 and less).
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
  __shared__ bool s_all;
  __shared__ int2 s_part;
  __shared__ int s_src[RANK_MOVES], s_dst[RANK_MOVES];
  __shared__ int64_t s_from[RANK_MOVES], s_to[RANK_MOVES];
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
  const bool few = held - keep <= RANK_MOVES;  // no more rows move than go: the first CTA moves them itself
  const int part = part_rows(held, split);
  const int j0 = (int)min((int64_t)held, (int64_t)rank * part), n = min(part, held - j0);
  uint32_t* spos = keys + part;
  if (tid == 0) { newest_here = LLONG_MIN; ties_here = 0; }
  if (tid < RANK_MOVES) { s_src[tid] = -1; s_dst[tid] = -1; }
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
    const float w = c.weight[slot];            // (a NaN is reported of rows that stay whatever they weigh, too, as above)
    if (w != w) set_status(a.status, SPTS_ERR_NONFINITE);
    return by_pos && stays_first(c.pos[slot]) ? 0xFFFFFFFFu : weight_key(w);
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
    const int upper = above + (int)bin.y, both = upper + (int)bin.x;
    if (above < need && upper >= need) { s_digit = BINS - 1 - 2 * tid; s_need = need - above; s_all = upper == need; }
    else if (upper < need && both >= need) { s_digit = BINS - 2 - 2 * tid; s_need = need - upper; s_all = both == need; }
    __syncthreads();
    prefix = (prefix << (d == 2 ? 10 : 11)) | s_digit;
    need = s_need;
    const bool all = s_all;
    __syncthreads();
    if (all) {                                 // all rows with these digits stay: the others do not matter
      prefix <<= shift;
      need = INT_MAX;
      break;
    }
  }
  // ---- a warp has part / 32 neighbouring rows from here on
  const bool cut = keep > 0;                   // (keep == 0: no row stays)
  const int per_warp = part / (RANK_THREADS / 32), w0 = warp * per_warp, w1 = min(n, w0 + per_warp);
  // rows that have just this key, where not all of them stay: how many lie in the parts and warps before
  int ties = 0;
  if (cut && need != INT_MAX) {
    int mine = 0;
    for (int i = w0 + lane; i < w1; i += 32) mine += key_at(i) == prefix;
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
  const int2 whole = make_int2(__reduce_add_sync(0xffffffffu, warp_holes), __reduce_add_sync(0xffffffffu, warp_movers));
  int* to_src = s_src;
  int* to_dst = s_dst;
  if (few && split > 1) {
    // the first CTA's lists, and the numbers of the parts before
    to_src = cluster.map_shared_rank(s_src, 0);
    to_dst = cluster.map_shared_rank(s_dst, 0);
    if (tid == 0) s_part = whole;
    cluster.sync();
    const int2 other = lane < rank ? *cluster.map_shared_rank(&s_part, lane) : make_int2(0, 0);
    holes += __reduce_add_sync(0xffffffffu, other.x);
    movers += __reduce_add_sync(0xffffffffu, other.y);
  }
  __syncwarp();
  for (int i0 = w0; i0 < w1; i0 += 32) {
    const int j = j0 + i0;
    const uint32_t bits = SMEM ? keys[w0 + (i0 - w0) / 32] : a.bits[word0 + (j >> 5)], there = w1 - i0 >= 32 ? 0xFFFFFFFFu : (1u << (w1 - i0)) - 1;
    const uint32_t front = j + 32 <= keep ? 0xFFFFFFFFu : j >= keep ? 0u : (1u << (keep - j)) - 1;       // rows below keep
    const uint32_t hole = ~bits & there & front, mover = bits & ~front;
    if (few) {
      const uint32_t below = (1u << lane) - 1;
      const int to_hole = holes + __popc(hole & below), to_mover = movers + __popc(mover & below);
      if ((hole >> lane & 1) && to_hole < RANK_MOVES) to_dst[to_hole] = j + lane;
      if ((mover >> lane & 1) && to_mover < RANK_MOVES) to_src[to_mover] = j + lane;
    } else if (lane == 0 && j % EVICT_CHUNK == 0) {
      a.before[(word0 >> 3) + j / EVICT_CHUNK] = make_int2(holes, movers);
    }
    holes += __popc(hole);
    movers += __popc(mover);
  }
  if (tid == 0 && !few) a.total[local * EVICT_SPLIT + rank] = whole;
  cluster.sync();                              // other CTAs of the cluster read the histograms and write the lists until here
  if (!few || rank > 0) return;
  if (tid < 2 * RANK_MOVES) {
    const int r = tid % RANK_MOVES, src = s_src[r], dst = s_dst[r];
    const bool there = src >= 0 && dst >= 0;
    (tid < RANK_MOVES ? s_from : s_to)[r] = there ? slot_of(c, b, tid < RANK_MOVES ? src : dst) : -1;
  }
  __syncthreads();
  const int pieces = a.row_bytes >> 4, n_moves = min(held - keep, RANK_MOVES);
  for (int u0 = tid; u0 < 2 * n_moves * pieces; u0 += 4 * RANK_THREADS) {
    uint4 x[4];
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const int u = u0 + v * RANK_THREADS, r = u / pieces;
      if (r < 2 * n_moves && s_from[r >> 1] >= 0)
        x[v] = reinterpret_cast<const uint4*>(((r & 1) ? c.v : c.k) + s_from[r >> 1] * a.row_bytes)[u - r * pieces];
    }
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const int u = u0 + v * RANK_THREADS, r = u / pieces;
      if (r < 2 * n_moves && s_from[r >> 1] >= 0 && s_to[r >> 1] >= 0)
        reinterpret_cast<uint4*>(const_cast<char*>((r & 1) ? c.v : c.k) + s_to[r >> 1] * a.row_bytes)[u - r * pieces] = x[v];
    }
  }
  if (tid < n_moves && s_from[tid] >= 0 && s_to[tid] >= 0) {
    c.weight[s_to[tid]] = c.weight[s_from[tid]];
    if (c.pos != nullptr) c.pos[s_to[tid]] = c.pos[s_from[tid]];
  }
}

// Persistent CTAs over groups of sixteen movers: mover r of a sequence and its hole r are found by the numbers of movers and holes before
// each chunk (in shared memory), and all pieces of their rows are copied side by side.  Movers lie behind the rows that stay in place and
// holes among them, so no row is both read and written.  The block that is done last sets the lengths, which the others read.  Launched as a
// dependent of the ranking, which has moved the rows of sequences that give up 32 or fewer.  Sixteen movers to a group spread even few of
// them over the SMs: with whole chunks of 256 rows to a CTA the two kernels took 46 us for 32768 rows of which 4096 stay, with groups 31.
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
evict_move_kernel(EvictArgs a, int n_seq, int split) {
  __shared__ long long pre[PREFIX_MAX + 1], sums[32];
  __shared__ int64_t src[MOVE_ROWS], dst[MOVE_ROWS];       // places of the rows
  __shared__ int2 before[MOVE_CHUNKS];
  __shared__ bool last;
  const Cache& c = a.c;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  dep_wait();
  block_prefix<MOVE_THREADS>(n_seq, pre, sums, [&](int l) {
    const int held = held_rows(c, a.first_seq + l), keep = a.keep[a.first_seq + l];
    if (keep < 0 || held - RANK_MOVES <= keep) return 0LL;
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
    const int row_bytes = a.row_bytes, pieces = row_bytes >> 4, total = 2 * n * pieces;
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
  if (items > 0) {
    if (tid == 0) last = count_arrival(a.arrived) == (int)gridDim.x - 1;
    __syncthreads();
    if (!last) return;
    if (tid == 0) *a.arrived = 0;
  } else if (blockIdx.x > 0) {
    return;                                    // (nothing moves, whatever length the others read)
  }
  for (int l = tid; l < n_seq; l += MOVE_THREADS) {
    const int keep = a.keep[a.first_seq + l];
    if (keep >= 0 && held_rows(c, a.first_seq + l) > keep) c.len[a.first_seq + l] = keep;
  }
}

// A cluster of `split` CTAs to a block of work.
spts_status launch_clusters(spts_ctx* ctx, void (*kernel)(PlainArgs), dim3 grid, int split, int smem, const PlainArgs& a) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(PL_THREADS);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = ctx->stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = split; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, kernel, a) != cudaSuccess) return SPTS_ERR_CUDA;
  ctx->launches++;
  return SPTS_OK;
}
// CTAs that share a block of work: as many as make eight blocks to an SM, a power of two.  (When this was chosen, 32 single tokens over 4096
// rows with two, four and eight to an SM: attention 175, 128, 123 us, weights 88, 93, 101; four chunks of
// 64: 316, 229, 228 and 140, 112, 106.)
int share_of(const spts_ctx* ctx, int64_t blocks, int most) {
  int split = 1;
  while (2 * split <= most && blocks * split < 8 * ctx->sm_count) split *= 2;
  return split;
}
// (By the batch's average: 63 single tokens beside a chunk of 512, 2048 rows each, go by tiles as well and take 1590 us, weights 2120, where
// the two by themselves take 212 + 586 and 239 + 327.)
bool few_rows(const spts_ctx* ctx, const spts_paged_kv* cache, int n_rows) {
  return (int64_t)n_rows * (ctx->desc.n_q_heads / ctx->desc.n_kv_heads) <= (int64_t)FEW_MOST * cache->n_seq;
}

template <typename T, int D>
spts_status attn_plain_t(spts_ctx* ctx, const spts_paged_kv* cache, const PlainArgs& a) {
  const bool few = few_rows(ctx, cache, a.n_rows);
  const int64_t tiles = (int64_t)a.n_rows * (a.H / a.Hkv) / (few ? FEW : TILE) + cache->n_seq;       // no fewer than there are
  // a share has 64 rows of the cache at least (32 sequences of up to 68 rows: without this limit 74 us)
  const int chunks = ceil_div(cache->max_pages * cache->page_size, TILE);
  const int split = share_of(ctx, tiles * a.Hkv, chunks < PL_SPLIT ? chunks : PL_SPLIT);
  const dim3 grid((unsigned)(tiles * split), a.Hkv);
  return few ? launch_clusters(ctx, paged_attn_row_kernel<T, D>, grid, split, 0, a)
             : launch_clusters(ctx, paged_attn_tile_kernel<T, D>, grid, split, attn_tile_smem<D>(), a);
}

template <typename T, int D>
spts_status weights_plain_t(spts_ctx* ctx, const spts_paged_kv* cache, const PlainArgs& a) {
  const bool few = few_rows(ctx, cache, a.n_rows);
  const int64_t most = (int64_t)cache->n_seq * ceil_div(cache->max_pages * cache->page_size, few ? PL_WARPS * WARP_KEYS : TILE);
  // a share has one head at least, of the tile kernel one head and tile of queries
  const int64_t parts = few ? a.Hkv : a.Hkv * ((int64_t)a.n_rows * (a.H / a.Hkv) / TILE + 1);
  const int split = share_of(ctx, most, parts < PL_SPLIT ? (int)parts : PL_SPLIT);
  const int64_t resident = 4 * ctx->sm_count / split;
  const dim3 grid((unsigned)((most < resident ? most : resident) * split));
  return few ? launch_clusters(ctx, paged_weights_row_kernel<T, D>, grid, split, 0, a)
             : launch_clusters(ctx, paged_weights_tile_kernel<T, D>, grid, split, weights_tile_smem<D>(), a);
}

template <typename T, int D>
bool plain_attr() {
  return cudaFuncSetAttribute(paged_attn_tile_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, attn_tile_smem<D>()) == cudaSuccess &&
         cudaFuncSetAttribute(paged_weights_tile_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, weights_tile_smem<D>()) == cudaSuccess;
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
  const PlainArgs a = {make_cache(cache), row_start, n_rows, ctx->desc.n_q_heads, ctx->desc.n_kv_heads, Q, ldq, O, ldo, lse, 0.f, ctx->ws.status};
  const bool d64 = ctx->desc.head_dim == 64;
  if (ctx->desc.dtype == SPTS_BF16) return d64 ? attn_plain_t<bf16, 64>(ctx, cache, a) : attn_plain_t<bf16, 128>(ctx, cache, a);
  return d64 ? attn_plain_t<float, 64>(ctx, cache, a) : attn_plain_t<float, 128>(ctx, cache, a);
}

spts_status launch_paged_weights(spts_ctx* ctx, const spts_paged_kv* cache, const void* Q, int64_t ldq, const int32_t* row_start,
                                 int n_rows, const float* lse, float decay) {
  if (n_rows == 1) ldq = 0;
  if (paged_tc(ctx)) return launch_paged_weights_tc(ctx, cache, Q, ldq, row_start, n_rows, lse, decay);
  const PlainArgs a = {make_cache(cache), row_start, n_rows, ctx->desc.n_q_heads, ctx->desc.n_kv_heads, Q, ldq, nullptr, 0, const_cast<float*>(lse), decay,
                       ctx->ws.status};
  const bool d64 = ctx->desc.head_dim == 64;
  if (ctx->desc.dtype == SPTS_BF16) return d64 ? weights_plain_t<bf16, 64>(ctx, cache, a) : weights_plain_t<bf16, 128>(ctx, cache, a);
  return d64 ? weights_plain_t<float, 64>(ctx, cache, a) : weights_plain_t<float, 128>(ctx, cache, a);
}

spts_status launch_paged_evict(spts_ctx* ctx, const spts_paged_kv* cache, const int32_t* keep, int n_sink, int n_recent) {
  const int es = ctx->desc.dtype == SPTS_BF16 ? 2 : 4, row_bytes = ctx->desc.n_kv_heads * ctx->desc.head_dim * es;
  const int capacity = cache->max_pages * cache->page_size;
  EvictArgs a;
  a.c = make_cache(cache); a.keep = keep; a.n_sink = n_sink; a.n_recent = n_recent; a.row_bytes = row_bytes;
  a.words = (int)align_up((size_t)capacity, EVICT_CHUNK) / 32;
  a.bits = ctx->ws.evict_bits; a.before = ctx->ws.evict_before; a.total = ctx->ws.evict_total; a.status = ctx->ws.status;
  a.arrived = ctx->ws.paged_arrived + 1;
  // one CTA ranks what it holds in a few rounds of its threads; longer sequences are shared by a cluster, whose barriers cost more.  The lengths
  // lie on the device, so this goes by the room that the table has: 48 sequences of up to 4111 rows take 19.4 us in tables of 4128 rows, 23.3 in
  // tables of 32768, 26.4 in tables of 262144, whose parts would not fit shared memory (one of 32768 rows: 28.0, 28.2 and 34.4).
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
    if (launch_dependent(evict_move_kernel, dim3(move), dim3(MOVE_THREADS), ctx->stream, a, n, split) != cudaSuccess) return SPTS_ERR_CUDA;
    ctx->launches++;
  }
  return SPTS_OK;
}

}  // namespace spts
