// The 4-bit KV cache: rows are quantised into it (kv4_append_kernel) and single tokens attend to it.
//
// kv4_attn_kernel (bf16): persistent CTAs, whose warps stream steps of 16 or 32 rows of the cache through shared memory into
// warp-level matrix instructions; see there.
// kv4_attn_plain_kernel: a cluster of up to eight CTAs per query head and sequence, CUDA cores, fp32 arithmetic, online softmax per
// warp, the warps' and CTAs' results joined in their order.  Bound by the latency of a warp's steps (loads, sum over lanes,
// exponential): 3 sequences of 1000 rows, 4 heads of 64 dims in fp32 6.4 us (one CTA per head, row by row, took 35); one of 32768
// rows, 32 heads of 128 in bf16 336 us (the matrix kernel: 18).  fp32 storage and SPTS_REFERENCE_KERNELS.
#include <cooperative_groups.h>

#include "q4_common.cuh"

namespace spts {

namespace {

using namespace q4;
namespace cg = cooperative_groups;

struct Kv4Dev {
  char* k_codes; char* v_codes; uint32_t* k_params; uint32_t* v_params;
  int32_t* pos; int32_t* len;
  int n_seq, capacity, group, Hkv;
};

// One unit = one (row, KV head) of K or of V: D / 8 lanes, eight dims each, 256 / D units to a warp pass; quantised, its words
// stored in the cache's order.  A warp takes up to `per` passes of one row (blockIdx.y: which, and of K or V), so that the row's
// sequence is looked up once and the pointers only move.
// 18,442 rows of 8 heads x 128 with their values read back take 60 us, where memory asks for 27 (each element read once, codes,
// params and values written once; in fp32 61 us, where it asks for 50): the quantiser's instructions (300 to a pass of 256 elements) bound it, at four blocks to an SM
// (three 65 us, five 67).  64 single rows: 4.8 us, two launches.
template <typename T, int D, int LANES>
__global__ void __launch_bounds__(256, 4)
kv4_append_kernel(Kv4Dev c, const T* __restrict__ K, int64_t ldk, const T* __restrict__ V, int64_t ldv,
                  const int32_t* __restrict__ pos, const int32_t* __restrict__ row_start, const int32_t* __restrict__ at,
                  int n_rows, int per, T* __restrict__ K_read, T* __restrict__ V_read, int* status) {
  constexpr int LPR = D / 8, UPW = 32 / LPR;       // lanes per unit, units per warp pass
  const int lane = threadIdx.x & 31, sub = lane % LPR;
  const int passes = (c.Hkv + UPW - 1) / UPW, parts = (passes + per - 1) / per;
  const bool is_v = (int)blockIdx.y >= parts;
  const int p0 = ((int)blockIdx.y - (is_v ? parts : 0)) * per, p1 = min(passes, p0 + per);
  const T* src0 = (is_v ? V : K) + p0 * 256 + 8 * lane;
  T* read0 = is_v ? V_read : K_read;
  const int64_t ld = is_v ? ldv : ldk;
  char* codes0 = is_v ? c.v_codes : c.k_codes;
  uint32_t* params0 = is_v ? c.v_params : c.k_params;
  // dims 32 t + 8 q .. of a row are word q D / 32 + t of a key; of a value they are two halfwords D / 16 bytes apart, and the
  // lanes of blocks t and t ^ 1 exchange one each to store whole words
  const int t = sub >> 2, q = sub & 3;
  const int at_word = is_v ? (2 * q + (t & 1)) * (D / 64) + (t >> 1) : q * (D / 32) + t;
  for (int row = blockIdx.x * 8 + (threadIdx.x >> 5); row < n_rows; row += gridDim.x * 8) {
    // the sequence that owns the row: the last b with row_start[b] <= row
    int b = row, first_row = row;
    if (row_start != nullptr) {
      int lo = 0, hi = c.n_seq;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (__ldg(&row_start[mid]) <= row) lo = mid; else hi = mid;
      }
      b = lo;
      first_row = max(0, __ldg(&row_start[b]));
      if (row < first_row || row >= __ldg(&row_start[b + 1])) continue;
    }
    const long slot = (long)(at != nullptr ? __ldg(&at[b]) : __ldg(&c.len[b])) + (row - first_row);
    const bool room = slot >= 0 && slot < c.capacity;
    if (!room && lane == 0) set_status(status, SPTS_ERR_WORKSPACE);
    if (pos != nullptr && c.pos != nullptr && room && blockIdx.y == 0 && lane == 0) c.pos[(size_t)b * c.capacity + slot] = pos[row];
    int kvh = p0 * UPW + lane / LPR;
    const T* src = src0 + (size_t)row * ld;
    T* read_to = read0 != nullptr ? read0 + (size_t)row * c.Hkv * D + p0 * 256 + 8 * lane : nullptr;
    const size_t r = ((size_t)b * c.Hkv + kvh) * c.capacity + (room ? slot : 0);
    uint32_t* codes = reinterpret_cast<uint32_t*>(codes0 + r * (D / 2)) + at_word;
    uint32_t* params = params0 + r * (LPR / LANES) + sub / LANES;
    Raw8<T> next;                                  // the next pass's elements are on their way while this one's are quantised
    next.zero();
    if (kvh < c.Hkv) next.load(src);
    for (int p = p0; p < p1; ++p) {
      const bool in = kvh < c.Hkv;
      float x[8];
      next.get(x);
      if (p + 1 < p1 && kvh + UPW < c.Hkv) next.load(src + 256);
      else next.zero();
      uint32_t prm;
      bool bad;
      float read[8];
      uint32_t w = quantize8<LANES>(K, x, prm, read, bad);
      if (is_v) {
        const uint32_t other = __shfl_xor_sync(0xffffffffu, (t & 1) ? w : w >> 16, 4);
        w = (t & 1) ? __byte_perm(other, w, 0x7610) : __byte_perm(w, other, 0x5410);
      }
      if (in) {
        if (bad) set_status(status, SPTS_ERR_NONFINITE);
        if (read_to != nullptr) store8(read_to, read);
        if (room) {
          *codes = w;
          if (sub % LANES == 0) *params = prm;
        }
      }
      kvh += UPW;
      src += 256;
      if (read_to != nullptr) read_to += 256;
      codes += (size_t)UPW * c.capacity * (D / 8);
      params += (size_t)UPW * c.capacity * (LPR / LANES);
    }
  }
}

// len[b] = at[b] + rows of b, clipped; a kernel of its own behind the append, whose blocks still read the old lengths.  Only rows
// that there are count: what a start claims outside [0, n_rows) was never written.
__global__ void kv4_len_kernel(int32_t* len, const int32_t* __restrict__ at, const int32_t* __restrict__ row_start, int n_seq,
                               int capacity, int n_rows, int* status) {
  const int b = blockIdx.x * blockDim.x + threadIdx.x;
  if (b >= n_seq) return;
  long n = 1;
  if (row_start != nullptr) {
    const int r0 = row_start[b], r1 = row_start[b + 1];
    if (r0 < 0 || r1 < r0 || r1 > n_rows) set_status(status, SPTS_ERR_INDEX);
    n = max(0L, (long)min(r1, n_rows) - max(r0, 0));
  }
  const long v = (long)(at != nullptr ? at[b] : len[b]) + n;
  len[b] = (int32_t)(v < 0 ? 0 : v > capacity ? capacity : v);
}

constexpr int PLAIN_WARPS = 16;
constexpr int PLAIN_ROWS = 4;                      // rows of a warp's step: their loads and sums over lanes run side by side
constexpr int PLAIN_SPLIT = 8;                     // CTAs per query head at most (a portable cluster)

// blockIdx.x = a cluster's CTAs, which share the rows of query head blockIdx.y in sequence blockIdx.z
template <typename T, int D>
__global__ void __launch_bounds__(PLAIN_WARPS * 32)
kv4_attn_plain_kernel(Kv4Dev c, const T* __restrict__ Q, int64_t ldq, int H, T* __restrict__ O, int64_t ldo) {
  constexpr int E = D / 32;                        // storage positions per lane
  __shared__ float sm_m[PLAIN_WARPS], sm_l[PLAIN_WARPS];
  __shared__ float sm_o[PLAIN_WARPS][D];
  __shared__ float sm_part[D + 2];                 // the CTA's O, sum and maximum
  cg::cluster_group cluster = cg::this_cluster();
  const int split = gridDim.x, rank = blockIdx.x;
  const int h = blockIdx.y, b = blockIdx.z, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int kvh = h / (H / c.Hkv);
  const int len = max(0, min(c.len[b], c.capacity));
  T* out = O + (size_t)b * ldo + (size_t)h * D;
  float q[E], o[E];
  int gk[E], gv[E], dv[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int p = lane * E + e;
    const int dk = 32 * ((p / 8) % (D / 32)) + 8 * (p / (D / 4)) + p % 8;
    dv[e] = 32 * ((p / 4) % (D / 32)) + 4 * (p / (D / 8)) + p % 4;
    gk[e] = dk / c.group; gv[e] = dv[e] / c.group;
    q[e] = to_f32(Q[(size_t)b * ldq + (size_t)h * D + dk]) * rsqrtf((float)D);
    o[e] = 0.f;
  }
  float m = -INFINITY, l = 0.f;
  const size_t base = ((size_t)b * c.Hkv + kvh) * c.capacity;
  const int ng = D / c.group;
  auto codes = [&](const char* at, size_t r) -> uint32_t {
    return E == 4 ? reinterpret_cast<const uint16_t*>(at + r * (D / 2))[lane] : reinterpret_cast<const uint8_t*>(at + r * (D / 2))[lane];
  };
  const int step = split * PLAIN_WARPS * PLAIN_ROWS;
  for (int64_t j = (int64_t)(rank * PLAIN_WARPS + warp) * PLAIN_ROWS; j < len; j += step) {
    uint32_t kw[PLAIN_ROWS], vw[PLAIN_ROWS], kp[PLAIN_ROWS][E], vp[PLAIN_ROWS][E];
#pragma unroll
    for (int i = 0; i < PLAIN_ROWS; ++i) {
      const size_t r = base + (j + i < len ? j + i : j);       // rows behind the end: the step's first one, of weight 0
      kw[i] = codes(c.k_codes, r);
      vw[i] = codes(c.v_codes, r);
#pragma unroll
      for (int e = 0; e < E; ++e) { kp[i][e] = c.k_params[r * ng + gk[e]]; vp[i][e] = c.v_params[r * ng + gv[e]]; }
    }
    float s[PLAIN_ROWS];
    float mn = m;
#pragma unroll
    for (int i = 0; i < PLAIN_ROWS; ++i) {
      s[i] = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e)
        s[i] = fmaf(q[e], fmaf(lo_bf16(kp[i][e]), code_less_8(kw[i], e), hi_bf16(kp[i][e])), s[i]);
    }
#pragma unroll
    for (int i = 0; i < PLAIN_ROWS; ++i) {
      s[i] = warp_sum(s[i]);
      if (j + i < len) mn = fmaxf(mn, s[i]);
    }
    // a NaN score (non-finite rows in the cache) goes on as NaN
    const float corr = m == -INFINITY ? 0.f : expf(m - mn);
    float pr[PLAIN_ROWS];
    l *= corr;
#pragma unroll
    for (int i = 0; i < PLAIN_ROWS; ++i) {
      pr[i] = j + i >= len || s[i] == -INFINITY ? 0.f : expf(s[i] - mn);
      l += pr[i];
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
      o[e] *= corr;
#pragma unroll
      for (int i = 0; i < PLAIN_ROWS; ++i)
        if (j + i < len)
          o[e] = fmaf(pr[i], fmaf(lo_bf16(vp[i][e]), code_less_8(vw[i], e), hi_bf16(vp[i][e])), o[e]);
    }
    m = mn;
  }
  if (lane == 0) { sm_m[warp] = m; sm_l[warp] = l; }
#pragma unroll
  for (int e = 0; e < E; ++e) sm_o[warp][dv[e]] = o[e];
  __syncthreads();
  if (threadIdx.x < D) {
    const int dim = threadIdx.x;
    float M = -INFINITY, L = 0.f, a = 0.f;
    for (int w = 0; w < PLAIN_WARPS; ++w) M = fmaxf(M, sm_m[w]);
    for (int w = 0; w < PLAIN_WARPS; ++w) {
      const float f = sm_m[w] == -INFINITY ? 0.f : expf(sm_m[w] - M);
      L += sm_l[w] * f;
      a = fmaf(sm_o[w][dim], f, a);
    }
    sm_part[dim] = a;
    if (dim == 0) { sm_part[D] = L; sm_part[D + 1] = M; }
  }
  cluster.sync();
  if (rank == 0 && threadIdx.x < D) {
    float M = -INFINITY, L = 0.f, a = 0.f;
    for (int x = 0; x < split; ++x) M = fmaxf(M, cluster.map_shared_rank(sm_part, x)[D + 1]);
    for (int x = 0; x < split; ++x) {
      const float* part = cluster.map_shared_rank(sm_part, x);
      const float f = part[D + 1] == -INFINITY ? 0.f : expf(part[D + 1] - M);
      L += part[D] * f;
      a = fmaf(part[threadIdx.x], f, a);
    }
    out[threadIdx.x] = from_f32<T>(len > 0 ? a / L : 0.f);
  }
  cluster.sync();                                  // no CTA leaves while its part is being read
}

// ---------------------------------------------------------------------------------------------------------------------
// Attention of single tokens on matrix instructions (m16n8k16, fp32 accumulation).
//
// A warp takes tiles of 16 cached rows of one KV head and all query heads that read it (up to 8 NB):
//   S[row, q] = K Q^T    M = 16 rows, N = queries, K = dims        O[dim, q] += V^T P    M = 16 dims, N = queries, K = 16 rows
// so that the codes are always the A operand and no lane is spent on absent queries beyond eight.  What bounds the kernel is
// the instructions between the codes and the matrix units, so they are few: codes enter as fp16 by masks alone (code_pair),
// scales and mids stay outside in fp32:
//   S = sum_groups scale_g (sum_i c_i q_i) + sum_g (mid_g - 8 scale_g) (sum_i q_i)
// q is brought to fp16 by a power of two per query (exact: bf16 has fewer bits; only elements below 2^-26 of the query's largest are
// rounded, off by up to 2^-34 of it).  The second sum is one more matrix step, in bf16, whose A registers are the params words as
// they lie in memory and whose B holds -8 sum q and sum q in two bf16 pieces each (off by 2^-17 relative).
//   O = sum_rows c p'_g - 8 sum_rows p'_g + sum_rows p mid_g,   p'_g = fp16(p scale_g / r), p in the last sum in two bf16 pieces
// (2^-17: mids may be far larger than scales, and the sum of the weights that divides O is that of the unrounded ones; with one
// piece a constant V came back off by up to 2^-8)
// r is a power of two near the size of the largest scale met, so p' uses fp16's eleven bits down to 2^-20 of the largest weight, and its
// absolute error below that is 2^-31; the -8 multiplies the rounded p' by a matrix step with a constant A, so it cancels up
// to fp32 sums.  P changes from the accumulator's layout to the B operand's by 8 x 8 transposes between lanes.
// The running maximum is a reference, not the maximum: it moves only when a score exceeds it by 2^6 (r likewise by 2), which
// after the first rows is rare, so the steps carry no reduction.
//
// Work split: the steps (one or two tiles) of all (sequence, KV head) units form one line that is cut into equal pieces, one per CTA
// (persistent), and a CTA deals its steps to its warps.  On the line a unit has its steps and, behind them, a fixed number that stands
// for its beginning (queries) and end (the warps meet); without it the CTAs with many short units came last.  A unit that lies in
// one CTA is finished there; a unit cut between CTAs leaves one partial result (maximum, sum, O) per CTA, and the CTA that arrives
// last adds them in the order of the CTAs, so results do not depend on the order of arrival.  One launch, lengths read on the device.
//
// Measured: one sequence of 131072 rows, 8 KV heads x 128 in groups of 32: 44 us, 3.8 TB/s of codes and params; 48 ragged sequences
// of up to 16384 rows, 4 KV heads: 54 us, 3.5 TB/s; one of 777 rows 9.3 us.  Issue slots are half full (310 instructions per 16
// rows, two warps per scheduler, ALU pipe 43 %, matrix pipe 29 %); four row tiles a step, twelve warps, two or four stages and
// products in other orders changed nothing, leaving the loads out neither.  (The figures beside the rules below were taken, either
// side, before the mids' weights had their second piece, which takes 1 to 2 us of these.)
constexpr int KV4_EXTRA = 32;           // a unit's fixed cost in steps (48 ragged sequences of up to 16384 rows: none 74 us, 8 69, 20 55, 32 52)
constexpr float KV4_LOG2E = 1.4426950408889634f;
constexpr float KV4_SLACK = 6.0f;       // weights stay below 2^6 ...
constexpr float KV4_BOOST = 64.f;       // ... and meet the scale, at most 4 r, 2^6 higher: p' below 2^14, normal fp16 down to 2^-20 of the largest

// 2^x to two units in the last place (results below the normal range become zero)
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t a) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
  return d;
}
template <int D, int NG, int NB, int W>
struct Kv4Tile {
  static constexpr int WARPS = W;
  // row tiles of a step: with one, the dependent chain of a step leaves the issue slots half empty at two warps per
  // scheduler (more warps would need the registers that the accumulators hold)
  static constexpr int RT = NB == 1 ? 2 : 1, ROWS = 16 * RT;
  static constexpr int NQ = 8 * NB;
  static constexpr int STAGES = 3;
  // one step in shared memory; the rows of V are 16 bytes apart so that a fragment's four rows lie in distinct banks
  static constexpr int KC = 0, VC = KC + ROWS * (D / 2), VSTRIDE = D / 2 + 16, KP = VC + ROWS * VSTRIDE, VP = KP + ROWS * NG * 4;
  static constexpr int STAGE_BYTES = VP + ROWS * NG * 4;
  static constexpr int RING_BYTES = WARPS * STAGES * STAGE_BYTES;
  static constexpr int OSTRIDE = D + 4;            // floats between the queries of a warp's partial O
  static constexpr int JOIN_BYTES = KV4_MAX_CTAS * NQ * 4;         // a factor per part and query, in the same place
  static constexpr int O_BYTES = WARPS * NQ * OSTRIDE * 4 > JOIN_BYTES ? WARPS * NQ * OSTRIDE * 4 : JOIN_BYTES;
  static constexpr int SMEM = RING_BYTES + O_BYTES;
};

// A position on the line of steps: sequence b, head unit h, step s of n (from n to n + extra: the unit's fixed cost, no step).
// Units are ordered by sequence, then head.
struct Kv4Unit { int b, h, n; };
struct Kv4Line {
  const int* pre;        // [n_seq + 1] steps of one head before each sequence (shared memory)
  const unsigned short* held;  // [n_seq + 1] sequences with rows before each sequence
  int n_seq, heads;      // head units per sequence
  int extra;
  __device__ __forceinline__ long start(int b) const { return (pre[b] + (long)extra * held[b]) * heads; }
  __device__ __forceinline__ Kv4Unit find(long x, int& s) const {
    int lo = 0, hi = n_seq;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (start(mid) <= x) lo = mid; else hi = mid;
    }
    Kv4Unit u;
    u.b = lo;
    u.n = pre[lo + 1] - pre[lo];
    const long r = x - start(lo);
    u.h = (int)(r / (u.n + extra));
    s = (int)(r - (long)u.h * (u.n + extra));
    return u;
  }
  __device__ __forceinline__ Kv4Unit next(Kv4Unit u) const {     // only called while steps are left
    if (++u.h < heads) return u;
    u.h = 0;
    do { ++u.b; u.n = pre[u.b + 1] - pre[u.b]; } while (u.n == 0);
    return u;
  }
};

// The steps of one warp within its CTA's piece of the line: every WARPS-th step of each unit's stretch.
struct Kv4Walk {
  Kv4Unit u;
  int s, end;            // the warp's step, and the end of the stretch in this unit
  long left;             // what is left of the piece behind this unit
  __device__ __forceinline__ void open(const Kv4Line& line, int first, long room, int warp) {      // this unit, from `first` on
    const int n = u.n + line.extra - first;
    end = min(u.n, first + (int)min((long)n, room));
    left = room - min((long)n, room);
    s = first + warp;
  }
  __device__ __forceinline__ bool more(const Kv4Line& line, int warp) {      // settles on the next step; false: none left
    while (s >= end) {
      if (left == 0) return false;
      u = line.next(u);
      open(line, 0, left, warp);
    }
    return true;
  }
};

template <int D, int NG, int NB, int W>
__global__ void __launch_bounds__(W * 32, 8 / W)
kv4_attn_kernel(Kv4Dev c, const bf16* __restrict__ Q, int64_t ldq, int H, int qblocks, bf16* __restrict__ O, int64_t ldo,
                float* __restrict__ part, int* __restrict__ arrived) {
  using T = Kv4Tile<D, NG, NB, W>;
  constexpr int WARPS = T::WARPS, NQ = T::NQ, NT = D / 32, RT = T::RT, ROWS = T::ROWS;
  constexpr int GT = NT / NG;                      // 32-dim blocks of a group
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ int pre[SPTS_KV4_MAX_SEQ + 1];
  __shared__ unsigned short held[SPTS_KV4_MAX_SEQ + 1];
  __shared__ long warp_sums[WARPS];
  __shared__ float sm_m[WARPS][NQ], sm_l[WARPS][NQ], sm_f[WARPS][NQ], sm_L[NQ], sm_M[NQ];
  __shared__ int last_flag;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, cc = lane & 3;
  const int G = H / c.Hkv, heads = c.Hkv * qblocks, per_block = NB == 1 ? G : 16;

  // ---- the line of steps
  auto steps_of = [&](int b) { return b < c.n_seq ? (max(0, min(__ldg(&c.len[b]), c.capacity)) + ROWS - 1) / ROWS : 0; };
  {
    long carry = 0;                                // steps, and in the bits from 40 on sequences with rows
    if (tid == 0) { pre[0] = 0; held[0] = 0; }
    for (int b0 = 0; b0 < c.n_seq; b0 += WARPS * 32) {
      long v = steps_of(b0 + tid);
      if (v > 0) v |= 1L << 40;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const long up = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += up;
      }
      if (lane == 31) warp_sums[warp] = v;
      __syncthreads();
      long before = carry, all = carry;
      for (int w = 0; w < WARPS; ++w) { if (w < warp) before += warp_sums[w]; all += warp_sums[w]; }
      if (b0 + tid < c.n_seq) {
        pre[b0 + tid + 1] = (int)((before + v) & 0xFFFFFFFFFFL);
        held[b0 + tid + 1] = (unsigned short)((before + v) >> 40);
      }
      carry = all;
      __syncthreads();
    }
  }
  Kv4Line line{pre, held, c.n_seq, heads, KV4_EXTRA};
  long total = line.start(c.n_seq);
  long ctas = max(1L, min((long)gridDim.x, total / (KV4_EXTRA + 1)));
  // Few units, as long on average as those of the first sequence (equally long ones above all): whole numbers of CTAs to each where
  // that leaves at most a sixteenth of them idle.  (A CTA with the end of one unit and the beginning of the next meets, leaves and
  // joins twice: 45.8 instead of 42.4 us for 8 x 131072 rows.)  Units of other lengths that pass the test are cut all the same,
  // evenly and without the fixed cost.
  {
    const long units = (long)c.n_seq * heads, most = min((long)gridDim.x, units * ((pre[1] + WARPS - 1) / WARPS)), whole = most / units * units;
    if (pre[1] > 0 && pre[1] * (long)c.n_seq == pre[c.n_seq] && 16 * whole >= 15 * most) {
      line.extra = 0;
      total = line.start(c.n_seq);
      ctas = whole;
    }
  }
  // sequences without rows
  for (int b = blockIdx.x; b < c.n_seq; b += gridDim.x)
    if (pre[b + 1] == pre[b])
      for (int i = tid; i < H * D; i += WARPS * 32) O[(size_t)b * ldo + i] = __float2bfloat16_rn(0.f);
  if (total == 0 || blockIdx.x >= ctas) return;
  const long x0 = total * blockIdx.x / ctas, x1 = total * (blockIdx.x + 1) / ctas;

  unsigned char* ring = smem + warp * (T::STAGES * T::STAGE_BYTES);
  float* sm_o = reinterpret_cast<float*>(smem + T::RING_BYTES);
  // a lane's share of a step's copies: D / 64 pieces of 16 bytes of either code block, one of the params (K's, then V's)
  const uint32_t ring_s = (uint32_t)__cvta_generic_to_shared(ring);
  const uint32_t dst_k = ring_s + T::KC + 16 * lane, dst_v = ring_s + T::VC + (lane / (D / 32)) * T::VSTRIDE + (lane % (D / 32)) * 16;
  const bool lane_p = lane < 4 * NG * RT;
  const uint32_t dst_p = ring_s + T::KP + 16 * lane;
  const char* src_k = nullptr; const char* src_v = nullptr; const char* src_kp = nullptr; const char* src_vp = nullptr;
  auto point = [&](const Kv4Walk& w) {             // at the lane's share of the walk's step
    const size_t row = ((size_t)w.u.b * c.Hkv + w.u.h / qblocks) * c.capacity + ROWS * (size_t)w.s;
    src_k = c.k_codes + row * (D / 2) + 16 * lane;
    src_v = c.v_codes + row * (D / 2) + 16 * lane;
    src_kp = (const char*)(c.k_params + row * NG) + 16 * lane;
    src_vp = (const char*)(c.v_params + row * NG) + 16 * lane;
  };
  uint32_t fetch_at = 0;                           // byte offset of the stage to fill
  auto fetch = [&]() {
#pragma unroll
    for (int i = 0; i < D / 64 * RT; ++i) {
      cp_async16(dst_k + fetch_at + 512 * i, src_k + 512 * i);
      cp_async16(dst_v + fetch_at + 512 / (D / 2) * i * T::VSTRIDE, src_v + 512 * i);
    }
    if (lane_p) {
      cp_async16(dst_p + fetch_at, src_kp);
      cp_async16(dst_p + fetch_at + (T::VP - T::KP), src_vp);
    }
  };

  Kv4Walk ahead, now;
  int first_s;                                     // the stretch of the current unit begins here
  {
    now.u = line.find(x0, first_s);
    now.open(line, first_s, x1 - x0, warp);
    if (first_s >= now.u.n) {                      // the piece begins behind a unit's last step
      if (now.left == 0) return;
      now.u = line.next(now.u);
      now.open(line, 0, now.left, warp);
      first_s = 0;
    }
    ahead = now;
  }
  bool fetching = ahead.more(line, warp);
  if (fetching) point(ahead);
  auto fetch_next = [&]() {
    if (fetching) {
      fetch();
      ahead.s += WARPS;
      if (ahead.s < ahead.end) {
        src_k += WARPS * ROWS * (D / 2);
        src_v += WARPS * ROWS * (D / 2);
        src_kp += WARPS * ROWS * NG * 4;
        src_vp += WARPS * ROWS * NG * 4;
      } else {
        fetching = ahead.more(line, warp);
        if (fetching) point(ahead);
      }
    }
    cp_async_commit();
    fetch_at = fetch_at + T::STAGE_BYTES == T::STAGES * T::STAGE_BYTES ? 0 : fetch_at + T::STAGE_BYTES;
  };
#pragma unroll
  for (int i = 0; i < T::STAGES - 1; ++i) fetch_next();

  // scores stay as they come out of the products; sl brings them to powers of two inside the exponential's argument
  const float sl = rsqrtf((float)D) * KV4_LOG2E, slack = KV4_SLACK / sl;
  uint32_t use_at = 0;
  while (true) {
    // ---- one unit's stretch [first_s, now.end)
    const Kv4Unit u = now.u;
    const int b = u.b, kvh = u.h / qblocks, hb = kvh * G + (u.h % qblocks) * per_block;
    const int nq = min(per_block, G - (u.h % qblocks) * per_block);
    const int len = max(0, min(__ldg(&c.len[b]), c.capacity));
    const int end = now.end;
    // Q as B fragments, and (-8 sum q, sum q) of every group in two bf16 pieces, all times the query's power of two; slq
    // brings a score in those units to a power of two's exponent
    uint32_t qf[NB][NT][4], qm[NB][2];
    float slq[NB][2];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const int qi = 8 * nb + g;
      float x[NT][8], top = 0.f;
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[t][j] = 0.f;
        if (qi < nq) load8(Q + (size_t)b * ldq + (size_t)(hb + qi) * D + 32 * t + 8 * cc, x[t]);
#pragma unroll
        for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(x[t][j]));
      }
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const float qs = scale_to_2_13(top);
      float mine = 0.f, sum = 0.f;
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float f = (j & 1) ? qs * ODD : qs;
          qf[nb][t][j] = pack2_f16(x[t][j] * f, x[t][j + 4] * f);
        }
        float s8 = ((x[t][0] + x[t][1]) + (x[t][2] + x[t][3])) + ((x[t][4] + x[t][5]) + (x[t][6] + x[t][7]));
        s8 += __shfl_xor_sync(0xffffffffu, s8, 1);
        s8 += __shfl_xor_sync(0xffffffffu, s8, 2);
        sum = t % GT == 0 ? s8 : sum + s8;
        if (cc == t / GT) mine = sum;
      }
      const float u = qs * CODE_UNIT, a = -8.f * mine * u, ah = round_bf16(a), sm = mine * u, mh = round_bf16(sm);
      qm[nb][0] = pack2(ah, mh);
      qm[nb][1] = pack2(a - ah, sm - mh);
      const float mysl = sl / u;
#pragma unroll
      for (int i = 0; i < 2; ++i) slq[nb][i] = __shfl_sync(0xffffffffu, mysl, 4 * (2 * cc + i));
    }
    float o[NB][NT][2][4], oz[NB][NG][4], om[NB][4], thr[NB][2], msl[NB][2], l[NB][2];    // thr: where the reference moves
    float r_inv = KV4_BOOST, r_lim = 0.f;         // 2^6 / r, and the scale where r moves
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        om[nb][i] = 0.f;
#pragma unroll
        for (int t = 0; t < NT; ++t) { o[nb][t][0][i] = 0.f; o[nb][t][1][i] = 0.f; }
#pragma unroll
        for (int t = 0; t < NG; ++t) oz[nb][t][i] = 0.f;
      }
      thr[nb][0] = thr[nb][1] = msl[nb][0] = msl[nb][1] = -INFINITY;
      l[nb][0] = l[nb][1] = 0.f;
    }
    for (; now.s < end; now.s += WARPS) {
      fetch_next();
      cp_async_wait<T::STAGES - 1>();
      __syncwarp();
      unsigned char* st = ring + use_at;
      use_at = use_at + T::STAGE_BYTES == T::STAGES * T::STAGE_BYTES ? 0 : use_at + T::STAGE_BYTES;
      const int valid = len - ROWS * now.s;        // rows of this step that are held
      if (valid < ROWS) {
        // what lies behind the last row may be anything: its params become zero (its codes are finite whatever they are)
        for (int i = valid * NG + lane; i < ROWS * NG; i += 32) {
          reinterpret_cast<uint32_t*>(st + T::KP)[i] = 0u;
          reinterpret_cast<uint32_t*>(st + T::VP)[i] = 0u;
        }
        __syncwarp();
      }
      // ---- S
      float sc[RT][NB][4];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        const int r0 = 16 * rt + g, r1 = r0 + 8;
        uint32_t kw0[NT], kw1[NT], kp0[NG], kp1[NG];
        if (NT == 4) {
          *reinterpret_cast<uint4*>(kw0) = *reinterpret_cast<const uint4*>(st + T::KC + r0 * (D / 2) + cc * 16);
          *reinterpret_cast<uint4*>(kw1) = *reinterpret_cast<const uint4*>(st + T::KC + r1 * (D / 2) + cc * 16);
        } else {
          *reinterpret_cast<uint2*>(kw0) = *reinterpret_cast<const uint2*>(st + T::KC + r0 * (D / 2) + cc * 8);
          *reinterpret_cast<uint2*>(kw1) = *reinterpret_cast<const uint2*>(st + T::KC + r1 * (D / 2) + cc * 8);
        }
        load_words<NG>(st + T::KP + r0 * NG * 4, kp0);
        load_words<NG>(st + T::KP + r1 * NG * 4, kp1);
        uint32_t pw0 = 0u, pw1 = 0u;
        if (cc < NG) {
          pw0 = *reinterpret_cast<const uint32_t*>(st + T::KP + (r0 * NG + cc) * 4);
          pw1 = *reinterpret_cast<const uint32_t*>(st + T::KP + (r1 * NG + cc) * 4);
        }
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
          for (int i = 0; i < 4; ++i) sc[rt][nb][i] = 0.f;
          mma16816(sc[rt][nb], pw0, pw1, pw0, pw1, qm[nb][0], qm[nb][1]);
        }
#pragma unroll
        for (int gr = 0; gr < NG; ++gr) {
          float acc[NB][4];
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[nb][i] = 0.f;
#pragma unroll
          for (int tt = 0; tt < GT; ++tt) {
            const int t = gr * GT + tt;
            const uint32_t a0 = code_pair<0>(kw0[t]), a1 = code_pair<0>(kw1[t]), a2 = code_pair<1>(kw0[t]), a3 = code_pair<1>(kw1[t]);
            const uint32_t b0 = code_pair<2>(kw0[t]), b1 = code_pair<2>(kw1[t]), b2 = code_pair<3>(kw0[t]), b3 = code_pair<3>(kw1[t]);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
              mma_f16(acc[nb], a0, a1, a2, a3, qf[nb][t][0], qf[nb][t][1]);
              mma_f16(acc[nb], b0, b1, b2, b3, qf[nb][t][2], qf[nb][t][3]);
            }
          }
          const float s0 = lo_bf16(kp0[gr]), s1 = lo_bf16(kp1[gr]);
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            float (&x)[4] = sc[rt][nb];
            x[0] = fmaf(s0, acc[nb][0], x[0]); x[1] = fmaf(s0, acc[nb][1], x[1]);
            x[2] = fmaf(s1, acc[nb][2], x[2]); x[3] = fmaf(s1, acc[nb][3], x[3]);
          }
        }
      }
      // ---- weights (in powers of two)
      if (valid < ROWS) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            if (16 * rt + g >= valid) { sc[rt][nb][0] = -INFINITY; sc[rt][nb][1] = -INFINITY; }
            if (16 * rt + g + 8 >= valid) { sc[rt][nb][2] = -INFINITY; sc[rt][nb][3] = -INFINITY; }
          }
      }
      float top_s = 0.f, top[NB][2];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) top[nb][0] = top[nb][1] = -INFINITY;
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int i = 0; i < 2; ++i) top[nb][i] = fmaxf(top[nb][i], fmaxf(sc[rt][nb][i], sc[rt][nb][2 + i]));
      // the largest scale of V, by its size (a group may hold its values with a negative one), among the params words, ROWS NG / 32
      // to a lane
#pragma unroll
      for (int i = 0; i < (ROWS * NG + 31) / 32; ++i)
        if (ROWS * NG % 32 == 0 || lane < ROWS * NG) top_s = fmaxf(top_s, fabsf(lo_bf16(reinterpret_cast<const uint32_t*>(st + T::VP)[32 * i + lane])));
      bool over = top_s > r_lim;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) over = over || top[nb][0] > thr[nb][0] || top[nb][1] > thr[nb][1];
      if (__any_sync(0xffffffffu, over)) {
        top_s = warp_max(top_s);
        float fr = 1.f;
        if (top_s > r_lim) {
          const float inv = scale_to_2_13(top_s) * (KV4_BOOST / 8192.f);       // 2^6 / r with r in (top_s / 2, top_s]
          fr = r_lim == 0.f ? 0.f : inv / r_inv;
          r_inv = inv;
          r_lim = 2.f * top_s;
        }
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            float x = top[nb][i];
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
            x *= slq[nb][i];
            const float mn = fmaxf(msl[nb][i], x);
            const float f = msl[nb][i] == mn ? 1.f : exp2f(msl[nb][i] - mn), fo = f * fr;
            msl[nb][i] = mn;
            thr[nb][i] = (mn + KV4_SLACK) / slq[nb][i];
            l[nb][i] *= f;
            om[nb][i] *= f; om[nb][2 + i] *= f;
#pragma unroll
            for (int t = 0; t < NG; ++t) { oz[nb][t][i] *= fo; oz[nb][t][2 + i] *= fo; }
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
              for (int j = 0; j < 2; ++j) { o[nb][t][j][i] *= fo; o[nb][t][j][2 + i] *= fo; }
          }
      }
      // ---- O
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        uint32_t vp0[NG], vp1[NG];
        load_words<NG>(st + T::VP + (16 * rt + g) * NG * 4, vp0);
        load_words<NG>(st + T::VP + (16 * rt + g + 8) * NG * 4, vp1);
        // mids: A row r holds group r % NG
        const uint32_t* vm = reinterpret_cast<const uint32_t*>(st + T::VP) + 16 * rt * NG + (g % NG);
        const uint32_t m0 = __byte_perm(vm[2 * cc * NG], vm[(2 * cc + 1) * NG], 0x7632);
        const uint32_t m2 = __byte_perm(vm[(2 * cc + 8) * NG], vm[(2 * cc + 9) * NG], 0x7632);
        uint32_t pb[NB][NG][2];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          float p[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) p[i] = exp2_fast(fmaf(sc[rt][nb][i], slq[nb][i & 1], -msl[nb][i & 1]));
          l[nb][0] += p[0] + p[2];
          l[nb][1] += p[1] + p[3];
          {
            const uint32_t h0 = pack2(p[0], p[1]), h1 = pack2(p[2], p[3]);
            mma16816(om[nb], m0, 0u, m2, 0u, transpose8x8(h0), transpose8x8(h1));
            mma16816(om[nb], m0, 0u, m2, 0u, transpose8x8(pack2(p[0] - lo_bf16(h0), p[1] - hi_bf16(h0))),
                     transpose8x8(pack2(p[2] - lo_bf16(h1), p[3] - hi_bf16(h1))));
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) p[i] *= r_inv;
#pragma unroll
          for (int gr = 0; gr < NG; ++gr) {
            const float s0 = lo_bf16(vp0[gr]), s1 = lo_bf16(vp1[gr]);
            pb[nb][gr][0] = transpose8x8(pack2_f16(p[0] * s0, p[1] * s0));
            pb[nb][gr][1] = transpose8x8(pack2_f16(p[2] * s1, p[3] * s1));
          }
        }
        uint32_t vw[4][NT / 2];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const unsigned char* r = st + T::VC + (16 * rt + 8 * (i >> 1) + 2 * cc + (i & 1)) * T::VSTRIDE + g * (D / 16);
          if (NT == 4) *reinterpret_cast<uint2*>(vw[i]) = *reinterpret_cast<const uint2*>(r);
          else vw[i][0] = *reinterpret_cast<const uint32_t*>(r);
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const uint32_t sel = (t & 1) ? 0x7632u : 0x5410u;
          const uint32_t x01 = __byte_perm(vw[0][t / 2], vw[1][t / 2], sel), x23 = __byte_perm(vw[2][t / 2], vw[3][t / 2], sel);
          const uint32_t a0 = code_pair<0>(x01), a1 = code_pair<1>(x01), a2 = code_pair<0>(x23), a3 = code_pair<1>(x23);
          const uint32_t b0 = code_pair<2>(x01), b1 = code_pair<3>(x01), b2 = code_pair<2>(x23), b3 = code_pair<3>(x23);
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            mma_f16(o[nb][t][0], a0, a1, a2, a3, pb[nb][t / GT][0], pb[nb][t / GT][1]);
            mma_f16(o[nb][t][1], b0, b1, b2, b3, pb[nb][t / GT][0], pb[nb][t / GT][1]);
          }
        }
        // -8 in the units of the even (A rows 0..7) and the odd codes (rows 8..15)
#pragma unroll
        for (int gr = 0; gr < NG; ++gr)
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
            mma_f16(oz[nb][gr], 0x80088008u, 0x80808080u, 0x80088008u, 0x80808080u, pb[nb][gr][0], pb[nb][gr][1]);
      }
      __syncwarp();                                // the stage may be filled again
    }
    // ---- the warps' results meet
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float s = l[nb][i];
        s += __shfl_xor_sync(0xffffffffu, s, 4);
        s += __shfl_xor_sync(0xffffffffu, s, 8);
        s += __shfl_xor_sync(0xffffffffu, s, 16);
        if (g == 0) { sm_m[warp][8 * nb + 2 * cc + i] = msl[nb][i]; sm_l[warp][8 * nb + 2 * cc + i] = s; }
      }
      const float r = 1.f / r_inv;                 // (r_inv holds the boost)
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        // lane (group, cc) of the mids' tile holds queries 2 cc, 2 cc + 1
        const float z0 = __shfl_sync(0xffffffffu, om[nb][0], (t / GT) * 4 + cc), z1 = __shfl_sync(0xffffffffu, om[nb][1], (t / GT) * 4 + cc);
        const float* oz_t = oz[nb][t / GT];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float* ov = o[nb][t][j];
          float* dst = sm_o + (size_t)(warp * NQ + 8 * nb + 2 * cc) * T::OSTRIDE + 32 * t + 4 * g + 2 * j;
          *reinterpret_cast<float2*>(dst) = make_float2(fmaf((ov[0] + oz_t[0]) * CODE_UNIT_INV, r, z0), fmaf((ov[2] + oz_t[2]) * (CODE_UNIT_INV * ODD), r, z0));
          *reinterpret_cast<float2*>(dst + T::OSTRIDE) = make_float2(fmaf((ov[1] + oz_t[1]) * CODE_UNIT_INV, r, z1), fmaf((ov[3] + oz_t[3]) * (CODE_UNIT_INV * ODD), r, z1));
        }
      }
    }
    __syncthreads();
    if (tid < NQ) {
      float M = -INFINITY, L = 0.f;
      bool nan = false;
#pragma unroll
      for (int w = 0; w < WARPS; ++w) M = fmaxf(M, sm_m[w][tid]);
#pragma unroll
      for (int w = 0; w < WARPS; ++w) {
        // a warp without rows has sum 0 and O = 0; one whose scores were NaN has sum NaN
        const float f = sm_m[w][tid] == -INFINITY ? 0.f : exp2f(sm_m[w][tid] - M);
        nan = nan || sm_l[w][tid] != sm_l[w][tid];
        sm_f[w][tid] = f;
        L += sm_l[w][tid] * f;
      }
      sm_M[tid] = M;
      sm_L[tid] = nan ? NAN : L;
    }
    __syncthreads();
    const bool whole = first_s == 0 && end == u.n;
    const int slot = 2 * (int)blockIdx.x + (first_s == 0 ? 1 : 0);
    for (int i = tid; i < nq * D; i += WARPS * 32) {
      const int q = i / D, dim = i - q * D;
      float a = 0.f;
#pragma unroll
      for (int w = 0; w < WARPS; ++w) a = fmaf(sm_o[(size_t)(w * NQ + q) * T::OSTRIDE + dim], sm_f[w][q], a);
      if (whole) O[(size_t)b * ldo + (size_t)(hb + q) * D + dim] = __float2bfloat16_rn(a / sm_L[q]);
      else {
        float* pp = part + ((size_t)slot * 16 + q) * (D + 2);
        if (dim == 0) { pp[0] = sm_M[q]; pp[1] = sm_L[q]; }
        pp[2 + dim] = a;
      }
    }
    if (!whole) {
      // CTAs of this unit: the one with its first step to the one with its last
      const long ux = line.start(b) + (long)u.h * (u.n + line.extra);
      const int c0 = (int)(((ux + 1) * ctas - 1) / total), c1 = (int)(((ux + u.n) * ctas - 1) / total);
      __threadfence();
      __syncthreads();
      if (tid == 0) last_flag = atomicAdd(&arrived[c0], 1) == c1 - c0;
      __syncthreads();
      if (last_flag) {
        __threadfence();
        // the parts' factors first, one lane per part; then every output element is a sum of independent loads (a loop that
        // loads, compares and adds part by part took 20 us here, a third of the kernel)
        const int parts = c1 - c0 + 1;
        float* fac = sm_o;
        auto part_of = [&](int x, int q) { return part + ((size_t)(2 * (c0 + x) + (x == 0 ? 1 : 0)) * 16 + q) * (D + 2); };
        for (int q = warp; q < nq; q += WARPS) {
          float M = -INFINITY, L = 0.f;
#pragma unroll 1
          for (int x = lane; x < parts; x += 32) M = fmaxf(M, __ldcg(part_of(x, q)));
          M = warp_max(M);
#pragma unroll 1
          for (int x = lane; x < parts; x += 32) {
            const float mx = __ldcg(part_of(x, q)), f = mx == -INFINITY ? 0.f : exp2_fast(mx - M);
            fac[x * nq + q] = f;
            L = fmaf(__ldcg(part_of(x, q) + 1), f, L);
          }
          L = warp_sum(L);
          if (lane == 0) sm_L[q] = L;
        }
        __syncthreads();
        for (int i = tid; i < nq * D / 2; i += WARPS * 32) {
          const int q = i / (D / 2), dim = 2 * (i - q * (D / 2));
          const float* src = part_of(0, q) + 2 + dim;
          const float2 v0 = __ldcg(reinterpret_cast<const float2*>(src));
          float a0 = v0.x * fac[q], a1 = v0.y * fac[q];
          src = part_of(1, q) + 2 + dim;
          constexpr int U = 6;                     // loads in flight; the parts behind c0 are 2 * 16 * (D + 2) floats apart
#pragma unroll 1
          for (int x0 = 1; x0 < parts; x0 += U) {
            float2 v[U];
#pragma unroll
            for (int k = 0; k < U; ++k)
              v[k] = x0 + k < parts ? __ldcg(reinterpret_cast<const float2*>(src + (size_t)(x0 - 1 + k) * 32 * (D + 2))) : make_float2(0.f, 0.f);
#pragma unroll
            for (int k = 0; k < U; ++k)
              if (x0 + k < parts) {
                const float f = fac[(x0 + k) * nq + q];
                a0 = fmaf(v[k].x, f, a0); a1 = fmaf(v[k].y, f, a1);
              }
          }
          *reinterpret_cast<uint32_t*>(O + (size_t)b * ldo + (size_t)(hb + q) * D + dim) = pack2(a0 / sm_L[q], a1 / sm_L[q]);
        }
        if (tid == 0) arrived[c0] = 0;             // for the next call
      }
    }
    // ---- the next unit of the piece
    if (now.left == 0) break;
    now.u = line.next(now.u);
    now.open(line, 0, now.left, warp);
    first_s = 0;
    __syncthreads();                               // sm_m, sm_l and sm_o are free again
  }
  cp_async_wait<0>();
}

Kv4Dev kv4_dev(const spts_ctx* ctx, const spts_kv4_cache* c) {
  return Kv4Dev{(char*)c->k_codes, (char*)c->v_codes, (uint32_t*)c->k_params, (uint32_t*)c->v_params, c->pos, c->len,
                c->n_seq, c->capacity, c->group, ctx->desc.n_kv_heads};
}

template <typename T, int D>
spts_status append_t(spts_ctx* ctx, const spts_kv4_cache* cache, const void* K, int64_t ldk, const void* V, int64_t ldv,
                     const int32_t* pos, const int32_t* row_start, const int32_t* at, int n_rows, void* K_read, void* V_read) {
  const Kv4Dev c = kv4_dev(ctx, cache);
  if (n_rows > 0) {
    // many rows: four passes to a warp; few: one, so that they spread over the SMs
    const int passes = ceil_div(c.Hkv, 256 / D);
    const int per = (long)n_rows * passes >= 16L * 8 * ctx->sm_count ? 4 : 1, parts = 2 * ceil_div(passes, per);
    int blocks = ceil_div(n_rows, 8);
    if (blocks > ceil_div(16 * ctx->sm_count, parts)) blocks = ceil_div(16 * ctx->sm_count, parts);
    auto kernel = c.group == 32 ? kv4_append_kernel<T, D, 4> : c.group == 64 || D == 64 ? kv4_append_kernel<T, D, 8> : kv4_append_kernel<T, D, D / 8>;
    kernel<<<dim3(blocks, parts), 256, 0, ctx->stream>>>(c, (const T*)K, ldk, (const T*)V, ldv, pos, row_start, at, n_rows, per,
                                                         (T*)K_read, (T*)V_read, ctx->ws.status);
    SPTS_CUDA_OK(ctx);
  }
  kv4_len_kernel<<<ceil_div(c.n_seq, 256), 256, 0, ctx->stream>>>(c.len, at, row_start, c.n_seq, c.capacity, n_rows, ctx->ws.status);
  SPTS_CUDA_OK(ctx);
  return SPTS_OK;
}

template <typename T, int D>
spts_status attn_plain_t(spts_ctx* ctx, const spts_kv4_cache* cache, const void* Q, int64_t ldq, void* O, int64_t ldo) {
  const Kv4Dev c = kv4_dev(ctx, cache);
  const int H = ctx->desc.n_q_heads;
  // CTAs per head: as many as still run at once (one of 512 threads and 95 registers on an SM, two at 64 dims)
  int split = PLAIN_SPLIT;
  while (split > 1 && (long)H * c.n_seq * split > 2L * ctx->sm_count) split /= 2;
  cudaLaunchConfig_t config{};
  config.gridDim = dim3(split, H, c.n_seq);
  config.blockDim = dim3(PLAIN_WARPS * 32);
  config.stream = ctx->stream;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = split;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  config.attrs = &attr;
  config.numAttrs = 1;
  if (cudaLaunchKernelEx(&config, kv4_attn_plain_kernel<T, D>, c, (const T*)Q, ldq, H, (T*)O, ldo) != cudaSuccess) return SPTS_ERR_CUDA;
  SPTS_CUDA_OK(ctx);
  return SPTS_OK;
}

template <int D, int NG, int NB, int W>
spts_status attn_w(spts_ctx* ctx, const spts_kv4_cache* cache, const void* Q, int64_t ldq, void* O, int64_t ldo) {
  using T = Kv4Tile<D, NG, NB, W>;
  const Kv4Dev c = kv4_dev(ctx, cache);
  const int H = ctx->desc.n_q_heads, G = H / c.Hkv;
  const int grid = 8 / W * ctx->sm_count < KV4_MAX_CTAS ? 8 / W * ctx->sm_count : KV4_MAX_CTAS;
  if (cudaFuncSetAttribute(kv4_attn_kernel<D, NG, NB, W>, cudaFuncAttributeMaxDynamicSharedMemorySize, T::SMEM) != cudaSuccess)
    return SPTS_ERR_CUDA;
  kv4_attn_kernel<D, NG, NB, W><<<grid, T::WARPS * 32, T::SMEM, ctx->stream>>>(c, (const bf16*)Q, ldq, H, NB == 1 ? 1 : ceil_div(G, 16),
                                                                            (bf16*)O, ldo, ctx->ws.kv4_part, ctx->ws.kv4_arrived);
  SPTS_CUDA_OK(ctx);
  return SPTS_OK;
}
// Four warps to a CTA and two CTAs to an SM where there are two units for every SM: a CTA's units follow one another, each with
// the latency of its beginning and its meeting, and then two go side by side (256 sequences of 100 rows, 8 KV heads: 33 us instead
// of 51; 64 of 2048 rows: 45 instead of 50).  Few long units are cut into half as many pieces by eight warps (one sequence of
// 131072 rows: 42 instead of 46; 5000, 300, 12000 and 40 rows, 2 KV heads: 23 instead of 35).
template <int D, int NG, int NB>
spts_status attn_t(spts_ctx* ctx, const spts_kv4_cache* cache, const void* Q, int64_t ldq, void* O, int64_t ldo) {
  const int kv = ctx->desc.n_kv_heads, G = ctx->desc.n_q_heads / kv;
  const long units = (long)cache->n_seq * kv * (NB == 1 ? 1 : ceil_div(G, 16));
  return units >= 2 * ctx->sm_count ? attn_w<D, NG, NB, 4>(ctx, cache, Q, ldq, O, ldo) : attn_w<D, NG, NB, 8>(ctx, cache, Q, ldq, O, ldo);
}
template <int D, int NG>
spts_status attn_heads(spts_ctx* ctx, const spts_kv4_cache* cache, const void* Q, int64_t ldq, void* O, int64_t ldo) {
  return ctx->desc.n_q_heads / ctx->desc.n_kv_heads <= 8 ? attn_t<D, NG, 1>(ctx, cache, Q, ldq, O, ldo)
                                                         : attn_t<D, NG, 2>(ctx, cache, Q, ldq, O, ldo);
}

}  // namespace

spts_status launch_kv4_append(spts_ctx* ctx, const spts_kv4_cache* cache, const void* K, int64_t ldk, const void* V,
                              int64_t ldv, const int32_t* pos, const int32_t* row_start, const int32_t* at, int n_rows,
                              void* K_read, void* V_read) {
  const bool wide = ctx->desc.head_dim == 128;
  if (ctx->desc.dtype == SPTS_BF16)
    return wide ? append_t<bf16, 128>(ctx, cache, K, ldk, V, ldv, pos, row_start, at, n_rows, K_read, V_read)
                : append_t<bf16, 64>(ctx, cache, K, ldk, V, ldv, pos, row_start, at, n_rows, K_read, V_read);
  return wide ? append_t<float, 128>(ctx, cache, K, ldk, V, ldv, pos, row_start, at, n_rows, K_read, V_read)
              : append_t<float, 64>(ctx, cache, K, ldk, V, ldv, pos, row_start, at, n_rows, K_read, V_read);
}

spts_status launch_kv4_attention(spts_ctx* ctx, const spts_kv4_cache* cache, const void* Q, int64_t ldq, void* O, int64_t ldo) {
  const bool wide = ctx->desc.head_dim == 128;
  if (!plain4(ctx)) {
    const int ng = ctx->desc.head_dim / cache->group;
    if (!wide) return ng == 2 ? attn_heads<64, 2>(ctx, cache, Q, ldq, O, ldo) : attn_heads<64, 1>(ctx, cache, Q, ldq, O, ldo);
    if (ng == 4) return attn_heads<128, 4>(ctx, cache, Q, ldq, O, ldo);
    return ng == 2 ? attn_heads<128, 2>(ctx, cache, Q, ldq, O, ldo) : attn_heads<128, 1>(ctx, cache, Q, ldq, O, ldo);
  }
  if (ctx->desc.dtype == SPTS_BF16)
    return wide ? attn_plain_t<bf16, 128>(ctx, cache, Q, ldq, O, ldo) : attn_plain_t<bf16, 64>(ctx, cache, Q, ldq, O, ldo);
  return wide ? attn_plain_t<float, 128>(ctx, cache, Q, ldq, O, ldo) : attn_plain_t<float, 64>(ctx, cache, Q, ldq, O, ldo);
}

}  // namespace spts
