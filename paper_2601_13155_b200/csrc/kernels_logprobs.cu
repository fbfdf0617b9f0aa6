// Log probabilities of given tokens with their ranks, the entropy and the most likely alternatives of rows of logits, in one launch
// and one read of the logits.
//
// A CTA takes a slice of a row, 4096 tokens at a time, sixteen to a thread, the next sixteen on their way.  With m the largest logit so far
// and x = (l - m) log2 e it holds A = sum 2^x and B = sum 2^x x; when m grows by g (in log2 units), A becomes A 2^-g and
// B (B - g A) 2^-g.  At the end lse = m + log A and entropy = (log2 A - B / A) ln 2: no difference of large sums.  A NaN or +inf makes A NaN.
// The target's logit is read first, so its rank is a count in the same pass.
// Alternatives: in the pass a warp notes the largest token of each stretch of 512 that it reads.  At least n_top tokens lie at or above the
// n_top-th largest of these, rounded down (and above the fourth largest of the eight warps' r-th largest threads, r = ceil(n_top / 4), which says more
// where stretches are few), so none of the best lies below; the few stretches that reach it are read once more, what lies above goes onto a
// list in shared memory, and of that the best are taken.  Where the list runs over (equal logits), the slice is gone through piece by piece.
// A row is shared by slices where rows are few; the slice that arrives last joins what the others left, in their order.
// Bound by memory where rows are many: 509 rows of 152063 take 69 us with 20 alternatives (4.5 TB/s), 54 without (5.8 TB/s); one row of 128256
// 9.6 us, a chain of latencies.  Lists kept piece by piece and threads that search their own tokens again took 157 and 100 us for the former.
#include "spts_common.cuh"

namespace spts {

namespace {

constexpr int LP_THREADS = 256, LP_WARPS = LP_THREADS / 32;
constexpr int LP_PER = 16;                     // tokens of a thread at a time, four 16-byte loads
constexpr int LP_PIECE = LP_THREADS * LP_PER;
constexpr int LP_STRETCHES = 1024;             // stretches that are told apart; in longer slices one is several pieces' 512
constexpr int LP_FEW = 96;                     // stretches that are ranked one against all
constexpr int LP_LIST = 512;                   // candidates in shared memory
constexpr uint32_t NO_TOKEN = 0x007FFFFFu;     // order of -inf: no candidate lies at or below it

struct LogprobArgs {
  const float* x; int64_t ld; int vocab;
  const int32_t* target;
  int n_top;
  float* logprob; int32_t* rank; float* entropy; float* top_logprob; int32_t* top_token;
  float* part; int* arrived;
};

// Larger value, larger number; NaN below all.
__device__ __forceinline__ uint32_t order_of(float v) {
  if (v != v) return 0u;
  const uint32_t u = __float_as_uint(v == 0.f ? 0.f : v);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t o) { return __uint_as_float((o & 0x80000000u) ? (o & 0x7FFFFFFFu) : ~o); }

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

struct Stats {
  float m, a, b;
  int rank;
};
// m starts at the lowest finite value, so that no difference from it is undefined but that of NaN and +inf
__device__ __forceinline__ Stats no_stats() { return {-3.402823466e38f, 0.f, 0.f, 0}; }
// What lies 2^-200 below the maximum adds nothing to B; x is held there, so -inf times zero does not come about.
__device__ __forceinline__ float held(float x) { return fmaxf(x, -200.f); }
__device__ __forceinline__ void raise(Stats& s, float m) {
  const float g = held((s.m - m) * LOG2E), e = ex2(g);
  s.b = fmaf(g, s.a, s.b) * e;
  s.a *= e;
  s.m = m;
}
__device__ __forceinline__ Stats join(Stats x, Stats y) {
  const float m = fmaxf(x.m, y.m);
  raise(x, m);
  raise(y, m);
  return {m, x.a + y.a, x.b + y.b, x.rank + y.rank};
}
__device__ __forceinline__ Stats warp_join(Stats s) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    Stats t;
    t.m = __shfl_xor_sync(0xffffffffu, s.m, o);
    t.a = __shfl_xor_sync(0xffffffffu, s.a, o);
    t.b = __shfl_xor_sync(0xffffffffu, s.b, o);
    t.rank = __shfl_xor_sync(0xffffffffu, s.rank, o);
    s = join(s, t);
  }
  return s;
}

struct TopShared {
  unsigned long long list[LP_LIST];            // order << 32 | ~token: the larger key comes first
  unsigned long long best[SPTS_LOGPROBS_MAX_TOP];
  unsigned long long warp_best[LP_WARPS];
  uint32_t warp_floor[LP_WARPS];               // of find_floor
  uint32_t stretch_floor;                      // (a word of its own: slower warps may still be reading the others)
  int n;                                       // candidates asked for, of which those below LP_LIST are there
  uint32_t most[LP_STRETCHES];                 // order of the largest token of a stretch
  int reach, reaching[LP_STRETCHES];           // stretches that reach the floor
};

// The list [n] becomes its k best, in order; returns how many there are.  All threads.
__device__ __forceinline__ int cut_list(TopShared& t, int n, int k) {
  unsigned long long mine[LP_LIST / LP_THREADS];
  int r[LP_LIST / LP_THREADS];
#pragma unroll
  for (int u = 0; u < LP_LIST / LP_THREADS; ++u) {
    const int i = threadIdx.x + u * LP_THREADS;
    mine[u] = i < n ? t.list[i] : 0ull;
    r[u] = LP_LIST;
    if (i < n) {
      r[u] = 0;
      for (int j = 0; j < n; ++j) r[u] += t.list[j] > mine[u];
    }
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < LP_LIST / LP_THREADS; ++u)
    if (r[u] < k) t.list[r[u]] = mine[u];
  if (threadIdx.x == 0) t.n = min(n, k);
  __syncthreads();
  return min(n, k);
}

// The least order on a list of k.
__device__ __forceinline__ uint32_t worst(const TopShared& t, int k) {
  uint32_t w = 0xFFFFFFFFu;
  for (int i = 0; i < k; ++i) w = min(w, (uint32_t)(t.list[i] >> 32));
  return w;
}

// An order at or above which at least k of the threads' largest tokens lie.  All threads.
__device__ __forceinline__ uint32_t find_floor(TopShared& t, uint32_t top, int k) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, r = (k + LP_WARPS / 2 - 1) / (LP_WARPS / 2);
  uint32_t mine = top, w = 0;
  for (int u = 0; u < r; ++u) {
    w = __reduce_max_sync(0xffffffffu, mine);
    if (lane == __ffs(__ballot_sync(0xffffffffu, mine == w)) - 1) mine = 0;
  }
  if (lane == 0) t.warp_floor[warp] = w;
  __syncthreads();
  const uint32_t f = t.warp_floor[lane & (LP_WARPS - 1)];
  int above = 0;
  for (int u = 0; u < LP_WARPS; ++u) {
    const uint32_t g = __shfl_sync(0xffffffffu, f, u);
    above += g > f || (g == f && u < (lane & (LP_WARPS - 1)));
  }
  return __shfl_sync(0xffffffffu, f, __ffs(__ballot_sync(0xffffffffu, above == LP_WARPS / 2 - 1 && lane < LP_WARPS)) - 1);
}

// A thread's tokens of order `from` and above go onto the list, those that find room; t.n counts all.
template <typename F>
__device__ __forceinline__ void append(TopShared& t, const float (&v)[LP_PER], uint32_t top, uint32_t from, F token) {
  if (top < from) return;
  const float least = value_of(from);          // (the order of numbers, NaN below them; no number lies above +inf's)
#pragma unroll
  for (int i = 0; i < LP_PER; ++i) {
    if (v[i] >= least) {
      const int at = atomicAdd(&t.n, 1);
      if (at < LP_LIST) t.list[at] = ((unsigned long long)order_of(v[i]) << 32) | (uint32_t)~token(i);
    }
  }
}

// The k best tokens of [v0, v1) where a list of those above some floor ran over (equal logits): piece by piece, all
// threads at the same one, and where more tokens of a piece are equal than the list holds, one by one.
template <typename L>
__device__ __noinline__ int scan_again(TopShared& t, int k, int64_t v0, int64_t v1, L load) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  uint32_t floor_order = NO_TOKEN;
  int listed = 0;
  __syncthreads();
  if (tid == 0) t.n = 0;
  __syncthreads();
  for (int64_t at = v0; at < v1; at += LP_PIECE) {
    float v[LP_PER];
    load(at, v);
    const auto token = [&](int i) { return (int)(at + 4 * (tid + (i / 4) * LP_THREADS) + i % 4); };
    uint32_t top = 0;
    for (int i = 0; i < LP_PER; ++i) top = max(top, order_of(v[i]));
    const auto take = [&](uint32_t from) {
      append(t, v, top, from, token);
      __syncthreads();
      const int n = t.n;
      __syncthreads();
      return n;
    };
    int n = take(floor_order + 1);
    if (n > LP_LIST) {
      if (tid == 0) t.n = listed;
      __syncthreads();
      n = take(max(floor_order + 1, find_floor(t, top, k)));
    }
    if (n > LP_LIST) {
      if (tid == 0) t.n = listed;
      const unsigned long long mine = tid < listed ? t.list[tid] : 0ull;
      unsigned long long bound = ~0ull;
      n = 0;
      for (; n < k; ++n) {
        unsigned long long b = mine < bound ? mine : 0ull;
        for (int i = 0; i < LP_PER; ++i) {
          const uint32_t o = order_of(v[i]);
          const unsigned long long key = ((unsigned long long)o << 32) | (uint32_t)~token(i);
          if (o > NO_TOKEN && key < bound && key > b) b = key;
        }
#pragma unroll
        for (int u = 16; u > 0; u >>= 1) b = max(b, __shfl_xor_sync(0xffffffffu, b, u));
        if (lane == 0) t.warp_best[warp] = b;
        __syncthreads();
        for (int w = 0; w < LP_WARPS; ++w) b = max(b, t.warp_best[w]);
        __syncthreads();
        if (b == 0ull) break;
        if (tid == 0) t.best[n] = b;
        bound = b;
      }
      __syncthreads();
      if (tid < n) t.list[tid] = t.best[tid];
      if (tid == 0) t.n = n;
      __syncthreads();
    }
    listed = n > k ? cut_list(t, n, k) : n;
    if (listed == k) floor_order = max(floor_order, worst(t, k));
  }
  return listed;
}

template <bool TOP>
__global__ void __launch_bounds__(LP_THREADS, 4) logprobs_kernel(LogprobArgs a, int slices, int per) {
  __shared__ Stats s_stats[LP_WARPS];
  __shared__ TopShared t;
  __shared__ bool last;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int row = blockIdx.x / slices, slice = blockIdx.x - row * slices;
  const float* x = a.x + (int64_t)row * a.ld;
  // token `base` (up to three before the row) lies on a 16-byte boundary, and so do all slices and pieces
  const int base = -(int)((reinterpret_cast<uintptr_t>(x) >> 2) & 3);
  const int64_t v0 = base + (int64_t)slice * per, v1 = min((int64_t)a.vocab, v0 + per);
  dep_wait();
  const int target = a.target != nullptr ? a.target[row] : -1;
  const bool scored = target >= 0 && target < a.vocab;
  const float xt = scored ? x[target] : 0.f;
  const int ties = (int)min((int64_t)target, v1);      // tokens below this one come before an equal target
  const int k = a.n_top;
  Stats s = no_stats();
  const int pieces = v1 > v0 ? (int)((v1 - v0 + LP_PIECE - 1) / LP_PIECE) : 0;
  const int together = max(1, (pieces + LP_STRETCHES / LP_WARPS - 1) / (LP_STRETCHES / LP_WARPS));      // pieces to a stretch
  if (TOP && tid == 0) { t.n = 0; t.reach = 0; }       // (the first barrier is behind the pass)
  uint32_t stretch = 0, *note = t.most + warp;
  int open = together;
  const auto load4 = [x, v1](int64_t i, float* v) {
    if (i >= 0 && i + 4 <= v1) {
      const float4 f = *reinterpret_cast<const float4*>(x + i);
      v[0] = f.x; v[1] = f.y; v[2] = f.z; v[3] = f.w;
    } else {
#pragma unroll
      for (int u = 0; u < 4; ++u) v[u] = i + u >= 0 && i + u < v1 ? x[i + u] : -INFINITY;
    }
  };
  const auto load = [load4, tid](int64_t at, float (&v)[LP_PER]) {
#pragma unroll
    for (int g = 0; g < LP_PER / 4; ++g) load4(at + 4 * (tid + g * LP_THREADS), v + 4 * g);
  };
  float next[LP_PER];
  load(v0, next);
  for (int64_t at = v0; at < v1; at += LP_PIECE) {
    float v[LP_PER];
#pragma unroll
    for (int i = 0; i < LP_PER; ++i) v[i] = next[i];
    if (at + LP_PIECE < v1) load(at + LP_PIECE, next);
    const auto token = [&](int i) { return (int)(at + 4 * (tid + (i / 4) * LP_THREADS) + i % 4); };
    float m = v[0];
#pragma unroll
    for (int i = 1; i < LP_PER; ++i) m = fmaxf(m, v[i]);
    if (TOP) {
      stretch = max(stretch, __reduce_max_sync(0xffffffffu, order_of(m)));
      if (--open == 0 || at + LP_PIECE >= v1) {
        if (lane == 0) *note = stretch;
        note += LP_WARPS;
        stretch = 0;
        open = together;
      }
    }
    if (m > s.m) raise(s, m);
    {
      const float2 low = make_float2(-s.m, -s.m), scale = make_float2(LOG2E, LOG2E);
      float2 sa = make_float2(0.f, 0.f), sb = sa;
#pragma unroll
      for (int i = 0; i < LP_PER; i += 2) {
        const float2 x = __fmul2_rn(__fadd2_rn(make_float2(v[i], v[i + 1]), low), scale);
        const float2 e = make_float2(ex2(x.x), ex2(x.y));
        sa = __fadd2_rn(sa, e);
        sb = __ffma2_rn(e, make_float2(held(x.x), held(x.y)), sb);
      }
      s.a += sa.x + sa.y;
      s.b += sb.x + sb.y;
    }
    if (scored) {
      // a larger token comes before the target; an equal one where its number is lower: pieces before the target, behind it, and its own
      if (at + LP_PIECE <= ties) {
#pragma unroll
        for (int i = 0; i < LP_PER; ++i) s.rank += v[i] >= xt;
      } else if (at >= ties) {
#pragma unroll
        for (int i = 0; i < LP_PER; ++i) s.rank += v[i] > xt;
      } else {
#pragma unroll
        for (int i = 0; i < LP_PER; ++i) s.rank += v[i] > xt || (v[i] == xt && token(i) < ties);
      }
      // (up to three places before the row hold -inf, too)
      if (xt == -INFINITY && at + 4 * tid < 0)
        for (int i = 0; i < 4; ++i) s.rank -= token(i) < 0;
    }
  }
  int listed = 0;
  if (TOP) {
    uint32_t from = max(NO_TOKEN + 1, find_floor(t, order_of(s.m), k));      // (a barrier: all stretches are noted)
    const int stretches = LP_WARPS * ((pieces + together - 1) / together);
    if (stretches >= k) {
      if (stretches <= LP_FEW) {
        // (each compares itself with all: 2 us where the search below takes 4)
        for (int i = tid; i < stretches; i += LP_THREADS) {
          const uint32_t mine = t.most[i];
          int above = 0;
          for (int j = 0; j < stretches; ++j) above += t.most[j] > mine || (t.most[j] == mine && j < i);
          if (above == k - 1) t.stretch_floor = mine;
        }
      } else if (warp == 0) {
        // the largest number of twenty bits (and twelve zeros) that k stretches reach, bit by bit
        uint32_t mine[LP_STRETCHES / 32], floor = 0;
#pragma unroll
        for (int u = 0; u < LP_STRETCHES / 32; ++u) mine[u] = lane + 32 * u < stretches ? t.most[lane + 32 * u] : 0u;
        for (uint32_t bit = 1u << 31; bit >= 1u << 12; bit >>= 1) {
          int reach = 0;
#pragma unroll
          for (int u = 0; u < LP_STRETCHES / 32; ++u)
            if (32 * u < stretches) reach += mine[u] >= (floor | bit);
          if (__reduce_add_sync(0xffffffffu, reach) >= k) floor |= bit;
        }
        if (lane == 0) t.stretch_floor = floor;
      }
      __syncthreads();
      from = max(from, t.stretch_floor);
    }
    for (int i = tid; i < stretches; i += LP_THREADS)
      if (t.most[i] >= from) t.reaching[atomicAdd(&t.reach, 1)] = i;
    __syncthreads();
    const float least = value_of(from);
    const auto keep = [&](float f, int token) {
      if (f >= least) {
        const int to = atomicAdd(&t.n, 1);
        if (to < LP_LIST) t.list[to] = ((unsigned long long)order_of(f) << 32) | (uint32_t)~token;
      }
    };
    for (int i = warp; i < t.reach; i += LP_WARPS) {
      const int st = t.reaching[i], who = (st % LP_WARPS) * 32 + lane;
      for (int p = st / LP_WARPS * together; p < min(pieces, (st / LP_WARPS + 1) * together); ++p) {
        float f[LP_PER];
#pragma unroll
        for (int g = 0; g < LP_PER / 4; ++g) load4(v0 + (int64_t)p * LP_PIECE + 4 * (who + g * LP_THREADS), f + 4 * g);
#pragma unroll
        for (int e = 0; e < LP_PER; ++e) keep(f[e], (int)(v0 + (int64_t)p * LP_PIECE) + 4 * (who + (e / 4) * LP_THREADS) + e % 4);
      }
    }
    __syncthreads();
    const int n = t.n;
    listed = n > LP_LIST ? scan_again(t, k, v0, v1, load) : n;
    listed = cut_list(t, listed, k);           // in order
  }

  s = warp_join(s);
  if (lane == 0) s_stats[warp] = s;
  __syncthreads();
  if (warp == 0) {
    s = lane < LP_WARPS ? s_stats[lane] : no_stats();
    s = warp_join(s);
  }
  if (slices > 1) {
    float* mine = a.part + (int64_t)blockIdx.x * LP_PART_FLOATS;
    if (tid == 0) {
      mine[0] = s.m; mine[1] = s.a; mine[2] = s.b; mine[3] = __int_as_float(s.rank);
    }
    if (TOP && tid < k) {
      reinterpret_cast<uint32_t*>(mine)[8 + 2 * tid] = tid < listed ? (uint32_t)(t.list[tid] >> 32) : 0u;
      reinterpret_cast<uint32_t*>(mine)[9 + 2 * tid] = tid < listed ? (uint32_t)t.list[tid] : 0u;
    }
    __syncthreads();
    if (tid == 0) last = count_arrival(&a.arrived[row]) == slices - 1;
    __syncthreads();
    if (!last) return;
    if (tid == 0) a.arrived[row] = 0;
    const float* all = a.part + (int64_t)row * slices * LP_PART_FLOATS;
    if (warp == 0) {
      s = no_stats();
      for (int i = lane; i < slices; i += 32) {
        const float* p = all + (int64_t)i * LP_PART_FLOATS;
        const Stats o = {__ldcg(p), __ldcg(p + 1), __ldcg(p + 2), __float_as_int(__ldcg(p + 3))};
        s = join(s, o);
      }
      s = warp_join(s);
    }
    if (TOP) {
      // The slices' lists are in order: at least k tokens lie at or above the q-th largest of their r-th ones, q r >= k.  Keys are distinct,
      // and no slice has more than k of them.
      const int r = (k + slices - 1) / slices, q = (k + r - 1) / r;
      const auto key_of = [&](int i, int j) {
        const uint32_t* p = reinterpret_cast<const uint32_t*>(all + (int64_t)i * LP_PART_FLOATS) + 8 + 2 * j;
        return ((unsigned long long)__ldcg(p) << 32) | __ldcg(p + 1);
      };
      const unsigned long long nth = tid < slices ? key_of(tid, r - 1) : 0ull;
      constexpr int KEYS = LP_MAX_SLICES * SPTS_LOGPROBS_MAX_TOP / LP_THREADS;
      unsigned long long key[KEYS];            // all on their way at once
#pragma unroll
      for (int u = 0; u < KEYS; ++u) {
        const int i = tid + u * LP_THREADS;
        key[u] = i < slices * k ? key_of(i / k, i % k) : 0ull;
      }
      __syncthreads();
      if (tid < slices) t.list[tid] = nth;
      if (tid == 0) { t.n = 0; t.best[0] = 0ull; }
      __syncthreads();
      if (tid < slices) {
        int above = 0;
        for (int j = 0; j < slices; ++j) above += t.list[j] > nth || (t.list[j] == nth && j < tid);
        if (above == q - 1) t.best[0] = nth;
      }
      __syncthreads();
      const unsigned long long least = max(t.best[0], 1ull);
      // no more than q - 1 slices have more than r of them at or above, so there are (q - 1) (k - r) + slices r at most
#pragma unroll
      for (int u = 0; u < KEYS; ++u) {
        if (key[u] >= least) {
          const int at = atomicAdd(&t.n, 1);
          if (at < LP_LIST) t.list[at] = key[u];
        }
      }
      __syncthreads();
      const int n = t.n;
      __syncthreads();
      if (n <= LP_LIST) {
        listed = cut_list(t, n, k);
      } else {
        unsigned long long bound = ~0ull;
        listed = 0;
        for (; listed < k; ++listed) {
          unsigned long long b = 0ull;
#pragma unroll
          for (int u = 0; u < KEYS; ++u)
            if (key[u] < bound && key[u] > b) b = key[u];
#pragma unroll
          for (int u = 16; u > 0; u >>= 1) b = max(b, __shfl_xor_sync(0xffffffffu, b, u));
          if (lane == 0) t.warp_best[warp] = b;
          __syncthreads();
          for (int w = 0; w < LP_WARPS; ++w) b = max(b, t.warp_best[w]);
          __syncthreads();
          if (b == 0ull) break;
          if (tid == 0) t.list[listed] = b;
          bound = b;
        }
        __syncthreads();
      }
    }
  }
  if (warp != 0) return;
  const float nan = __int_as_float(0x7FC00000);
  const bool bad = s.a != s.a, empty = s.a == 0.f;
  const float log_a = log2f(s.a) * LN2;
  if (lane == 0) {
    if (a.logprob != nullptr) a.logprob[row] = !scored ? 0.f : bad ? nan : empty ? -INFINITY : (xt - s.m) - log_a;
    if (a.rank != nullptr) a.rank[row] = scored ? s.rank : -1;
    if (a.entropy != nullptr) a.entropy[row] = bad ? nan : empty ? 0.f : log_a - s.b / s.a * LN2;
  }
  if (TOP && lane < k) {
    const bool there = lane < listed;
    const unsigned long long key = there ? t.list[lane] : 0ull;
    const int64_t at = (int64_t)row * k + lane;
    if (a.top_token != nullptr) a.top_token[at] = there ? (int32_t)~(uint32_t)key : -1;
    if (a.top_logprob != nullptr) a.top_logprob[at] = bad ? nan : there ? (value_of((uint32_t)(key >> 32)) - s.m) - log_a : -INFINITY;
  }
}

}  // namespace

spts_status launch_token_logprobs(spts_ctx* ctx, const float* logits, int64_t ld, int n, int vocab, const int32_t* targets, int n_top,
                                  float* logprob, int32_t* rank, float* entropy, float* top_logprob, int32_t* top_token) {
  if (n == 1) ld = 0;
  LogprobArgs a = {logits, ld, vocab, targets, n_top, logprob, rank, entropy, top_logprob, top_token, ctx->ws.lp_part, ctx->ws.lp_arrived};
  // The number of slices whose rounds of resident CTAs are over first, in microseconds: a round moves its bytes at 5 TB/s, one CTA alone
  // at 16 GB/s (a piece in a microsecond); then it looks for its alternatives, and the last slice of a row joins what the others left.
  const int resident = 4 * ctx->sm_count, most = ceil_div(vocab, LP_PIECE / 2);
  const double ends = n_top > 0 ? 6.0 : 2.0;
  int slices = 1;
  double least = 1e30;
  for (int s = 1; s <= LP_MAX_SLICES && s <= most && (s == 1 || (n <= LOGITS_MAX_ROWS && (int64_t)s * n <= LP_MAX_SHARES)); ++s) {
    const int64_t ctas = (int64_t)n * s, rest = ctas % resident;
    const double bytes = 4.0 * vocab / s, alone = bytes / 16e3;
    const auto round = [&](double c) { return (c * bytes / 5e6 > alone ? c * bytes / 5e6 : alone) + ends; };
    const double time = (double)(ctas / resident) * round(resident) + (rest ? round((double)rest) : 0.0) + (s > 1 ? 4.0 : 0.0);
    if (time < least) { least = time; slices = s; }
  }
  const int per = slices == 1 ? vocab + 3 : (int)align_up((size_t)ceil_div(vocab + 3, slices), 4);
  if (launch_dependent(n_top > 0 ? logprobs_kernel<true> : logprobs_kernel<false>, dim3((unsigned)((int64_t)n * slices)), dim3(LP_THREADS), ctx->stream, a,
                       slices, per) != cudaSuccess)
    return SPTS_ERR_CUDA;
  ctx->launches++;
  return SPTS_OK;
}

}  // namespace spts
