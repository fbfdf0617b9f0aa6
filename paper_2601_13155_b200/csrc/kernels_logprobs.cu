// Log probabilities of given tokens with their ranks, the entropy and the most likely alternatives of rows of logits, in one launch
// and one read of the logits.
//
// A CTA takes a slice of a row, 4096 tokens at a time, eight to a thread.  With m the largest logit so far it holds A = sum e^(l - m) and
// B = sum e^(l - m) (l - m); when m grows by g, A becomes A e^-g and B (B - g A) e^-g.  At the end lse = m + log A and
// entropy = log A - B / A: no difference of large sums.  The target's logit is read first, so its rank is a count in the same pass.
// Alternatives: tokens above the worst of the n_top best so far go onto a list in shared memory, which is cut back to the n_top best, in order,
// when it grows long.  Of a first piece almost all tokens would go there; a floor is found beforehand: the eighth largest of the 16 warps' r-th
// largest token of a lane, r = ceil(n_top / 8), below which nothing among the best can lie.  Where so many tokens are equal that
// the list still runs over, the best are taken one after the other.
// A row is shared by slices where rows are few; the slice that arrives last joins what the others left, in their order.
#include "spts_common.cuh"

namespace spts {

namespace {

constexpr int LP_THREADS = 512, LP_WARPS = LP_THREADS / 32;
constexpr int LP_PER = 8;                      // tokens of a thread at a time, two 16-byte loads
constexpr int LP_PIECE = LP_THREADS * LP_PER;
constexpr int LP_LIST = 512;                   // candidates in shared memory
constexpr int LP_CUT = 128;                    // the list is cut back from here on: a thread per candidate compares it with all others
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

__device__ __forceinline__ float exp_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x * 1.4426950408889634f));
  return y;
}

struct Stats {
  float m, a, b;
  int rank;
  bool bad;          // a NaN or +inf was seen
};
// m starts at the lowest finite value, so that no difference is undefined
__device__ __forceinline__ Stats no_stats() { return {-3.402823466e38f, 0.f, 0.f, 0, false}; }
// What lies more than 150 below the maximum adds nothing in fp32; the difference is held there, so -inf times zero cannot come about.
__device__ __forceinline__ float below(float l, float m) { return fmaxf(l - m, -150.f); }
__device__ __forceinline__ void raise(Stats& s, float m) {
  const float g = below(s.m, m), e = exp_fast(g);
  s.b = (s.b + g * s.a) * e;
  s.a *= e;
  s.m = m;
}
__device__ __forceinline__ Stats join(Stats x, Stats y) {
  const float m = fmaxf(x.m, y.m);
  raise(x, m);
  raise(y, m);
  return {m, x.a + y.a, x.b + y.b, x.rank + y.rank, x.bad || y.bad};
}
__device__ __forceinline__ Stats warp_join(Stats s) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    Stats t;
    t.m = __shfl_xor_sync(0xffffffffu, s.m, o);
    t.a = __shfl_xor_sync(0xffffffffu, s.a, o);
    t.b = __shfl_xor_sync(0xffffffffu, s.b, o);
    t.rank = __shfl_xor_sync(0xffffffffu, s.rank, o);
    t.bad = __shfl_xor_sync(0xffffffffu, (int)s.bad, o) != 0;
    s = join(s, t);
  }
  return s;
}

struct TopShared {
  unsigned long long list[LP_LIST];            // order << 32 | ~token: the larger key comes first
  unsigned long long best[SPTS_LOGPROBS_MAX_TOP];
  unsigned long long warp_best[LP_WARPS];
  uint32_t warp_floor[LP_WARPS];
  int n;                                       // candidates asked for, of which those below LP_LIST are there
};

// The list [n] becomes its k best, in order; returns how many there are.  All threads.
__device__ __forceinline__ int cut_list(TopShared& t, int n, int k) {
  const int tid = threadIdx.x;
  const unsigned long long mine = tid < n ? t.list[tid] : 0ull;
  int r = 0;
  if (tid < n)
    for (int j = 0; j < n; ++j) r += t.list[j] > mine;
  __syncthreads();
  if (tid < n && r < k) t.list[r] = mine;
  if (tid == 0) t.n = min(n, k);
  __syncthreads();
  return min(n, k);
}

template <bool TOP>
__global__ void __launch_bounds__(LP_THREADS, 2) logprobs_kernel(LogprobArgs a, int slices, int per) {
  __shared__ Stats s_stats[LP_WARPS];
  __shared__ TopShared t;
  __shared__ bool last;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int row = blockIdx.x / slices, slice = blockIdx.x - row * slices;
  const float* x = a.x + (int64_t)row * a.ld;
  // token `base` (up to three before the row) lies on a 16-byte boundary, and so do all slices and pieces
  const int base = -(int)((reinterpret_cast<uintptr_t>(x) >> 2) & 3);
  const int64_t v0 = base + (int64_t)slice * per, v1 = min((int64_t)a.vocab, v0 + per);
  const int target = a.target != nullptr ? a.target[row] : -1;
  const bool scored = target >= 0 && target < a.vocab;
  const float xt = scored ? x[target] : 0.f;
  const int ties = (int)min((int64_t)target, v1);      // tokens below this one come before an equal target
  const int k = a.n_top;
  Stats s = no_stats();
  if (TOP && tid == 0) t.n = 0;
  uint32_t floor_order = NO_TOKEN;             // candidates lie above
  int listed = 0;
  if (TOP) __syncthreads();

  auto load = [&](int64_t at, float (&v)[LP_PER]) {
#pragma unroll
    for (int g = 0; g < LP_PER / 4; ++g) {
      const int64_t i = at + 4 * (tid + g * LP_THREADS);
      if (i >= 0 && i + 4 <= v1) {
        const float4 f = *reinterpret_cast<const float4*>(x + i);
        v[4 * g] = f.x; v[4 * g + 1] = f.y; v[4 * g + 2] = f.z; v[4 * g + 3] = f.w;
      } else {
#pragma unroll
        for (int u = 0; u < 4; ++u) v[4 * g + u] = i + u >= 0 && i + u < v1 ? x[i + u] : -INFINITY;
      }
    }
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
    if (m > s.m) raise(s, m);
#pragma unroll
    for (int i = 0; i < LP_PER; ++i) {
      const float d = below(v[i], s.m), e = exp_fast(d);
      s.a += e;
      s.b = fmaf(e, d, s.b);
      s.bad |= !(v[i] < INFINITY);
    }
    if (scored) {
#pragma unroll
      for (int i = 0; i < LP_PER; ++i) s.rank += v[i] > xt || (v[i] == xt && token(i) < ties);
      // (up to three places before the row hold -inf, too)
      if (xt == -INFINITY && at + 4 * tid < 0)
        for (int i = 0; i < 4; ++i) s.rank -= token(i) < 0;
    }
    if (TOP) {
      uint32_t least = floor_order + 1;
      uint32_t o[LP_PER], top = 0;
#pragma unroll
      for (int i = 0; i < LP_PER; ++i) { o[i] = order_of(v[i]); top = max(top, o[i]); }
      // of a list of k
      auto worst = [&]() {
        uint32_t w = 0xFFFFFFFFu;
        for (int i = 0; i < k; ++i) w = min(w, (uint32_t)(t.list[i] >> 32));
        return w;
      };
      auto find_floor = [&]() {
        const int r = (k + 7) / 8;
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
        return __shfl_sync(0xffffffffu, f, __ffs(__ballot_sync(0xffffffffu, above == 7 && lane < LP_WARPS)) - 1);
      };
      auto append = [&](uint32_t from) {
        if (__any_sync(0xffffffffu, top >= from)) {
#pragma unroll
          for (int i = 0; i < LP_PER; ++i) {
            const uint32_t take = __ballot_sync(0xffffffffu, o[i] >= from);
            if (take == 0) continue;
            int at_list = 0;
            if (lane == 0) at_list = atomicAdd(&t.n, __popc(take));
            at_list = __shfl_sync(0xffffffffu, at_list, 0) + __popc(take & ((1u << lane) - 1));
            if (o[i] >= from && at_list < LP_LIST) t.list[at_list] = ((unsigned long long)o[i] << 32) | (uint32_t)~token(i);
          }
        }
        __syncthreads();
        const int n = t.n;
        __syncthreads();
        return n;
      };
      int n = LP_LIST + 1;
      if (at > v0) n = append(least);
      if (n > LP_LIST) {
        // too many, or the first piece: those listed before are cut back, and a floor is found
        if (tid == 0) t.n = listed;
        __syncthreads();
        if (listed > k) {
          listed = cut_list(t, listed, k);
          floor_order = worst();
        }
        least = max(floor_order + 1, find_floor());
        n = append(least);
        if (n > LP_LIST) {
          // equal tokens beyond number: the best of the list and of this piece, one by one
          if (tid == 0) t.n = listed;
          unsigned long long bound = ~0ull;
          const unsigned long long mine = tid < listed ? t.list[tid] : 0ull;
          int got = 0;
          for (; got < k; ++got) {
            unsigned long long b = mine < bound ? mine : 0ull;
#pragma unroll
            for (int i = 0; i < LP_PER; ++i) {
              const unsigned long long key = ((unsigned long long)o[i] << 32) | (uint32_t)~token(i);
              if (o[i] > NO_TOKEN && key < bound && key > b) b = key;
            }
#pragma unroll
            for (int u = 16; u > 0; u >>= 1) b = max(b, __shfl_xor_sync(0xffffffffu, b, u));
            if (lane == 0) t.warp_best[warp] = b;
            __syncthreads();
            for (int w = 0; w < LP_WARPS; ++w) b = max(b, t.warp_best[w]);
            __syncthreads();
            if (b == 0ull) break;
            if (tid == 0) t.best[got] = b;
            bound = b;
          }
          __syncthreads();
          if (tid < got) t.list[tid] = t.best[tid];
          if (tid == 0) t.n = got;
          __syncthreads();
          n = got;
        }
      }
      const bool grown = n != listed;
      listed = n;
      if (listed > LP_CUT || (at == v0 && listed > k)) listed = cut_list(t, listed, k);
      if (grown && listed == k) floor_order = worst();
    }
  }
  if (TOP) listed = cut_list(t, listed, k);    // in order

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
      mine[0] = s.m; mine[1] = s.a; mine[2] = s.b; mine[3] = __int_as_float(s.rank); mine[4] = s.bad ? 1.f : 0.f;
    }
    if (TOP && tid < k) {
      reinterpret_cast<uint32_t*>(mine)[8 + 2 * tid] = tid < listed ? (uint32_t)(t.list[tid] >> 32) : 0u;
      reinterpret_cast<uint32_t*>(mine)[9 + 2 * tid] = tid < listed ? (uint32_t)t.list[tid] : 0u;
    }
    __threadfence();
    __syncthreads();
    if (tid == 0) last = atomicAdd(&a.arrived[row], 1) == slices - 1;
    __syncthreads();
    if (!last) return;
    __threadfence();
    if (tid == 0) a.arrived[row] = 0;
    const float* all = a.part + (int64_t)row * slices * LP_PART_FLOATS;
    if (warp == 0) {
      s = no_stats();
      for (int i = lane; i < slices; i += 32) {
        const float* p = all + (int64_t)i * LP_PART_FLOATS;
        const Stats o = {__ldcg(p), __ldcg(p + 1), __ldcg(p + 2), __float_as_int(__ldcg(p + 3)), __ldcg(p + 4) != 0.f};
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
      for (int i = tid; i < slices * k; i += LP_THREADS) {
        const unsigned long long key = key_of(i / k, i % k);
        if (key >= least) {
          const int at = atomicAdd(&t.n, 1);
          if (at < LP_LIST) t.list[at] = key;
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
          for (int i = tid; i < slices * k; i += LP_THREADS) {
            const unsigned long long key = key_of(i / k, i % k);
            if (key < bound && key > b) b = key;
          }
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
  const bool empty = !(s.a > 0.f);
  const float log_a = logf(s.a);
  if (lane == 0) {
    if (a.logprob != nullptr) a.logprob[row] = !scored ? 0.f : s.bad ? nan : empty ? -INFINITY : (xt - s.m) - log_a;
    if (a.rank != nullptr) a.rank[row] = scored ? s.rank : -1;
    if (a.entropy != nullptr) a.entropy[row] = s.bad ? nan : empty ? 0.f : log_a - s.b / s.a;
  }
  if (TOP && lane < k) {
    const bool there = lane < listed;
    const unsigned long long key = there ? t.list[lane] : 0ull;
    const int64_t at = (int64_t)row * k + lane;
    if (a.top_token != nullptr) a.top_token[at] = there ? (int32_t)~(uint32_t)key : -1;
    if (a.top_logprob != nullptr) a.top_logprob[at] = s.bad ? nan : there ? (value_of((uint32_t)(key >> 32)) - s.m) - log_a : -INFINITY;
  }
}

}  // namespace

spts_status launch_token_logprobs(spts_ctx* ctx, const float* logits, int64_t ld, int n, int vocab, const int32_t* targets, int n_top,
                                  float* logprob, int32_t* rank, float* entropy, float* top_logprob, int32_t* top_token) {
  if (n == 1) ld = 0;
  LogprobArgs a = {logits, ld, vocab, targets, n_top, logprob, rank, entropy, top_logprob, top_token, ctx->ws.lp_part, ctx->ws.lp_arrived};
  // as many slices as three CTAs to an SM, none shorter than half a piece
  int slices = 3 * ctx->sm_count / n;
  const int most = ceil_div(vocab, LP_PIECE / 2);
  slices = slices > most ? most : slices;
  slices = slices > LP_MAX_SLICES ? LP_MAX_SLICES : slices;
  slices = n > LOGITS_MAX_ROWS || slices < 1 || (int64_t)slices * n > LP_MAX_SHARES ? 1 : slices;
  const int per = slices == 1 ? vocab + 3 : (int)align_up((size_t)ceil_div(vocab + 3, slices), 4);
  if (n_top > 0) logprobs_kernel<true><<<(unsigned)((int64_t)n * slices), LP_THREADS, 0, ctx->stream>>>(a, slices, per);
  else logprobs_kernel<false><<<(unsigned)((int64_t)n * slices), LP_THREADS, 0, ctx->stream>>>(a, slices, per);
  SPTS_CUDA_OK(ctx);
  return SPTS_OK;
}

}  // namespace spts
