// Rules on the logits of a generation (penalties for tokens of the history, biases, grammar mask) and the greedy token,
// in one launch.
//
// A CTA owns a slice of a row's vocabulary and holds, in shared memory, a word per token of it: whether and how often the token
// occurred in the row's history, and whether a bias entry names it.  It reads the row's whole history and notes what falls into
// its slice: that is one read of it per slice from L2, but the alternative (each CTA reads a share and notes it in the owner's
// distributed shared memory) pays for every repeated token with a remote access to one address, and text repeats.  Then the
// slice's logits pass through once, four neighbouring tokens to a thread, with only the mask to apply; marked tokens are left
// out of the maximum and listed, and the listed ones, densely, go through the rules (applied in the pass itself they cost every
// warp the rules' instructions for its one marked token: 66 us for 64 rows of 152063).
// The slices' best tokens meet in a 64-bit maximum per row, from which the slice that arrives last takes the token.
//
// One row of 128256 after 33,000 tokens: 9.0 us, bound by the chain launch - tables - history - logits - maximum.  64 rows of 152063
// after 5100: 34 us, where memory asks for 12 (logits in and out); the instructions of tables, lists and history bound it
// (without any of them: 16 us).
#include "spts_common.cuh"

namespace spts {

namespace {

constexpr int LG_THREADS = 512;
constexpr int LG_BATCH = 2;             // groups of four logits of a thread in flight
constexpr int LG_HISTORY = 2;           // 16-byte pieces of the history of a thread in flight
constexpr int LG_BYTES = 8;             // shared memory per token of the slice: its word, 2 on the list, 2 for a bias entry
constexpr int LG_SLICE = 14336;         // tokens of a slice at most: two CTAs' tables in an SM's shared memory

struct LogitsArgs {
  const float* x; int64_t ld; int n, vocab;
  spts_logits_rules r;
  float* out; int64_t ldo;
  int32_t* token;
  unsigned long long* key; int* arrived;       // per row; zero between calls
};

// Larger value, then lower index, is the larger key; values are not NaN.
__device__ __forceinline__ unsigned long long key_of(float v, int i) {
  const uint32_t u = __float_as_uint(v == 0.f ? 0.f : v);
  return ((unsigned long long)((u & 0x80000000u) ? ~u : (u | 0x80000000u)) << 32) | (uint32_t)(0x7FFFFFFF - i);
}

// the largest entry number wins
__device__ __forceinline__ void last_entry(uint32_t* p, int e) { atomicMax(p, (uint32_t)e); }
__device__ __forceinline__ void last_entry(uint16_t* p, int e) {
  unsigned short seen = *p;
  while (seen < e) {
    const unsigned short was = atomicCAS(p, seen, (unsigned short)e);
    if (was == seen) break;
    seen = was;
  }
}

__device__ __forceinline__ void range(const int32_t* start, int b, int n_all, int& i0, int& i1) {
  i0 = min(max(0, start[b]), n_all);
  i1 = min(n_all, start[b + 1]);
}

constexpr uint32_t OCCURRED = 0x80000000u, BIASED = 0x40000000u, TIMES = 0x3FFFFFFFu;       // of a token's word

// E: an entry number of the row's bias list, 16 bits where the list is short enough
template <typename E>
__global__ void __launch_bounds__(LG_THREADS, 2) logits_kernel(LogitsArgs a, int slices, int per) {
  extern __shared__ __align__(16) unsigned char smem[];
  // [per] words, [per] last bias entry + 1, [per] listed tokens (slices are multiples of 32)
  uint32_t* word = reinterpret_cast<uint32_t*>(smem);
  E* entry = reinterpret_cast<E*>(word + per);
  uint16_t* list = reinterpret_cast<uint16_t*>(entry + per);
  __shared__ unsigned long long keys[LG_THREADS / 32];
  __shared__ int listed;
  const int b = blockIdx.x / slices, slice = blockIdx.x - b * slices, tid = threadIdx.x;
  const bool hist = a.r.history != nullptr, bias = a.r.bias_token != nullptr, tables = hist || bias;
  const float* x = a.x + (size_t)b * a.ld;
  float* out = a.out != nullptr ? a.out + (size_t)b * a.ldo : nullptr;
  const uint32_t* mask = a.r.mask != nullptr ? a.r.mask + (size_t)b * a.r.ld_mask : nullptr;
  const float rep = a.r.repetition != nullptr ? a.r.repetition[b] : 1.f;
  const float pre = a.r.presence != nullptr ? a.r.presence[b] : 0.f;
  const float fre = a.r.frequency != nullptr ? a.r.frequency[b] : 0.f;
  // token `base` (up to three before the row) lies on a 16-byte boundary, and so do all slices
  const int base = -(int)((reinterpret_cast<uintptr_t>(x) >> 2) & 3);
  const bool out4 = out != nullptr && ((reinterpret_cast<uintptr_t>(out + base) & 15) == 0);
  // the row's part of the lists: history [i0, i1), generated from g0 on, [p0, p1) of the prompt's part whole 16-byte pieces
  int i0 = 0, i1 = 0, g0 = 0, p0 = 0, p1 = 0, b0 = 0, b1 = 0;
  if (hist) {
    range(a.r.history_start, b, a.r.n_history, i0, i1);
    i1 = max(i0, i1);
    g0 = a.r.generated_start != nullptr ? min(max(a.r.generated_start[b], i0), i1) : i0;
    const bool by4 = (reinterpret_cast<uintptr_t>(a.r.history) & 15) == 0;
    p0 = by4 ? min((i0 + 3) & ~3, g0) : g0;
    p1 = by4 ? max(p0, g0 & ~3) : g0;
    if (p0 & 3) p1 = p0;                          // (no whole piece)
  }
  if (bias) range(a.r.bias_start, b, a.r.n_bias, b0, b1);
  unsigned long long best = 0;                    // (below every key)
  const int v0 = base + slice * per;             // tokens [v0, v0 + per), as far as there are such
  // groups of four tokens [j0, j1) lie in the row; up to three tokens before and behind them are taken one by one
  const int v1 = min(a.vocab, v0 + per), j0 = v0 < 0 ? 1 : 0, j1 = v1 > v0 ? (v1 - v0) >> 2 : 0;
  const float4* x4 = reinterpret_cast<const float4*>(x + v0);
  float4 l[LG_BATCH];
  uint32_t m0[LG_BATCH], m1[LG_BATCH];
  auto load = [&](int j) {
#pragma unroll
    for (int k = 0; k < LG_BATCH; ++k, j += LG_THREADS) {
      l[k] = make_float4(0.f, 0.f, 0.f, 0.f);
      m0[k] = m1[k] = 0xFFFFFFFFu;
      if (j < j1) {
        l[k] = x4[j];
        if (mask != nullptr) { m0[k] = __ldg(mask + ((v0 + 4 * j) >> 5)); m1[k] = __ldg(mask + ((v0 + 4 * j + 3) >> 5)); }
      }
    }
  };
  load(j0 + tid);
  // the first pieces of the lists are on their way before the tables are cleared
  const int4* h4 = reinterpret_cast<const int4*>(a.r.history);
  int4 first[LG_HISTORY];
  int first_bias = -1, first_made = -1;
#pragma unroll
  for (int k = 0; k < LG_HISTORY; ++k) first[k] = p0 / 4 + tid + k * LG_THREADS < p1 / 4 ? __ldg(h4 + p0 / 4 + tid + k * LG_THREADS) : make_int4(-1, -1, -1, -1);
  if (g0 + tid < i1) first_made = __ldg(a.r.history + g0 + tid);
  if (b0 + tid < b1) first_bias = __ldg(a.r.bias_token + b0 + tid);
  if (tables) {
    const uint32_t span = (uint32_t)per;
    const int n16 = per * (4 + (int)sizeof(E)) / 16;             // a multiple of 32 tokens: whole 16-byte words
    for (int i = tid; i < n16; i += LG_THREADS) reinterpret_cast<uint4*>(smem)[i] = make_uint4(0u, 0u, 0u, 0u);
    if (tid == 0) listed = 0;
    __syncthreads();
    // a token's place in the slice; tokens that there are not have none
    const auto place = [&](int t) { return t < 0 || t >= a.vocab ? 0xFFFFFFFFu : (uint32_t)(t - v0); };
    const auto mark = [&](int t) {
      const uint32_t o = place(t);
      if (o < span) word[o] = OCCURRED;
    };
    if (hist) {
      // whole 16-byte pieces of the prompt's part, then the ends and the generated part one by one
      for (int j = p0 / 4 + tid; j < p1 / 4; j += LG_HISTORY * LG_THREADS) {
        int4 t[LG_HISTORY];
#pragma unroll
        for (int k = 0; k < LG_HISTORY; ++k)
          t[k] = j == p0 / 4 + tid ? first[k] : j + k * LG_THREADS < p1 / 4 ? __ldg(h4 + j + k * LG_THREADS) : make_int4(-1, -1, -1, -1);
#pragma unroll
        for (int k = 0; k < LG_HISTORY; ++k) {
          mark(t[k].x); mark(t[k].y); mark(t[k].z); mark(t[k].w);
        }
      }
      for (int i = i0 + tid; i < p0; i += LG_THREADS) mark(__ldg(a.r.history + i));
      for (int i = p1 + tid; i < g0; i += LG_THREADS) mark(__ldg(a.r.history + i));
      __syncthreads();                          // the marks above are plain stores; from here on words change by atomics
      for (int i = g0 + tid; i < i1; i += LG_THREADS) {
        const uint32_t o = place(i == g0 + tid ? first_made : __ldg(a.r.history + i));
        if (o < span) { atomicOr(word + o, OCCURRED); atomicAdd(word + o, 1u); }
      }
    }
    for (int i = b0 + tid; i < b1; i += LG_THREADS) {
      const uint32_t o = place(i == b0 + tid ? first_bias : __ldg(a.r.bias_token + i));
      if (o < span) { atomicOr(word + o, BIASED); last_entry(entry + o, i - b0 + 1); }
    }
    __syncthreads();
  }
  // ---- the slice's logits, as they are or masked; marked tokens stay out of the maximum and are listed
  float top = -INFINITY;
  int topi = 0;
  const int lane = tid & 31;
  for (int jb = j0 + tid; jb - lane < j1; jb += LG_BATCH * LG_THREADS) {
    if (jb != j0 + tid) load(jb);
#pragma unroll
    for (int k = 0; k < LG_BATCH; ++k) {
      const int j = jb + k * LG_THREADS, v = v0 + 4 * j;
      if (j - lane >= j1) break;                 // the whole warp
      const bool in = j < j1;
      const uint32_t allowed = __funnelshift_r(m0[k], m1[k], v & 31);
      float y[4] = {l[k].x, l[k].y, l[k].z, l[k].w};
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (!in || !((allowed >> i) & 1u)) y[i] = -INFINITY;
      if (in) {
        if (out4) *reinterpret_cast<float4*>(out + v) = make_float4(y[0], y[1], y[2], y[3]);
        else if (out != nullptr) { out[v] = y[0]; out[v + 1] = y[1]; out[v + 2] = y[2]; out[v + 3] = y[3]; }
      }
      if (tables) {
        const uint4 w = in ? reinterpret_cast<const uint4*>(word)[j] : make_uint4(0u, 0u, 0u, 0u);
        if ((w.x | w.y | w.z | w.w) != 0u) {
          const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
          int at = atomicAdd(&listed, (w.x != 0u) + (w.y != 0u) + (w.z != 0u) + (w.w != 0u));
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (ww[i]) { list[at++] = (uint16_t)(4 * j + i); y[i] = -INFINITY; }
        }
      }
      const float m = fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3]));          // (passes over NaN)
      if (m > top) {                             // a thread's tokens ascend: the first of equals stays
        top = m;
        topi = v + (y[0] == m ? 0 : y[1] == m ? 1 : y[2] == m ? 2 : 3);
      }
    }
  }
  if (tid < 8) {                                 // the ends: tokens before the first group, then those behind the last
    const int v = tid < 4 ? v0 + tid : v0 + 4 * max(j0, j1) + tid - 4;
    if (v >= 0 && v < v1 && (tid >= 4 || j0 == 1)) {
      float y = x[v];
      if (mask != nullptr && !((__ldg(mask + (v >> 5)) >> (v & 31)) & 1u)) y = -INFINITY;
      if (out != nullptr) out[v] = y;
      if (tables && word[v - v0] != 0u) list[atomicAdd(&listed, 1)] = (uint16_t)(v - v0);
      else if (y > -INFINITY) best = max(best, key_of(y, v));
    }
  }
  if (top > -INFINITY) best = max(best, key_of(top, topi));
  // ---- the listed tokens
  if (tables) {
    __syncthreads();                            // what was written above is written again
    const int many = listed;
    for (int i = tid; i < many; i += LG_THREADS) {
      const int o = list[i], v = v0 + o;
      const uint32_t w = word[o];
      float y = x[v];                            // (in place: the logit itself, or -inf where the mask forbids the token anyway)
      if (w & OCCURRED) {
        y = y > 0.f ? __fdiv_rn(y, rep) : __fmul_rn(y, rep);
        const uint32_t c = w & TIMES;
        if (c > 0) y = __fsub_rn(__fsub_rn(y, __fmul_rn(fre, (float)c)), pre);
      }
      if (w & BIASED) y = __fadd_rn(y, a.r.bias_value[b0 + (int)entry[o] - 1]);
      if (mask != nullptr && !((__ldg(mask + (v >> 5)) >> (v & 31)) & 1u)) y = -INFINITY;
      if (out != nullptr) out[v] = y;
      if (y > -INFINITY) best = max(best, key_of(y, v));
    }
  }
  if (a.token == nullptr) return;
  for (int o = 16; o > 0; o >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, o));
  if ((tid & 31) == 0) keys[tid >> 5] = best;
  __syncthreads();
  if (tid < 32) {
    best = tid < LG_THREADS / 32 ? keys[tid] : 0;
    for (int o = 16; o > 0; o >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, o));
    if (tid == 0) {
      atomicMax(a.key + b, best);
      __threadfence();
      if (atomicAdd(a.arrived + b, 1) == slices - 1) {
        const unsigned long long k = atomicExch(a.key + b, 0ull);            // ready for the next call
        a.arrived[b] = 0;
        a.token[b] = k == 0 ? -1 : 0x7FFFFFFF - (int)(uint32_t)k;
      }
    }
  }
}

}  // namespace

spts_status launch_process_logits(spts_ctx* ctx, const float* logits, int64_t ld, int n, int vocab,
                                  const spts_logits_rules& rules, float* out, int64_t ldo, int32_t* token) {
  const bool tables = rules.history != nullptr || rules.bias_token != nullptr;
  const bool wide = rules.n_bias > 65534;                        // a row's entries may not fit 16 bits
  const int bytes = wide ? LG_BYTES + 2 : LG_BYTES;
  for (int r0 = 0; r0 < n; r0 += LOGITS_MAX_ROWS) {
    const int rows = n - r0 < LOGITS_MAX_ROWS ? n - r0 : LOGITS_MAX_ROWS;
    // Slices of at most LG_SLICE tokens, whose tables let two CTAs of 512 threads onto an SM (64 rows of 152063: 34 us; four of 256
    // with 6144 tokens 38, three of 384 with 8192 38, five of 256 40), as many as the rounds of resident CTAs that these take have
    // room for, and down to 1024 tokens where rows are few (one row of 128256 with a history of 33,000: 9.0 us; slices of 4096
    // 12.5, sixteen of 1024 threads 12.8).
    const int seats = 2 * ctx->sm_count, least = ceil_div(vocab, LG_SLICE), rounds = ceil_div(rows * least, seats);
    int slices = rounds * seats / rows > least ? rounds * seats / rows : least;
    if (slices > ceil_div(vocab, 1024)) slices = ceil_div(vocab, 1024);
    const int per = (int)align_up((size_t)ceil_div(vocab + 3, slices), 32);
    LogitsArgs a{logits + (size_t)r0 * ld, ld, rows, vocab, rules, out != nullptr ? out + (size_t)r0 * ldo : nullptr, ldo,
                 token != nullptr ? token + r0 : nullptr, ctx->ws.lg_key, ctx->ws.lg_arrived};
    if (r0 > 0) {
      spts_logits_rules& r = a.r;
      if (r.history_start) r.history_start += r0;
      if (r.generated_start) r.generated_start += r0;
      if (r.repetition) r.repetition += r0;
      if (r.presence) r.presence += r0;
      if (r.frequency) r.frequency += r0;
      if (r.bias_start) r.bias_start += r0;
      if (r.mask) r.mask += (size_t)r0 * r.ld_mask;
    }
    auto kernel = wide ? logits_kernel<uint32_t> : logits_kernel<uint16_t>;
    const size_t smem = tables ? (size_t)per * bytes : 0;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (LG_SLICE + 32) * bytes) != cudaSuccess) return SPTS_ERR_CUDA;
    kernel<<<slices * rows, LG_THREADS, smem, ctx->stream>>>(a, slices, per);
    SPTS_CUDA_OK(ctx);
  }
  return SPTS_OK;
}

}  // namespace spts
