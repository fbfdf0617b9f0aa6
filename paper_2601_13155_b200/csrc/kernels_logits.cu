// Rules on the logits of a generation (penalties for tokens of the history, biases, grammar mask) and the greedy token,
// in one launch.
//
// A cluster of CTAs owns a row; every CTA owns a slice of the vocabulary and holds, in shared memory, whether and how
// often each token of its slice occurred and which bias entry counts for it.  Every CTA reads the row's whole history and
// notes what falls into its slice: that is 16 reads of it from L2, but the alternative (each CTA reads a share and notes it
// in the owner's distributed shared memory) pays for every repeated token with a remote access to one address, and text
// repeats (one row of 128256 with a history of 33024: 18 us).  Then every CTA passes over its slice of the logits once, and
// the slices' best tokens meet in CTA 0.
// Bound by memory at many rows (logits in and out), by the chain launch - tables - history - logits - argmax at one; so
// the logits are loaded eight to a thread at a time (one at a time took 31 dependent trips to memory per thread: 31 us for
// one row of 128256), and the first eight before the tables are even cleared.
#include <cooperative_groups.h>

#include "spts_common.cuh"

namespace cg = cooperative_groups;

namespace spts {

namespace {

constexpr int LG_THREADS = 512;
constexpr int LG_BATCH = 8;             // logits of a thread in flight
constexpr int LG_HISTORY = 4;           // 16-byte pieces of the history of a thread in flight
constexpr int LG_BYTES = 6;             // shared memory per token of the slice: its word, and 2 for a bias entry
// tokens of a CTA's slice that are worked on at a time
constexpr int LG_WINDOW = 36864;

struct LogitsArgs {
  const float* x; int64_t ld; int n, vocab;
  spts_logits_rules r;
  float* out; int64_t ldo;
  int32_t* token;
};

__device__ __forceinline__ void take(float& best, int& besti, float v, int i) {
  if (v > best || (v == best && i < besti)) { best = v; besti = i; }
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
  i0 = max(0, start[b]);
  i1 = min(n_all, start[b + 1]);
}

constexpr uint32_t OCCURRED = 0x80000000u, BIASED = 0x40000000u, TIMES = 0x3FFFFFFFu;       // of a token's word

// E: an entry number of the row's bias list, 16 bits where the list is short enough
template <typename E>
__global__ void __launch_bounds__(LG_THREADS) logits_kernel(LogitsArgs a, int per, int window) {
  extern __shared__ __align__(16) unsigned char smem[];
  // [window] words: occurred, biased, times generated; [window] last bias entry + 1 (windows are multiples of 32)
  uint32_t* word = reinterpret_cast<uint32_t*>(smem);
  E* entry = reinterpret_cast<E*>(word + window);
  __shared__ float bv[32];
  __shared__ int bi[32];
  __shared__ float top_v;
  __shared__ int top_i;
  cg::cluster_group cl = cg::this_cluster();
  const int rank = (int)cl.block_rank(), nct = (int)cl.num_blocks();
  const int b = blockIdx.x / nct, tid = threadIdx.x;
  const bool hist = a.r.history != nullptr, bias = a.r.bias_token != nullptr, tables = hist || bias;
  const float* x = a.x + (size_t)b * a.ld;
  float* out = a.out != nullptr ? a.out + (size_t)b * a.ldo : nullptr;
  const uint32_t* mask = a.r.mask != nullptr ? a.r.mask + (size_t)b * a.r.ld_mask : nullptr;
  const float rep = a.r.repetition != nullptr ? a.r.repetition[b] : 1.f;
  const float pre = a.r.presence != nullptr ? a.r.presence[b] : 0.f;
  const float fre = a.r.frequency != nullptr ? a.r.frequency[b] : 0.f;
  float best = -INFINITY;
  int besti = 0x7FFFFFFF;
  for (int w0 = 0; w0 < per; w0 += window) {
    const int wn = min(window, per - w0);
    const int v0 = rank * per + w0, v1 = min(a.vocab, v0 + wn);
    const uint32_t span = (uint32_t)max(0, v1 - v0);
    float l[LG_BATCH];
    uint32_t mw[LG_BATCH];
    // logits v, v + LG_THREADS, ...; v0 and the steps are multiples of 32, so a thread's bit in a mask word is its lane's
    auto load = [&](int v) {
#pragma unroll
      for (int k = 0; k < LG_BATCH; ++k) {
        const int i = v + k * LG_THREADS;
        l[k] = i < v1 ? __ldcs(x + i) : 0.f;
        mw[k] = i < v1 && mask != nullptr ? __ldg(mask + (i >> 5)) : 0xFFFFFFFFu;
      }
    };
    load(v0 + tid);
    int b0 = 0, b1 = 0;
    if (bias) range(a.r.bias_start, b, a.r.n_bias, b0, b1);
    if (tables) {
      const int n16 = window * (4 + (int)sizeof(E)) / 16;             // a multiple of 32 tokens: whole 16-byte words
      for (int i = tid; i < n16; i += LG_THREADS) reinterpret_cast<uint4*>(smem)[i] = make_uint4(0u, 0u, 0u, 0u);
      int i0 = 0, i1 = 0, g0 = 0;
      if (hist) {
        range(a.r.history_start, b, a.r.n_history, i0, i1);
        g0 = a.r.generated_start != nullptr ? min(max(a.r.generated_start[b], i0), i1) : i0;
      }
      __syncthreads();
      if (hist) {
        // whole 16-byte pieces of the prompt's part, then the ends and the generated part one by one
        const bool by4 = (reinterpret_cast<uintptr_t>(a.r.history) & 15) == 0;
        const int p0 = by4 ? min((i0 + 3) & ~3, g0) : g0, p1 = by4 ? max(p0, g0 & ~3) : g0;
        const int4* h4 = reinterpret_cast<const int4*>(a.r.history);
        for (int j = p0 / 4 + tid; j < p1 / 4; j += LG_HISTORY * LG_THREADS) {
          int4 t[LG_HISTORY];
#pragma unroll
          for (int k = 0; k < LG_HISTORY; ++k) t[k] = j + k * LG_THREADS < p1 / 4 ? __ldg(h4 + j + k * LG_THREADS) : make_int4(-1, -1, -1, -1);
#pragma unroll
          for (int k = 0; k < LG_HISTORY; ++k) {
            const uint32_t o0 = t[k].x - v0, o1 = t[k].y - v0, o2 = t[k].z - v0, o3 = t[k].w - v0;
            if (o0 < span) word[o0] = OCCURRED;
            if (o1 < span) word[o1] = OCCURRED;
            if (o2 < span) word[o2] = OCCURRED;
            if (o3 < span) word[o3] = OCCURRED;
          }
        }
        for (int i = i0 + tid; i < p0; i += LG_THREADS) {
          const uint32_t o = __ldg(a.r.history + i) - v0;
          if (o < span) word[o] = OCCURRED;
        }
        for (int i = p1 + tid; i < g0; i += LG_THREADS) {
          const uint32_t o = __ldg(a.r.history + i) - v0;
          if (o < span) word[o] = OCCURRED;
        }
        __syncthreads();                          // the marks above are plain stores; from here on words change by atomics
        for (int i = g0 + tid; i < i1; i += LG_THREADS) {
          const uint32_t o = __ldg(a.r.history + i) - v0;
          if (o < span) { atomicOr(word + o, OCCURRED); atomicAdd(word + o, 1u); }
        }
      }
      if (bias) {
        for (int i = b0 + tid; i < b1; i += LG_THREADS) {
          const uint32_t o = __ldg(a.r.bias_token + i) - v0;
          if (o < span) { atomicOr(word + o, BIASED); last_entry(entry + o, i - b0 + 1); }
        }
      }
      __syncthreads();
    }
    const uint32_t bit = 1u << (tid & 31);
    for (int v = v0 + tid; v < v1; v += LG_BATCH * LG_THREADS) {
      if (v != v0 + tid) load(v);
      uint32_t tw[LG_BATCH];
#pragma unroll
      for (int k = 0; k < LG_BATCH; ++k) tw[k] = tables && v + k * LG_THREADS < v1 ? word[v - v0 + k * LG_THREADS] : 0u;
#pragma unroll
      for (int k = 0; k < LG_BATCH; ++k) {
        const int i = v + k * LG_THREADS;
        float y = l[k];
        if (tw[k] != 0u) {
          if (tw[k] & OCCURRED) {
            y = y > 0.f ? __fdiv_rn(y, rep) : __fmul_rn(y, rep);
            const uint32_t c = tw[k] & TIMES;
            if (c > 0) y = __fsub_rn(__fsub_rn(y, __fmul_rn(fre, (float)c)), pre);
          }
          if (tw[k] & BIASED) y = __fadd_rn(y, a.r.bias_value[b0 + (int)entry[i - v0] - 1]);
        }
        if (!(mw[k] & bit)) y = -INFINITY;
        if (i < v1) {
          if (out != nullptr) out[i] = y;
          if (y > best || besti == 0x7FFFFFFF) { if (y == y) { best = y; besti = i; } }        // a thread's indices ascend
        }
      }
    }
    if (w0 + window < per) __syncthreads();       // the tables are emptied again
  }
  if (a.token == nullptr) return;
  for (int o = 16; o > 0; o >>= 1) take(best, besti, __shfl_xor_sync(0xffffffffu, best, o), __shfl_xor_sync(0xffffffffu, besti, o));
  if ((tid & 31) == 0) { bv[tid >> 5] = best; bi[tid >> 5] = besti; }
  __syncthreads();
  if (tid < 32) {
    best = tid < LG_THREADS / 32 ? bv[tid] : -INFINITY;
    besti = tid < LG_THREADS / 32 ? bi[tid] : 0x7FFFFFFF;
    for (int o = 16; o > 0; o >>= 1) take(best, besti, __shfl_xor_sync(0xffffffffu, best, o), __shfl_xor_sync(0xffffffffu, besti, o));
    if (tid == 0) { top_v = best; top_i = besti; }
  }
  cl.sync();
  if (rank == 0 && tid == 0) {
    for (int r = 0; r < nct; ++r) take(best, besti, *cl.map_shared_rank(&top_v, r), *cl.map_shared_rank(&top_i, r));
    a.token[b] = best == -INFINITY ? -1 : besti;
  }
  cl.sync();                                      // CTA 0 has read the others' shared memory
}

}  // namespace

spts_status launch_process_logits(spts_ctx* ctx, const float* logits, int64_t ld, int n, int vocab,
                                  const spts_logits_rules& rules, float* out, int64_t ldo, int32_t* token) {
  const LogitsArgs a{logits, ld, n, vocab, rules, out, ldo, token};
  const bool tables = rules.history != nullptr || rules.bias_token != nullptr;
  // sixteen CTAs to a row where each still has several logits per thread, else eight (the portable size)
  const int cluster = vocab > 16 * LG_THREADS * 2 ? 16 : 8;
  const bool wide = rules.n_bias > 65534;                        // a row's entries may not fit 16 bits
  const int per = (int)align_up((size_t)ceil_div(vocab, cluster), 32);
  const int most = wide ? LG_WINDOW * LG_BYTES / (LG_BYTES + 2) / 32 * 32 : LG_WINDOW;
  const int window = !tables || per < most ? per : most;
  void (*kernel)(LogitsArgs, int, int) = wide ? logits_kernel<uint32_t> : logits_kernel<uint16_t>;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(cluster * n);
  cfg.blockDim = dim3(LG_THREADS);
  cfg.dynamicSmemBytes = tables ? (size_t)window * (wide ? LG_BYTES + 2 : LG_BYTES) : 0;
  cfg.stream = ctx->stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cluster;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, LG_WINDOW * LG_BYTES) != cudaSuccess ||
      cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess)
    return SPTS_ERR_CUDA;
  if (cudaLaunchKernelEx(&cfg, kernel, a, per, window) != cudaSuccess) return SPTS_ERR_CUDA;
  SPTS_CUDA_OK(ctx);
  return SPTS_OK;
}

}  // namespace spts
