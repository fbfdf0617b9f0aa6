// Rules on the logits of a generation (penalties for tokens of the history, biases, grammar mask) and the greedy token,
// in one launch.
//
// A cluster of CTAs owns a row; every CTA owns a slice of the vocabulary and holds, in shared memory, whether and how
// often each token of its slice occurred and which bias entry counts for it.  The history is read once per row: every
// CTA takes its share of the entries and notes each in the shared memory of the CTA that owns the token (distributed
// shared memory).  Then every CTA passes over its slice of the logits once, and the slices' best tokens meet in CTA 0.
#include <cooperative_groups.h>

#include "spts_common.cuh"

namespace cg = cooperative_groups;

namespace spts {

namespace {

constexpr int LG_THREADS = 512;
constexpr int LG_CLUSTER = 8;
// tokens of a CTA's slice that are worked on at a time: 9 bytes of shared memory each
constexpr int LG_WINDOW = 20480;

struct LogitsArgs {
  const float* x; int64_t ld; int n, vocab;
  spts_logits_rules r;
  float* out; int64_t ldo;
  int32_t* token;
};

__device__ __forceinline__ void take(float& best, int& besti, float v, int i) {
  if (v > best || (v == best && i < besti)) { best = v; besti = i; }
}

__device__ __forceinline__ void range(const int32_t* start, int b, int n_all, int& i0, int& i1) {
  i0 = max(0, start[b]);
  i1 = min(n_all, start[b + 1]);
}

__global__ void __launch_bounds__(LG_THREADS) logits_kernel(LogitsArgs a, int per, int window) {
  extern __shared__ __align__(16) unsigned char smem[];
  // [window] times generated, [window] last bias entry + 1, [window] bytes: occurred
  uint32_t* count = reinterpret_cast<uint32_t*>(smem);
  int32_t* entry = reinterpret_cast<int32_t*>(count + window);
  uint8_t* seen = reinterpret_cast<uint8_t*>(entry + window);
  __shared__ float bv[32];
  __shared__ int bi[32];
  __shared__ float top_v;
  __shared__ int top_i;
  cg::cluster_group cl = cg::this_cluster();
  const int rank = (int)cl.block_rank(), nct = (int)cl.num_blocks();
  const int b = blockIdx.x / nct, tid = threadIdx.x;
  const bool hist = a.r.history != nullptr, bias = a.r.bias_token != nullptr;
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
    if (hist || bias) {
      for (int i = tid; i < window; i += LG_THREADS) { count[i] = 0u; entry[i] = 0; seen[i] = 0; }
      cl.sync();                                  // everyone's tables are empty
      if (hist) {
        int i0, i1;
        range(a.r.history_start, b, a.r.n_history, i0, i1);
        const int g0 = a.r.generated_start != nullptr ? a.r.generated_start[b] : i0;
        for (int i = i0 + rank * LG_THREADS + tid; i < i1; i += nct * LG_THREADS) {
          const int t = a.r.history[i];
          if (t < 0 || t >= a.vocab) continue;
          const int owner = t / per, off = t - owner * per - w0;
          if (off < 0 || off >= wn) continue;
          *cl.map_shared_rank(seen + off, owner) = 1;
          if (i >= g0) atomicAdd(cl.map_shared_rank(count + off, owner), 1u);
        }
      }
      if (bias) {
        int i0, i1;
        range(a.r.bias_start, b, a.r.n_bias, i0, i1);
        for (int i = i0 + rank * LG_THREADS + tid; i < i1; i += nct * LG_THREADS) {
          const int t = a.r.bias_token[i];
          if (t < 0 || t >= a.vocab) continue;
          const int owner = t / per, off = t - owner * per - w0;
          if (off >= 0 && off < wn) atomicMax(cl.map_shared_rank(entry + off, owner), i + 1);
        }
      }
      cl.sync();                                  // all entries have arrived
    }
    const int v0 = rank * per + w0;
    const int v1 = min(a.vocab, v0 + wn);
    for (int v = v0 + tid; v < v1; v += LG_THREADS) {
      float l = x[v];
      if (hist) {
        const uint32_t c = count[v - v0];
        if (seen[v - v0]) l = l > 0.f ? __fdiv_rn(l, rep) : __fmul_rn(l, rep);
        if (c > 0) l = __fsub_rn(__fsub_rn(l, __fmul_rn(fre, (float)c)), pre);
      }
      if (bias) {
        const int e = entry[v - v0];
        if (e > 0) l = __fadd_rn(l, a.r.bias_value[e - 1]);
      }
      if (mask != nullptr && !((mask[v >> 5] >> (v & 31)) & 1u)) l = -INFINITY;
      if (out != nullptr) out[v] = l;
      take(best, besti, l, v);
    }
    if (w0 + window < per) __syncthreads();       // the tables are emptied again (the others meet in the next cluster sync)
  }
  if (a.token == nullptr) {
    if (hist || bias) cl.sync();                  // nobody leaves while a neighbour may still write here
    return;
  }
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
  LogitsArgs a{logits, ld, n, vocab, rules, out, ldo, token};
  const int per = (int)align_up((size_t)ceil_div(vocab, LG_CLUSTER), 32);
  const int window = per < LG_WINDOW ? per : LG_WINDOW;
  const bool tables = rules.history != nullptr || rules.bias_token != nullptr;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(LG_CLUSTER * n);
  cfg.blockDim = dim3(LG_THREADS);
  cfg.dynamicSmemBytes = tables ? (size_t)window * 9 : 0;
  cfg.stream = ctx->stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = LG_CLUSTER;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (cudaFuncSetAttribute(logits_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, LG_WINDOW * 9) != cudaSuccess) return SPTS_ERR_CUDA;
  if (cudaLaunchKernelEx(&cfg, logits_kernel, a, per, window) != cudaSuccess) return SPTS_ERR_CUDA;
  SPTS_CUDA_OK(ctx);
  return SPTS_OK;
}

}  // namespace spts
