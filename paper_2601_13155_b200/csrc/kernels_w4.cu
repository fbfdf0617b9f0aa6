// Matrix-vector products with 4-bit weights (value = scale * (code - 8) + mid per group along the input axis) and the
// quantiser that fills them.
//
// w4_gemv_plain_kernel: one warp per output feature, CUDA cores, fp32 arithmetic; a lane takes eight codes (one word)
// per step.  fp32 storage and SPTS_REFERENCE_KERNELS.
#include "q4_common.cuh"

namespace spts {

namespace {

using namespace q4;

template <typename T>
__global__ void __launch_bounds__(256)
w4_quantize_kernel(const T* __restrict__ W, long n_words, int lanes, uint32_t* __restrict__ codes,
                   uint32_t* __restrict__ params, int* status) {
  const long i0 = (long)blockIdx.x * 256 + threadIdx.x, stride = (long)gridDim.x * 256;
  // every lane of a warp takes the same number of steps (the group's shuffles need all of them)
  for (long i = i0; (i & ~31L) < n_words; i += stride) {
    const bool in = i < n_words;                   // whole groups: n_words is a multiple of the lanes of a group
    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (in) load8(W + 8 * i, x);
    uint32_t p;
    bool bad;
    const uint32_t w = quantize8(x, lanes, p, nullptr, bad);
    if (in) {
      codes[i] = w;
      if (i % lanes == 0) {
        params[i / lanes] = p;
        if (bad) set_status(status, SPTS_ERR_NONFINITE);
      }
    }
  }
}

// One token's result through the form of the call: y (gate with u for the up projection) -> the stored value.
struct W4Out {
  const void* residual; int64_t ldr;
  void* Y; int64_t ldy;
  int fp32_out;
};
template <typename T>
__device__ __forceinline__ void w4_store(const W4Out& o, int t, int row, float y) {
  if (o.residual != nullptr) y = to_f32(((const T*)o.residual)[(size_t)t * o.ldr + row]) + y;
  if (o.fp32_out) ((float*)o.Y)[(size_t)t * o.ldy + row] = y;
  else ((T*)o.Y)[(size_t)t * o.ldy + row] = from_f32<T>(y);
}
__device__ __forceinline__ float silu_mul(float g, float u) { return g / (1.0f + expf(-g)) * u; }

template <typename T, int NT, bool TWO>
__global__ void __launch_bounds__(256)
w4_gemv_plain_kernel(const uint32_t* __restrict__ codes, const uint32_t* __restrict__ params,
                     const uint32_t* __restrict__ codes2, const uint32_t* __restrict__ params2, int out, int in, int group,
                     const T* __restrict__ X, int64_t ldx, int n, int norm, float eps, W4Out o) {
  const int row = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (row >= out) return;
  const int t0 = blockIdx.y * NT;
  const int words = in / 8, per_group = group / 8;
  float acc[NT], acc2[NT], ss[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) { acc[t] = 0.f; acc2[t] = 0.f; ss[t] = 0.f; }
  for (int w = lane; w < words; w += 32) {
    const uint32_t c = codes[(size_t)row * words + w], p = params[(size_t)row * (words / per_group) + w / per_group];
    uint32_t c2 = 0, p2 = 0;
    if (TWO) { c2 = codes2[(size_t)row * words + w]; p2 = params2[(size_t)row * (words / per_group) + w / per_group]; }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      if (t0 + t < n) {
        float x[8];
        load8(X + (size_t)(t0 + t) * ldx + 8 * w, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          acc[t] = fmaf(fmaf(lo_bf16(p), (float)((int)((c >> (4 * i)) & 15) - 8), hi_bf16(p)), x[i], acc[t]);
          if (TWO) acc2[t] = fmaf(fmaf(lo_bf16(p2), (float)((int)((c2 >> (4 * i)) & 15) - 8), hi_bf16(p2)), x[i], acc2[t]);
          ss[t] = fmaf(x[i], x[i], ss[t]);
        }
      }
    }
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    if (t0 + t < n) {
      float y = warp_sum(acc[t]);
      const float y2 = TWO ? warp_sum(acc2[t]) : 0.f;
      const float s2 = warp_sum(ss[t]);
      if (lane == 0) {
        const float rs = norm ? 1.0f / sqrtf(s2 / (float)in + eps) : 1.0f;
        y *= rs;
        if (TWO) y = silu_mul(y, y2 * rs);
        w4_store<T>(o, t0 + t, row, y);
      }
    }
  }
}

template <typename T, int NT>
spts_status launch_plain(spts_ctx* ctx, const W4GemvArgs& a) {
  const W4Out o{a.residual, a.ldr, a.Y, a.ldy, a.fp32_out};
  const dim3 grid(ceil_div(a.out, 8), ceil_div(a.n, NT));
  const uint32_t* c1 = (const uint32_t*)a.codes; const uint32_t* p1 = (const uint32_t*)a.params;
  const uint32_t* c2 = (const uint32_t*)a.codes2; const uint32_t* p2 = (const uint32_t*)a.params2;
  if (c2 != nullptr)
    w4_gemv_plain_kernel<T, NT, true><<<grid, 256, 0, ctx->stream>>>(c1, p1, c2, p2, a.out, a.in, a.group, (const T*)a.X, a.ldx, a.n,
                                                                     a.norm, ctx->desc.rms_eps, o);
  else
    w4_gemv_plain_kernel<T, NT, false><<<grid, 256, 0, ctx->stream>>>(c1, p1, c2, p2, a.out, a.in, a.group, (const T*)a.X, a.ldx, a.n,
                                                                      a.norm, ctx->desc.rms_eps, o);
  SPTS_CUDA_OK(ctx);
  return SPTS_OK;
}

}  // namespace

spts_status launch_w4_gemv(spts_ctx* ctx, const W4GemvArgs& a) {
  if (ctx->desc.dtype == SPTS_FP32) return a.n == 1 ? launch_plain<float, 1>(ctx, a) : launch_plain<float, 4>(ctx, a);
  return a.n == 1 ? launch_plain<bf16, 1>(ctx, a) : launch_plain<bf16, 4>(ctx, a);
}

spts_status launch_w4_quantize(spts_ctx* ctx, const void* W, int out, int in, int group, void* codes, void* params) {
  const long n_words = (long)out * (in / 8);
  long blocks = (n_words + 255) / 256;
  if (blocks > 16L * ctx->sm_count) blocks = 16L * ctx->sm_count;
  if (ctx->desc.dtype == SPTS_BF16)
    w4_quantize_kernel<bf16><<<(int)blocks, 256, 0, ctx->stream>>>((const bf16*)W, n_words, group / 8, (uint32_t*)codes,
                                                                   (uint32_t*)params, ctx->ws.status);
  else
    w4_quantize_kernel<float><<<(int)blocks, 256, 0, ctx->stream>>>((const float*)W, n_words, group / 8, (uint32_t*)codes,
                                                                    (uint32_t*)params, ctx->ws.status);
  SPTS_CUDA_OK(ctx);
  return SPTS_OK;
}

}  // namespace spts
