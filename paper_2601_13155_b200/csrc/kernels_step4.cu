// What a decode step with 4-bit weights and caches needs besides its products, its attention and the rules on its logits:
// the tokens' embedding rows, and the rotation of q and k between the q / k / v projection and the cache.  Both are a few
// kilobytes of work between larger kernels, a launch's latency each: 4.5 and 2.9 us for 1 to 8 tokens of 4096 features, 32 + 2 x 8 heads
// (serialised, cold).
#include "spts_common.cuh"

namespace spts {

namespace {

template <typename T>
__global__ void __launch_bounds__(256) embed_rows_kernel(const T* __restrict__ embed, const int32_t* __restrict__ token, int vocab, int D,
                                                         T* __restrict__ x, int* status) {
  const int row = blockIdx.x, t = token[row];
  const bool in = t >= 0 && t < vocab;
  if (!in && threadIdx.x == 0) set_status(status, SPTS_ERR_INDEX);
  for (int i = threadIdx.x; i < D; i += 256) x[(size_t)row * D + i] = in ? embed[(size_t)t * D + i] : from_f32<T>(0.f);
}

// in [n, (H + 2 Hkv) d] fp32 -> out in the storage type: q and k rotated (pairs (i, i + d / 2)), v as it is; one rounding.
template <typename T>
__global__ void __launch_bounds__(256) rope_rows_kernel(const float* __restrict__ in, const float2* __restrict__ cs, int heads_rot,
                                                        int heads, int d, T* __restrict__ out) {
  const int half = d / 2, row = blockIdx.y;
  const size_t base = (size_t)row * heads * d;
  for (int i = blockIdx.x * 256 + threadIdx.x; i < heads * half; i += gridDim.x * 256) {
    const int h = i / half, j = i - h * half;
    const float a = in[base + (size_t)h * d + j], b = in[base + (size_t)h * d + half + j];
    float2 r = make_float2(1.f, 0.f);
    if (h < heads_rot) r = cs[(size_t)row * half + j];
    out[base + (size_t)h * d + j] = from_f32<T>(a * r.x - b * r.y);
    out[base + (size_t)h * d + half + j] = from_f32<T>(b * r.x + a * r.y);
  }
}

}  // namespace

spts_status launch_embed_rows(spts_ctx* ctx, const void* embed, const int32_t* token, int n, void* x) {
  const auto& d = ctx->desc;
  if (d.dtype == SPTS_BF16)
    embed_rows_kernel<bf16><<<n, 256, 0, ctx->stream>>>((const bf16*)embed, token, d.vocab, d.hidden, (bf16*)x, ctx->ws.status);
  else
    embed_rows_kernel<float><<<n, 256, 0, ctx->stream>>>((const float*)embed, token, d.vocab, d.hidden, (float*)x, ctx->ws.status);
  SPTS_CUDA_OK(ctx);
  return SPTS_OK;
}

spts_status launch_rope_rows(spts_ctx* ctx, const float* in, const float2* cs, int n, void* out) {
  const auto& d = ctx->desc;
  const int heads = d.n_q_heads + 2 * d.n_kv_heads, rot = d.n_q_heads + d.n_kv_heads;
  const dim3 grid(ceil_div(heads * d.head_dim / 2, 256), n);
  if (d.dtype == SPTS_BF16) rope_rows_kernel<bf16><<<grid, 256, 0, ctx->stream>>>(in, cs, rot, heads, d.head_dim, (bf16*)out);
  else rope_rows_kernel<float><<<grid, 256, 0, ctx->stream>>>(in, cs, rot, heads, d.head_dim, (float*)out);
  SPTS_CUDA_OK(ctx);
  return SPTS_OK;
}

}  // namespace spts
