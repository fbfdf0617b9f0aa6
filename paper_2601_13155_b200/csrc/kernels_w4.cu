// Matrix-vector products with 4-bit weights (value = scale * (code - 8) + mid per group along the input axis) and the
// quantiser that fills them.
//
// w4_gemv_kernel (bf16): matrix instructions on the codes; see there.
// w4_gemv_plain_kernel: one warp per output feature, CUDA cores, fp32 arithmetic; a lane takes eight codes (one word)
// per step.  fp32 storage and SPTS_REFERENCE_KERNELS.
#include "q4_common.cuh"

namespace spts {

namespace {

using namespace q4;

template <typename T, int LANES>
__global__ void __launch_bounds__(256)
w4_quantize_kernel(const T* __restrict__ W, long n_words, uint32_t* __restrict__ codes,
                   uint32_t* __restrict__ params, int* status) {
  const long i0 = (long)blockIdx.x * 256 + threadIdx.x, stride = (long)gridDim.x * 256;
  // every lane of a warp takes the same number of steps (the group's shuffles need all of them)
  for (long i = i0; (i & ~31L) < n_words; i += stride) {
    const bool in = i < n_words;                   // whole groups: n_words is a multiple of LANES
    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (in) load8(W + 8 * i, x);
    uint32_t p;
    bool bad;
    const uint32_t w = quantize8<LANES>(W, x, p, nullptr, bad);
    if (in) {
      codes[i] = w;
      if (i % LANES == 0) {
        params[i / LANES] = p;
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

// ---------------------------------------------------------------------------------------------------------------------
// bf16: matrix instructions (m16n8k16, fp32 accumulation).  M = 16 weight rows, N = up to 8 tokens, K = input features, so
// the codes are the A operand and up to eight tokens cost what one does; the instruction's idle columns are what buys the
// cheap decoding (a CUDA-core product needs an fp32 conversion and a multiply-add per weight, here two codes become two
// bf16 with one shift and one logic operation, and 256 weights meet the tokens in one instruction).
//   y = sum_groups scale_g sum_i (16 + c_i) x_i + (mid_g - 24 scale_g) sum_i x_i
// The sums of x come from a matrix step with A = 1 over the B fragments that are loaded anyway.
//
// A CTA's eight warps split the input axis in chunks of 128 (warp w takes chunks w, w + 8, ...: the CTA reads 512 contiguous
// bytes of each row at a time) and meet in shared memory per tile of 16 MT rows; the grid is persistent, and every warp's
// ring of asynchronous copies runs on across tiles, so the memory system never drains at a tile's end.
// Order of k inside a 32-block: any order serves a dot product, so lane (g, c) takes the eight consecutive codes 8c .. 8c + 7
// of its row (one word) and the eight consecutive x of its token (one 16-byte load).
template <int J> __device__ __forceinline__ uint32_t code_pair16(uint32_t w) {
  const uint32_t s = J == 0 ? w << 3 : w >> (4 * J - 3);
  return (s & 0x00780078u) | 0x41804180u;
}
constexpr int W4_WARPS = 8;
constexpr int W4_CHUNK = 128;

template <int NB, int MT, int NGC>
struct W4Tile {
  static constexpr int STAGES = NB == 4 ? 3 : 4;
  static constexpr int CSTRIDE = 80;                          // 64 bytes of codes a row; 80: the words of 8 rows x 4 lanes in distinct banks
  static constexpr int PARAMS = 16 * CSTRIDE, SUB = PARAMS + 16 * NGC * 4, STAGE = MT * SUB;
  static constexpr int RING = W4_WARPS * STAGES * STAGE;
  static constexpr int RED = W4_WARPS * NB * MT * 128 * 4;    // [warp][token][row of the tile]
  static constexpr int SMEM = RING + RED;
};

template <int NB, int MT, int NGC, bool TWO>
__global__ void __launch_bounds__(W4_WARPS * 32, 2)
w4_gemv_kernel(const char* __restrict__ codes, const uint32_t* __restrict__ params, const char* __restrict__ codes2,
               const uint32_t* __restrict__ params2, int out, int in, const bf16* __restrict__ X, int64_t ldx, int n, int norm,
               float eps, W4Out o) {
  using T = W4Tile<NB, MT, NGC>;
  constexpr int ROWS = TWO ? 8 * MT : 16 * MT;                // output features of a tile
  constexpr int GT = 4 / NGC;                                 // 32-blocks of a group
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ float sm_ss[W4_WARPS][8 * NB];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, cc = lane & 3;
  const int chunks = (in + W4_CHUNK - 1) / W4_CHUNK, tiles = (out + ROWS - 1) / ROWS, groups = in / (128 / NGC);
  const size_t row_bytes = in / 2;
  float* red = reinterpret_cast<float*>(smem + T::RING);
  unsigned char* ring = smem + warp * (T::STAGES * T::STAGE);
  const uint32_t ring_s = (uint32_t)__cvta_generic_to_shared(ring);

  auto fetch = [&](int tile, int chunk, int stage) {
    const uint32_t dst = ring_s + stage * T::STAGE;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      const bool second = TWO && mt >= MT / 2;
      const int r0 = tile * ROWS + 16 * (second ? mt - MT / 2 : mt);
      const char* cp = second ? codes2 : codes;
      const uint32_t* pp = second ? params2 : params;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int row = min(r0 + 8 * i + g, out - 1);
        if (chunk * W4_CHUNK + 32 * cc < in)                  // codes behind the end meet x = 0: any bits are finite numbers
          cp_async16(dst + mt * T::SUB + (8 * i + g) * T::CSTRIDE + 16 * cc, cp + row * row_bytes + chunk * 64 + 16 * cc);
      }
#pragma unroll
      for (int i = lane; i < 16 * NGC; i += 32) {
        const int row = min(r0 + i / NGC, out - 1), gr = chunk * NGC + i % NGC;
        cp_async4(dst + mt * T::SUB + T::PARAMS + 4 * i, pp + (size_t)row * groups + min(gr, groups - 1), gr < groups);
      }
    }
  };
  int ft = blockIdx.x, fc = warp, fetch_stage = 0, use_stage = 0;          // the next chunk to fetch
  auto fetch_next = [&]() {
    if (ft < tiles && fc < chunks) {
      fetch(ft, fc, fetch_stage);
      fc += W4_WARPS;
      if (fc >= chunks) { fc = warp; ft += gridDim.x; }
    }
    cp_async_commit();
    fetch_stage = fetch_stage + 1 == T::STAGES ? 0 : fetch_stage + 1;
  };
#pragma unroll
  for (int i = 0; i < T::STAGES - 1; ++i) fetch_next();

  bool first = true;
  for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    float y[NB][MT][4], ss[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      ss[nb] = 0.f;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int i = 0; i < 4; ++i) y[nb][mt][i] = 0.f;
    }
    for (int chunk = warp; chunk < chunks; chunk += W4_WARPS) {
      uint4 xw[NB][4];                                        // the tokens' x as they lie in memory
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const int k = chunk * W4_CHUNK + 32 * t + 8 * cc;
          xw[nb][t] = make_uint4(0u, 0u, 0u, 0u);
          if (8 * nb + g < n && k < in) xw[nb][t] = __ldg(reinterpret_cast<const uint4*>(X + (size_t)(8 * nb + g) * ldx + k));
        }
      fetch_next();
      cp_async_wait<T::STAGES - 1>();
      __syncwarp();
      const unsigned char* st = ring + use_stage * T::STAGE;
      use_stage = use_stage + 1 == T::STAGES ? 0 : use_stage + 1;
#pragma unroll
      for (int gr = 0; gr < NGC; ++gr) {
        float acc[NB][MT][4], xs[NB][4];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            xs[nb][i] = 0.f;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) acc[nb][mt][i] = 0.f;
          }
#pragma unroll
        for (int tt = 0; tt < GT; ++tt) {
          const int t = gr * GT + tt;
          uint32_t b[NB][4];                                  // pairs (x_j, x_j+4)
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            const uint4 v = xw[nb][t];
            b[nb][0] = __byte_perm(v.x, v.z, 0x5410); b[nb][1] = __byte_perm(v.x, v.z, 0x7632);
            b[nb][2] = __byte_perm(v.y, v.w, 0x5410); b[nb][3] = __byte_perm(v.y, v.w, 0x7632);
            mma16816(xs[nb], 0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u, b[nb][0], b[nb][1]);
            mma16816(xs[nb], 0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u, b[nb][2], b[nb][3]);
            if (first && norm) {
              const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
              for (int i = 0; i < 4; ++i) { ss[nb] = fmaf(lo_bf16(w[i]), lo_bf16(w[i]), ss[nb]); ss[nb] = fmaf(hi_bf16(w[i]), hi_bf16(w[i]), ss[nb]); }
            }
          }
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            const unsigned char* base = st + mt * T::SUB + 16 * t + 4 * cc;
            const uint32_t w0 = *reinterpret_cast<const uint32_t*>(base + g * T::CSTRIDE);
            const uint32_t w1 = *reinterpret_cast<const uint32_t*>(base + (g + 8) * T::CSTRIDE);
            const uint32_t a0 = code_pair16<0>(w0), a1 = code_pair16<0>(w1), a2 = code_pair16<1>(w0), a3 = code_pair16<1>(w1);
            const uint32_t c0 = code_pair16<2>(w0), c1 = code_pair16<2>(w1), c2 = code_pair16<3>(w0), c3 = code_pair16<3>(w1);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
              mma16816(acc[nb][mt], a0, a1, a2, a3, b[nb][0], b[nb][1]);
              mma16816(acc[nb][mt], c0, c1, c2, c3, b[nb][2], b[nb][3]);
            }
          }
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          const uint32_t* pw = reinterpret_cast<const uint32_t*>(st + mt * T::SUB + T::PARAMS) + gr;
          const uint32_t p0 = pw[g * NGC], p1 = pw[(g + 8) * NGC];
          const float s0 = lo_bf16(p0), s1 = lo_bf16(p1);
          const float m0 = fmaf(-24.f, s0, hi_bf16(p0)), m1 = fmaf(-24.f, s1, hi_bf16(p1));
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              y[nb][mt][i] = fmaf(m0, xs[nb][i], fmaf(s0, acc[nb][mt][i], y[nb][mt][i]));
              y[nb][mt][2 + i] = fmaf(m1, xs[nb][i], fmaf(s1, acc[nb][mt][2 + i], y[nb][mt][2 + i]));
            }
        }
      }
      __syncwarp();                                           // the stage may be filled again
    }
    // ---- the warps' shares meet: red[warp][token][mt][row]
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float* r = red + ((size_t)(warp * 8 * NB + 8 * nb + 2 * cc + i) * MT + mt) * 16 + g;
          r[0] = y[nb][mt][i];
          r[8] = y[nb][mt][2 + i];
        }
    if (first && norm) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        float s = ss[nb];
        s += __shfl_xor_sync(0xffffffffu, s, 1);
        s += __shfl_xor_sync(0xffffffffu, s, 2);
        if (cc == 0) sm_ss[warp][8 * nb + g] = s;
      }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n * ROWS; i += W4_WARPS * 32) {
      const int t = i / ROWS, r = i - t * ROWS, row = tile * ROWS + r;
      if (row < out) {
        float v = 0.f, v2 = 0.f, q = 0.f;
#pragma unroll
        for (int w = 0; w < W4_WARPS; ++w) {
          v += red[(size_t)(w * 8 * NB + t) * MT * 16 + r];
          if (TWO) v2 += red[(size_t)(w * 8 * NB + t) * MT * 16 + ROWS + r];
          if (norm) q += sm_ss[w][t];
        }
        if (norm) {
          const float rs = 1.0f / sqrtf(q / (float)in + eps);
          v *= rs;
          v2 *= rs;
        }
        w4_store<bf16>(o, t, row, TWO ? silu_mul(v, v2) : v);
      }
    }
    first = false;
    __syncthreads();
  }
  cp_async_wait<0>();
}

template <int NB, int MT, int NGC, bool TWO>
spts_status launch_tile(spts_ctx* ctx, const W4GemvArgs& a) {
  using T = W4Tile<NB, MT, NGC>;
  const W4Out o{a.residual, a.ldr, a.Y, a.ldy, a.fp32_out};
  const int tiles = ceil_div(a.out, TWO ? 8 * MT : 16 * MT);
  const int grid = tiles < 2 * ctx->sm_count ? tiles : 2 * ctx->sm_count;
  if (cudaFuncSetAttribute(w4_gemv_kernel<NB, MT, NGC, TWO>, cudaFuncAttributeMaxDynamicSharedMemorySize, T::SMEM) != cudaSuccess)
    return SPTS_ERR_CUDA;
  w4_gemv_kernel<NB, MT, NGC, TWO><<<grid, W4_WARPS * 32, T::SMEM, ctx->stream>>>(
      (const char*)a.codes, (const uint32_t*)a.params, (const char*)a.codes2, (const uint32_t*)a.params2, a.out, a.in,
      (const bf16*)a.X, a.ldx, a.n, a.norm, ctx->desc.rms_eps, o);
  SPTS_CUDA_OK(ctx);
  return SPTS_OK;
}
template <int NB, int NGC>
spts_status launch_rows(spts_ctx* ctx, const W4GemvArgs& a) {
  if (a.codes2 != nullptr) return launch_tile<NB, 2, NGC, true>(ctx, a);
  return ceil_div(a.out, 32) >= 2 * ctx->sm_count ? launch_tile<NB, 2, NGC, false>(ctx, a) : launch_tile<NB, 1, NGC, false>(ctx, a);
}
template <int NB>
spts_status launch_group(spts_ctx* ctx, const W4GemvArgs& a) {
  if (a.group == 128) return launch_rows<NB, 1>(ctx, a);
  return a.group == 64 ? launch_rows<NB, 2>(ctx, a) : launch_rows<NB, 4>(ctx, a);
}

}  // namespace

spts_status launch_w4_gemv(spts_ctx* ctx, const W4GemvArgs& a) {
  if (!plain4(ctx)) return a.n <= 8 ? launch_group<1>(ctx, a) : a.n <= 16 ? launch_group<2>(ctx, a) : launch_group<4>(ctx, a);
  if (ctx->desc.dtype == SPTS_FP32) return a.n == 1 ? launch_plain<float, 1>(ctx, a) : launch_plain<float, 4>(ctx, a);
  return a.n == 1 ? launch_plain<bf16, 1>(ctx, a) : launch_plain<bf16, 4>(ctx, a);
}

template <typename T>
static void quantize_t(spts_ctx* ctx, const void* W, long n_words, int blocks, int group, void* codes, void* params) {
  void (*kernel)(const T*, long, uint32_t*, uint32_t*, int*) =
      group == 32 ? w4_quantize_kernel<T, 4> : group == 64 ? w4_quantize_kernel<T, 8> : w4_quantize_kernel<T, 16>;
  kernel<<<blocks, 256, 0, ctx->stream>>>((const T*)W, n_words, (uint32_t*)codes, (uint32_t*)params, ctx->ws.status);
}

spts_status launch_w4_quantize(spts_ctx* ctx, const void* W, int out, int in, int group, void* codes, void* params) {
  const long n_words = (long)out * (in / 8);
  long blocks = (n_words + 255) / 256;
  if (blocks > 16L * ctx->sm_count) blocks = 16L * ctx->sm_count;
  if (ctx->desc.dtype == SPTS_BF16) quantize_t<bf16>(ctx, W, n_words, (int)blocks, group, codes, params);
  else quantize_t<float>(ctx, W, n_words, (int)blocks, group, codes, params);
  SPTS_CUDA_OK(ctx);
  return SPTS_OK;
}

}  // namespace spts
