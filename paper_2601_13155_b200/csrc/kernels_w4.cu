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
// bf16: matrix instructions (m16n8k16, fp32 accumulation).  M = 16 weight rows, N = up to 8 NB tokens, K = input features, so
// the codes are the A operand and up to eight tokens cost what one does.  What bounds the kernel beside memory is the
// instructions between the codes and the matrix units, so they are few: codes enter as fp16 by masks alone (code_pair), eight
// codes for five instructions, and
//   y = sum_groups scale_g sum_i c_i x_i + sum_g (mid_g - 8 scale_g) (sum_i x_i)
// has its second part in one more matrix step per four groups, in bf16, whose A registers are the params words as they lie in
// memory and whose B holds -8 sum x and sum x in bf16 pieces (two of them, 2^-17 relative; three for fp32 outputs).
//
// x is laid out for that once per call by w4_prepare_kernel (a CTA per token): brought to fp16 by a power of two (exact: bf16
// has fewer bits, and what falls below fp16's range is 2^-35 of the token's largest element), in the order of the B fragments,
// with the groups' sums and the factor that takes the power of two back (and the row norm with it).  The product kernel is its
// programmatic dependent: it fills its rings with weights while x is prepared.
//
// Work split.  A warp takes 16 MT rows (gate and up rows alternating in MT when there are two matrices).  With at most eight
// tokens the WK = 8 warps of a CTA split the input axis in chunks of 128 (the CTA reads 512 contiguous bytes of each row at a
// time); with more, x is what is read most, so the warps take different rows and the same chunks (WK = 1), and seven of eight
// reads of x hit L1.  Where that leaves SMs without work, the input axis is also cut between CTAs (`slices`), and the CTA that
// arrives last adds their shares in order.  The grid is persistent, and every warp's ring of asynchronous copies runs on across
// tiles.
constexpr int W4_WARPS = 8;
constexpr int W4_CHUNK = 128;

// The order of k inside a chunk: step t of the chunk's four, lane c, eight consecutive codes (one word).  A lane's words lie
// side by side within a group, so that they are one shared-memory load.
template <int NGC> __host__ __device__ constexpr int w4_k(int t, int c) {
  return NGC == 1 ? 32 * c + 8 * t : NGC == 2 ? 64 * (t >> 1) + 16 * c + 8 * (t & 1) : 32 * t + 8 * c;
}

// x [n, in] -> frag [chunk][t][tokens][c] (16 bytes: four fp16 pairs), sums [chunk][tokens][c] (three pairs of pieces), factor [n]
template <int NGC>
__global__ void __launch_bounds__(512)
w4_prepare_kernel(const bf16* __restrict__ X, int64_t ldx, int in, int tokens, int norm, float eps, uint4* __restrict__ frag,
                  uint4* __restrict__ sums, float* __restrict__ factor) {
  __shared__ float red[2][16];
  const int token = blockIdx.x, tid = threadIdx.x, lane = tid & 31;
  const bf16* x = X + (size_t)token * ldx;
  dep_launch();
  float top = 0.f, ss = 0.f;
  for (int k = 8 * tid; k < in; k += 8 * 512) {
    float v[8];
    load8(x + k, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) { top = fmaxf(top, fabsf(v[i])); ss = fmaf(v[i], v[i], ss); }
  }
  top = warp_max(top);
  ss = warp_sum(ss);
  if (lane == 0) { red[0][tid >> 5] = top; red[1][tid >> 5] = ss; }
  __syncthreads();
  top = red[0][0]; ss = red[1][0];
#pragma unroll
  for (int w = 1; w < 16; ++w) { top = fmaxf(top, red[0][w]); ss += red[1][w]; }
  const float xs = scale_to_2_13(top), u = xs * CODE_UNIT;
  if (tid == 0) factor[token] = (norm ? 1.0f / sqrtf(ss / (float)in + eps) : 1.0f) / u;
  const int chunks = (in + W4_CHUNK - 1) / W4_CHUNK, total = chunks * 16;
  for (int i0 = tid & ~31; i0 < total; i0 += 512) {
    const int i = i0 + lane, chunk = i >> 4, t = (i >> 2) & 3, c = i & 3;
    const int k = chunk * W4_CHUNK + w4_k<NGC>(t, c);
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (i < total && k < in) load8(x + k, v);
    float s = ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
    if (i < total) {
      const float xo = xs * ODD;
      frag[((size_t)(chunk * 4 + t) * tokens + token) * 4 + c] =
          make_uint4(pack2_f16(v[0] * xs, v[4] * xs), pack2_f16(v[1] * xo, v[5] * xo), pack2_f16(v[2] * xs, v[6] * xs),
                     pack2_f16(v[3] * xo, v[7] * xo));
    }
    constexpr int LANES = 16 / NGC;                // that hold a group
#pragma unroll
    for (int o = 1; o < LANES; o <<= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (i < total && i % LANES == 0) {
      const float sm = s * u, a = -8.f * sm;
      const float ah = round_bf16(a), mh = round_bf16(sm), am = round_bf16(a - ah), mm = round_bf16(sm - mh);
      sums[((size_t)chunk * tokens + token) * 4 + (i % 16) / LANES] =
          make_uint4(pack2(ah, mh), pack2(am, mm), pack2((a - ah) - am, (sm - mh) - mm), 0u);
    }
  }
}

template <int NB, int MT, int NGC, int WK>
struct W4Tile {
  static constexpr int WR = W4_WARPS / WK;
  static constexpr int STAGES = 4;
  static constexpr int CSTRIDE = NGC == 1 ? 64 : NGC == 2 ? 96 : 80;      // bytes between rows: a load's lanes lie in distinct banks
  static constexpr int PARAMS = 16 * MT * CSTRIDE, STAGE = PARAMS + 16 * MT * NGC * 4;
  static constexpr int RING = W4_WARPS * STAGES * STAGE;
  static constexpr int RED = WK * 8 * NB * WR * MT * 16 * 4;              // [wk][token][wr][mt][row]
  static constexpr int SMEM = RING + RED;
};

struct W4Mat { const char* codes; const uint32_t* params; };

template <int NB, int MT, int NGC, bool TWO, int WK>
__global__ void __launch_bounds__(W4_WARPS * 32, 2)
w4_gemv_kernel(W4Mat m1, W4Mat m2, int out, int in, int n, int slices, const uint4* __restrict__ frag, const uint4* __restrict__ sums,
               const float* __restrict__ factor, float* __restrict__ part, int* __restrict__ arrived, W4Out o) {
  using T = W4Tile<NB, MT, NGC, WK>;
  constexpr int WR = T::WR, WROWS = TWO ? 8 * MT : 16 * MT, ROWS = WR * WROWS;      // output features of a warp, of a tile
  constexpr int TOKENS = 8 * NB, RSTRIDE = WR * MT * 16;
  constexpr int GT = 4 / NGC;                                 // steps of a group
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ int last_flag;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, cc = lane & 3;
  const int wk = warp % WK, wr = warp / WK;
  const int chunks = (in + W4_CHUNK - 1) / W4_CHUNK, tiles = (out + ROWS - 1) / ROWS, groups = in / (128 / NGC);
  const int items = tiles * slices;
  const size_t row_bytes = in / 2;
  float* red = reinterpret_cast<float*>(smem + T::RING);
  unsigned char* ring = smem + warp * (T::STAGES * T::STAGE);
  const uint32_t ring_s = (uint32_t)__cvta_generic_to_shared(ring);
  const bool whole = groups % NGC == 0;                       // every chunk is: a row's params of a chunk are one copy

  // the walk of the copies: item, chunk, the warp's row pointers in that item
  int f_item = blockIdx.x, f_chunk = 0, f_end = 0;
  const char* f_codes[MT][2];
  const uint32_t* f_params = nullptr;                         // lane r: row r of the warp's 16 MT rows
  uint32_t fetch_at = 0, use_at = 0;
  auto f_open = [&]() {                                       // settles on the next item in which this warp has a chunk
    for (; f_item < items; f_item += gridDim.x) {
      const int tile = f_item / slices, slice = f_item - tile * slices;
      f_chunk = (int)((long)chunks * slice / slices) + wk;
      f_end = (int)((long)chunks * (slice + 1) / slices);
      if (f_chunk >= f_end) continue;
      const int r0 = tile * ROWS + wr * WROWS;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        const bool second = TWO && (mt & 1);
        const W4Mat& m = second ? m2 : m1;
        const int rm = r0 + 16 * (TWO ? mt >> 1 : mt);
#pragma unroll
        for (int i = 0; i < 2; ++i) f_codes[mt][i] = m.codes + min(rm + 8 * i + g, out - 1) * row_bytes + (size_t)f_chunk * 64 + 16 * cc;
      }
      const int mt = lane >> 4;
      const bool second = TWO && (mt & 1);
      f_params = (second ? m2.params : m1.params) + (size_t)min(r0 + 16 * (TWO ? mt >> 1 : mt) + (lane & 15), out - 1) * groups;
      return;
    }
  };
  f_open();
  auto fetch_next = [&]() {
    if (f_item < items) {
      const uint32_t dst = ring_s + fetch_at;
      if (f_chunk * W4_CHUNK + 32 * cc < in) {                // codes behind the end meet x = 0: any bits are finite numbers
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int i = 0; i < 2; ++i) cp_async16(dst + (16 * mt + 8 * i + g) * T::CSTRIDE + 16 * cc, f_codes[mt][i]);
      }
      if (lane < 16 * MT) {
        const uint32_t* p = f_params + f_chunk * NGC;
        const uint32_t pd = dst + T::PARAMS + lane * NGC * 4;
        if (NGC == 4 && whole) cp_async16(pd, p);
        else if (NGC == 2 && whole) cp_async8(pd, p);
        else {
#pragma unroll
          for (int i = 0; i < NGC; ++i) {
            const bool has = f_chunk * NGC + i < groups;
            cp_async4(pd + 4 * i, has ? p + i : f_params, has);
          }
        }
      }
      f_chunk += WK;
      if (f_chunk < f_end) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int i = 0; i < 2; ++i) f_codes[mt][i] += 64 * WK;
      } else {
        f_item += gridDim.x;
        f_open();
      }
    }
    cp_async_commit();
    fetch_at = fetch_at + T::STAGE == T::STAGES * T::STAGE ? 0 : fetch_at + T::STAGE;
  };
#pragma unroll
  for (int i = 0; i < T::STAGES - 1; ++i) fetch_next();
  dep_wait();                                                 // x is prepared

  for (int item = blockIdx.x; item < items; item += gridDim.x) {
    const int tile = item / slices, slice = item - tile * slices;
    const int c1 = (int)((long)chunks * (slice + 1) / slices);
    float y[NB][MT][4];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int i = 0; i < 4; ++i) y[nb][mt][i] = 0.f;
    for (int chunk = (int)((long)chunks * slice / slices) + wk; chunk < c1; chunk += WK) {
      uint4 xf[NB][4], xs[NB];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const bool has = 8 * nb + g < n;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          xf[nb][t] = make_uint4(0u, 0u, 0u, 0u);
          if (has) xf[nb][t] = __ldg(frag + ((size_t)(chunk * 4 + t) * TOKENS + 8 * nb + g) * 4 + cc);
        }
        xs[nb] = make_uint4(0u, 0u, 0u, 0u);
        if (has && cc < NGC) xs[nb] = __ldg(sums + ((size_t)chunk * TOKENS + 8 * nb + g) * 4 + cc);
      }
      fetch_next();
      cp_async_wait<T::STAGES - 1>();
      __syncwarp();
      const unsigned char* st = ring + use_at;
      use_at = use_at + T::STAGE == T::STAGES * T::STAGE ? 0 : use_at + T::STAGE;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        const unsigned char* row0 = st + (16 * mt + g) * T::CSTRIDE;
        const unsigned char* row1 = row0 + 8 * T::CSTRIDE;
        const unsigned char* prm0 = st + T::PARAMS + (16 * mt + g) * NGC * 4;
        const unsigned char* prm1 = prm0 + 8 * NGC * 4;
        {
          uint32_t p0 = 0u, p1 = 0u;
          if (cc < NGC) { p0 = *reinterpret_cast<const uint32_t*>(prm0 + 4 * cc); p1 = *reinterpret_cast<const uint32_t*>(prm1 + 4 * cc); }
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            mma16816(y[nb][mt], p0, p1, p0, p1, xs[nb].x, xs[nb].y);
            if (o.fp32_out) mma16816(y[nb][mt], p0, p1, 0u, 0u, xs[nb].z, 0u);
          }
        }
        uint32_t w0[4], w1[4], q0[NGC], q1[NGC];
        load_words<NGC>(prm0, q0);
        load_words<NGC>(prm1, q1);
#pragma unroll
        for (int gr = 0; gr < NGC; ++gr) {
          load_words<GT>(row0 + (64 / NGC) * gr + 4 * GT * cc, *reinterpret_cast<uint32_t (*)[GT]>(w0 + gr * GT));
          load_words<GT>(row1 + (64 / NGC) * gr + 4 * GT * cc, *reinterpret_cast<uint32_t (*)[GT]>(w1 + gr * GT));
        }
#pragma unroll
        for (int gr = 0; gr < NGC; ++gr) {
          float acc[NB][4];
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[nb][i] = 0.f;
#pragma unroll
          for (int tt = 0; tt < GT; ++tt) {
            const int t = gr * GT + tt;
            const uint32_t a0 = code_pair<0>(w0[t]), a1 = code_pair<0>(w1[t]), a2 = code_pair<1>(w0[t]), a3 = code_pair<1>(w1[t]);
            const uint32_t b0 = code_pair<2>(w0[t]), b1 = code_pair<2>(w1[t]), b2 = code_pair<3>(w0[t]), b3 = code_pair<3>(w1[t]);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
              mma_f16(acc[nb], a0, a1, a2, a3, xf[nb][t].x, xf[nb][t].y);
              mma_f16(acc[nb], b0, b1, b2, b3, xf[nb][t].z, xf[nb][t].w);
            }
          }
          const float s0 = lo_bf16(q0[gr]), s1 = lo_bf16(q1[gr]);
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            y[nb][mt][0] = fmaf(s0, acc[nb][0], y[nb][mt][0]); y[nb][mt][1] = fmaf(s0, acc[nb][1], y[nb][mt][1]);
            y[nb][mt][2] = fmaf(s1, acc[nb][2], y[nb][mt][2]); y[nb][mt][3] = fmaf(s1, acc[nb][3], y[nb][mt][3]);
          }
        }
      }
      __syncwarp();                                           // the stage may be filled again
    }
    // ---- the warps' shares meet: red[wk][token][wr][mt][row]
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int token = 8 * nb + 2 * cc + i;
        if (token < n) {
          float* r = red + (size_t)(wk * TOKENS + token) * RSTRIDE + wr * MT * 16 + g;
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) { r[16 * mt] = y[nb][mt][i]; r[16 * mt + 8] = y[nb][mt][2 + i]; }
        }
      }
    __syncthreads();
    auto sum_wk = [&](int t, int r) {
      float v = 0.f;
#pragma unroll
      for (int w = 0; w < WK; ++w) v += red[(size_t)(w * TOKENS + t) * RSTRIDE + r];
      return v;
    };
    bool finish = true;
    if (slices > 1) {
      float* mine = part + (size_t)item * TOKENS * RSTRIDE;
      for (int i = threadIdx.x; i < n * RSTRIDE; i += W4_WARPS * 32) mine[i] = sum_wk(i / RSTRIDE, i % RSTRIDE);
      __threadfence();
      __syncthreads();
      if (threadIdx.x == 0) last_flag = atomicAdd(&arrived[tile], 1) == slices - 1;
      __syncthreads();
      finish = last_flag;
      if (finish) {
        __threadfence();
        if (threadIdx.x == 0) arrived[tile] = 0;              // for the next call
      }
    }
    if (finish) {
      for (int i = threadIdx.x; i < n * ROWS; i += W4_WARPS * 32) {
        const int t = i / ROWS, r = i - t * ROWS, row = tile * ROWS + r;
        if (row >= out) continue;
        // where the row's value lies: the warp's, then its tile of 16 (with two matrices gate and up tiles alternate)
        const int w = r / WROWS, rw = r - w * WROWS, at = w * MT * 16 + (TWO ? (rw >> 4) * 32 + (rw & 15) : rw);
        float v = 0.f, v2 = 0.f;
        if (slices == 1) {
          v = sum_wk(t, at);
          if (TWO) v2 = sum_wk(t, at + 16);
        } else {
          const float* p = part + (size_t)tile * slices * TOKENS * RSTRIDE + (size_t)t * RSTRIDE + at;
#pragma unroll 4
          for (int s = 0; s < slices; ++s) {
            v += __ldcg(p + (size_t)s * TOKENS * RSTRIDE);
            if (TWO) v2 += __ldcg(p + (size_t)s * TOKENS * RSTRIDE + 16);
          }
        }
        const float f = __ldg(factor + t);
        v *= f;
        w4_store<bf16>(o, t, row, TWO ? silu_mul(v, v2 * f) : v);
      }
    }
    __syncthreads();
  }
  cp_async_wait<0>();
}

template <int NB, int MT, int NGC, bool TWO, int WK>
spts_status launch_tile(spts_ctx* ctx, const W4GemvArgs& a) {
  using T = W4Tile<NB, MT, NGC, WK>;
  const W4Out o{a.residual, a.ldr, a.Y, a.ldy, a.fp32_out};
  const int rows = T::WR * (TWO ? 8 * MT : 16 * MT), tiles = ceil_div(a.out, rows), chunks = ceil_div(a.in, W4_CHUNK);
  const int most = 2 * ctx->sm_count < W4_MAX_ITEMS ? 2 * ctx->sm_count : W4_MAX_ITEMS;
  // the input axis is cut where there are fewer tiles than SMs, to two CTAs per SM but not below one chunk per warp
  int slices = tiles < ctx->sm_count ? most / tiles : 1;
  if (slices > chunks / WK) slices = chunks / WK > 1 ? chunks / WK : 1;
  const int grid = tiles * slices < most ? tiles * slices : most;
  uint4* frag = (uint4*)ctx->ws.w4_x;
  uint4* sums = frag + (size_t)chunks * 16 * 8 * NB;
  float* factor = (float*)(sums + (size_t)chunks * 4 * 8 * NB);
  w4_prepare_kernel<NGC><<<a.n, 512, 0, ctx->stream>>>((const bf16*)a.X, a.ldx, a.in, 8 * NB, a.norm, ctx->desc.rms_eps, frag, sums, factor);
  SPTS_CUDA_OK(ctx);
  auto kernel = w4_gemv_kernel<NB, MT, NGC, TWO, WK>;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, T::SMEM) != cudaSuccess) return SPTS_ERR_CUDA;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(W4_WARPS * 32);
  cfg.dynamicSmemBytes = T::SMEM;
  cfg.stream = ctx->stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, kernel, W4Mat{(const char*)a.codes, (const uint32_t*)a.params},
                         W4Mat{(const char*)a.codes2, (const uint32_t*)a.params2}, a.out, a.in, a.n, slices, (const uint4*)frag,
                         (const uint4*)sums, (const float*)factor, ctx->ws.w4_part, ctx->ws.w4_arrived, o) != cudaSuccess)
    return SPTS_ERR_CUDA;
  SPTS_CUDA_OK(ctx);
  return SPTS_OK;
}
template <int NB, int NGC>
spts_status launch_rows(spts_ctx* ctx, const W4GemvArgs& a) {
  constexpr int WK = NB == 1 ? 8 : 1;
  if (a.codes2 != nullptr) return launch_tile<NB, 2, NGC, true, WK>(ctx, a);
  // one tile of 16 rows to a warp where two would leave SMs without a CTA
  if (NB == 1 && ceil_div(a.out, 32) < 2 * ctx->sm_count) return launch_tile<NB, NB == 1 ? 1 : 2, NGC, false, WK>(ctx, a);
  return launch_tile<NB, 2, NGC, false, WK>(ctx, a);
}
template <int NB>
spts_status launch_group(spts_ctx* ctx, const W4GemvArgs& a) {
  if (a.group == 128) return launch_rows<NB, 1>(ctx, a);
  return a.group == 64 ? launch_rows<NB, 2>(ctx, a) : launch_rows<NB, 4>(ctx, a);
}

}  // namespace

spts_status launch_w4_gemv(spts_ctx* ctx, const W4GemvArgs& all) {
  if (plain4(ctx)) {
    if (ctx->desc.dtype == SPTS_FP32) return all.n == 1 ? launch_plain<float, 1>(ctx, all) : launch_plain<float, 4>(ctx, all);
    return all.n == 1 ? launch_plain<bf16, 1>(ctx, all) : launch_plain<bf16, 4>(ctx, all);
  }
  // as many tokens at a time as the workspace holds in their prepared form (all of them up to 32768 features)
  const int padded = (int)align_up((size_t)all.in, W4_CHUNK);
  const int at_a_time = 8 * (int)(W4_X_ELEMENTS / 8 / padded) < SPTS_W4_MAX_N ? 8 * (int)(W4_X_ELEMENTS / 8 / padded) : SPTS_W4_MAX_N;
  const size_t es = 2, eo = all.fp32_out ? 4 : 2;
  for (int t0 = 0; t0 < all.n; t0 += at_a_time) {
    W4GemvArgs a = all;
    a.n = all.n - t0 < at_a_time ? all.n - t0 : at_a_time;
    a.X = (const char*)all.X + (size_t)t0 * all.ldx * es;
    if (all.residual != nullptr) a.residual = (const char*)all.residual + (size_t)t0 * all.ldr * es;
    a.Y = (char*)all.Y + (size_t)t0 * all.ldy * eo;
    spts_status s = a.n <= 8 ? launch_group<1>(ctx, a) : a.n <= 16 ? launch_group<2>(ctx, a) : a.n <= 24 ? launch_group<3>(ctx, a)
                                                                                               : launch_group<4>(ctx, a);
    if (s != SPTS_OK) return s;
  }
  return SPTS_OK;
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
