// Matrix-vector products with 4-bit weights (value = scale * (code - 8) + mid per group along the input axis) and the
// quantiser that fills them.
//
// w4_gemv_kernel (bf16): matrix instructions on the codes; see there.
// w4_gemv_plain_kernel: one or two output features per warp, CUDA cores, fp32 arithmetic; a lane takes eight codes (one word)
// per step.  Bound by its instructions (five for every code) and the latency of its loads: one token, 14336 x 4096: 28 us (the matrix
// kernel: 11).  fp32 storage and SPTS_REFERENCE_KERNELS.
#include "q4_common.cuh"

namespace spts {

namespace {

using namespace q4;

// Eight elements to a lane, a group to LANES neighbouring lanes (quantize8).  14336 x 4096 in bf16: 70 us, 2.1 TB/s (in fp32 64 us,
// 4.1 TB/s), bound by its instructions as the append is, at six blocks to an SM (72 us; five 76, four 78).
template <typename T, int LANES>
__global__ void __launch_bounds__(256, 6)
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

// R features to a warp, which share its loads of x, and up to NT tokens, which share the decoded weights
template <typename T, int NT, bool TWO, int R>
__global__ void __launch_bounds__(256)
w4_gemv_plain_kernel(const uint32_t* __restrict__ codes, const uint32_t* __restrict__ params,
                     const uint32_t* __restrict__ codes2, const uint32_t* __restrict__ params2, int out, int in, int group,
                     const T* __restrict__ X, int64_t ldx, int n, int norm, float eps, W4Out o) {
  constexpr int M = TWO ? 2 : 1;
  const int row0 = (blockIdx.x * 8 + (threadIdx.x >> 5)) * R, lane = threadIdx.x & 31;
  if (row0 >= out) return;
  const int t0 = blockIdx.y * NT;
  const int words = in / 8, groups = in / group, shift = group == 32 ? 2 : group == 64 ? 3 : 4;       // words to a group
  float acc[R][M][NT], ss[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    ss[t] = 0.f;
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int m = 0; m < M; ++m) acc[r][m][t] = 0.f;
  }
  for (int w = lane; w < words; w += 32) {
    float v[R][M][8];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int m = 0; m < M; ++m) {
        const size_t row = min(row0 + r, out - 1);
        const uint32_t c = (m == 0 ? codes : codes2)[row * words + w], p = (m == 0 ? params : params2)[row * groups + (w >> shift)];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[r][m][i] = fmaf(lo_bf16(p), code_less_8(c, i), hi_bf16(p));
      }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      if (t0 + t < n) {
        float x[8];
        load8(X + (size_t)(t0 + t) * ldx + 8 * w, x);
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int m = 0; m < M; ++m)
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[r][m][t] = fmaf(v[r][m][i], x[i], acc[r][m][t]);
        if (norm) {
#pragma unroll
          for (int i = 0; i < 8; ++i) ss[t] = fmaf(x[i], x[i], ss[t]);
        }
      }
    }
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    if (t0 + t < n) {
      const float s2 = norm ? warp_sum(ss[t]) : 0.f;
      const float rs = norm ? 1.0f / sqrtf(s2 / (float)in + eps) : 1.0f;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float y = warp_sum(acc[r][0][t]) * rs;
        if (TWO) y = silu_mul(y, warp_sum(acc[r][M - 1][t]) * rs);
        if (lane == 0 && row0 + r < out) w4_store<T>(o, t0 + t, row0 + r, y);
      }
    }
  }
}

template <typename T, int NT, bool TWO, int R>
spts_status launch_plain_rows(spts_ctx* ctx, const W4GemvArgs& a) {
  const W4Out o{a.residual, a.ldr, a.Y, a.ldy, a.fp32_out};
  w4_gemv_plain_kernel<T, NT, TWO, R><<<dim3(ceil_div(a.out, 8 * R), ceil_div(a.n, NT)), 256, 0, ctx->stream>>>(
      (const uint32_t*)a.codes, (const uint32_t*)a.params, (const uint32_t*)a.codes2, (const uint32_t*)a.params2, a.out, a.in, a.group,
      (const T*)a.X, a.ldx, a.n, a.norm, ctx->desc.rms_eps, o);
  SPTS_CUDA_OK(ctx);
  return SPTS_OK;
}
template <typename T, int NT>
spts_status launch_plain(spts_ctx* ctx, const W4GemvArgs& a) {
  // four tokens: two features to a warp where that leaves a block for every SM (fp32, 4 x 8192 x 4096: 26 us, one feature 42)
  if constexpr (NT > 1)
    if (ceil_div(a.out, 16) >= ctx->sm_count)
      return a.codes2 != nullptr ? launch_plain_rows<T, NT, true, 2>(ctx, a) : launch_plain_rows<T, NT, false, 2>(ctx, a);
  return a.codes2 != nullptr ? launch_plain_rows<T, NT, true, 1>(ctx, a) : launch_plain_rows<T, NT, false, 1>(ctx, a);
}

// ---------------------------------------------------------------------------------------------------------------------
// bf16: matrix instructions (m16n8k16, fp32 accumulation).  M = 16 weight rows, N = up to 8 NB tokens, K = input features, so
// the codes are the A operand and up to eight tokens cost what one does.  What bounds the kernel beside memory is the
// instructions between the codes and the matrix units, so they are few: codes enter as fp16 by masks alone (code_pair), eight
// codes for five instructions, and
//   y = sum_groups scale_g sum_i c_i x_i + sum_g (mid_g - 8 scale_g) (sum_i x_i)
// has its second part in one more matrix step per four groups, in bf16, whose A registers are the params words as they lie in
// memory and whose B holds -8 sum x and sum x in three bf16 pieces each (2^-26 relative; with two, 2^-17, 0.08 % of the
// bf16 outputs differed from the rounded exact ones; the third costs 2 % of 21 x 3584 x 18944).
//
// x is laid out for that once per call: brought to fp16 by a power of two (exact: bf16 has fewer bits; only elements below 2^-26 of
// the token's largest are rounded, off by up to 2^-34 of it), in the order of the B fragments, with the groups' sums and the factor
// that takes the power of two back (and the row norm with it).  Few elements (LOCAL) every CTA lays out for itself in shared
// memory while its first weights are on their way; more are laid out once by w4_prepare_kernel (a CTA per token), whose
// programmatic dependent the product kernel is: it fills its rings with weights meanwhile.
//
// Work split.  A warp takes 16 MT rows (gate and up rows alternating in MT when there are two matrices), a CTA's WR x WK warps
// a tile of WR such blocks and WK chunks of 256 of the input axis at a time.  The steps (WK chunks of a tile) of all tiles form
// one line that is cut into equal pieces, one per CTA (persistent); a tile that lies in one piece is finished there, of a tile
// cut between CTAs each leaves its share, and w4_join_kernel adds them in the order of the CTAs.  (The CTA that arrives last
// added them at first: one CTA's loads for 21 tokens x 256 rows x 21 shares took 50 us.)  Every warp's ring of asynchronous
// copies runs on across tiles.
//
// Measured: 1 x 128256 x 4096 54 us, 5.5 TB/s of codes and params (a copy's rate asks for 46; deeper rings and three CTAs to an SM were
// slower); 1 x 4096 x 4096 6.3 us (launch, x, one ring's latency); two matrices 8 x 14336 x 4096 19.5 us, of which x's layout
// about 4; 21 x 3584 x 18944 in groups of 32 30 us (the same two launches 4 + 4; the product at two warps per
// scheduler, 800 instructions to 32 rows x 256 features, matrix pipe 37 %).  L1 prefetches of x, three or four stages and two
// CTAs of 128 registers made the last one 2 to 8 % slower.  (The figures beside the rules below were taken, either side, before bf16
// outputs had the sums' third piece.)
constexpr int W4_WARPS = 8;
// 256 features: a row's codes of a chunk are one line of 128 bytes, its params 8 to 32 bytes.  (With chunks of 128 the copies
// spend twice as many line accesses per byte, and the loop's own instructions weigh twice as much.)
constexpr int W4_CHUNK = 256;
constexpr int W4_WK = 4;
// elements of x that a CTA lays out for itself: 2.5 bytes each beside a ring of up to 82 KB, two CTAs to an SM
constexpr int W4_LOCAL = 8192;

// NG groups to a chunk (2, 4 or 8): a lane c holds GT = 8 / NG neighbouring words (of eight codes) of a row's group, one
// shared-memory load; any order of k serves a dot product, so x's fragments follow: step t of the chunk's eight is word t % GT
// of group t / GT.
template <int NG> struct W4Order {
  static constexpr int GT = 8 / NG, LANES = 4 * GT;              // LANES of the layout hold a group
  static constexpr int SUMS = NG < 4 ? 4 : NG;                   // entries of the groups' sums
  static constexpr int BLOCK = 512 + 16 * SUMS;                  // bytes of a token's block
  __host__ __device__ static constexpr int k(int t, int c) { return (t / GT) * (W4_CHUNK / NG) + c * (W4_CHUNK / NG / 4) + 8 * (t % GT); }
};

// x [n, in] -> per chunk and token fragments [t][c] (16 bytes: four fp16 pairs), then sums [group] (three pairs of pieces; zero
// where there is no such group), in rows of 64 bytes `row` apart, tokens `next` and chunks `stride` apart; factor [n].  One token
// (with x null: zeros), by a CTA of THREADS.
template <int NG, int THREADS>
__device__ __forceinline__ void w4_prepare(const bf16* __restrict__ x, int token, int in, int norm, float eps, unsigned char* blocks,
                                           int row, int next, size_t stride, float* factor) {
  using L = W4Order<NG>;
  constexpr int WARPS = THREADS / 32;
  __shared__ float red[2][WARPS];
  const int tid = threadIdx.x, lane = tid & 31;
  float top = 0.f, ss = 0.f;
  const int there = x != nullptr ? in : 0;
  // a warp takes a chunk at a time, lane 4 t + c, and keeps its first ones between the two passes
  constexpr int KEEP = THREADS == 1024 ? 2 : 4;
  const int k0 = (tid >> 5) * W4_CHUNK + L::k(lane >> 2, lane & 3);
  Raw8<bf16> kept[KEEP];
#pragma unroll
  for (int i = 0; i < KEEP; ++i) {
    kept[i].zero();
    if (k0 + i * WARPS * W4_CHUNK < there) kept[i].load(x + k0 + i * WARPS * W4_CHUNK);
  }
  const auto look = [&](const Raw8<bf16>& raw) {
    float v[8];
    raw.get(v);
#pragma unroll
    for (int i = 0; i < 8; ++i) { top = fmaxf(top, fabsf(v[i])); ss = fmaf(v[i], v[i], ss); }
  };
#pragma unroll
  for (int i = 0; i < KEEP; ++i)
    if ((tid >> 5) * W4_CHUNK + i * WARPS * W4_CHUNK < there) look(kept[i]);
  for (int k = k0 + KEEP * WARPS * W4_CHUNK; k < there; k += WARPS * W4_CHUNK) {
    Raw8<bf16> raw;
    raw.load(x + k);
    look(raw);
  }
  top = warp_max(top);
  ss = warp_sum(ss);
  __syncthreads();                                 // (the token before has been read)
  if (lane == 0) { red[0][tid >> 5] = top; red[1][tid >> 5] = ss; }
  __syncthreads();
  top = red[0][0]; ss = red[1][0];
#pragma unroll
  for (int w = 1; w < WARPS; ++w) { top = fmaxf(top, red[0][w]); ss += red[1][w]; }
  const float xs = scale_to_2_13(top), xo = xs * ODD, u = xs * CODE_UNIT;
  if (tid == 0) factor[token] = (norm ? 1.0f / sqrtf(ss / (float)in + eps) : 1.0f) / xs;
  const int chunks = (in + W4_CHUNK - 1) / W4_CHUNK;
  const auto lay = [&](int chunk, const Raw8<bf16>& raw) {
    float v[8];
    raw.get(v);
    float s = ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
    unsigned char* block = blocks + chunk * stride + (size_t)token * next;
    const auto at = [&](int i) { return reinterpret_cast<uint4*>(block + (size_t)(i >> 2) * row + 16 * (i & 3)); };
    *at(lane) = make_uint4(pack2_f16(v[0] * xs, v[4] * xs), pack2_f16(v[1] * xo, v[5] * xo), pack2_f16(v[2] * xs, v[6] * xs),
                           pack2_f16(v[3] * xo, v[7] * xo));
#pragma unroll
    for (int o = 1; o < L::LANES; o <<= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane % L::LANES == 0) {
      const float sm = s * u, a = -8.f * sm;
      const float ah = round_bf16(a), mh = round_bf16(sm), am = round_bf16(a - ah), mm = round_bf16(sm - mh);
      *at(32 + lane / L::LANES) = make_uint4(pack2(ah, mh), pack2(am, mm), pack2((a - ah) - am, (sm - mh) - mm), 0u);
    }
    if (lane < L::SUMS - NG) *at(32 + NG + lane) = make_uint4(0u, 0u, 0u, 0u);
  };
#pragma unroll
  for (int i = 0; i < KEEP; ++i)
    if ((tid >> 5) + i * WARPS < chunks) lay((tid >> 5) + i * WARPS, kept[i]);
  for (int chunk = (tid >> 5) + KEEP * WARPS; chunk < chunks; chunk += WARPS) {
    Raw8<bf16> raw;
    raw.zero();
    const int k = chunk * W4_CHUNK + L::k(lane >> 2, lane & 3);
    if (k < there) raw.load(x + k);
    lay(chunk, raw);
  }
}
template <int NG>
__global__ void __launch_bounds__(1024)
w4_prepare_kernel(const bf16* __restrict__ X, int64_t ldx, int in, int n, int norm, float eps, unsigned char* __restrict__ blocks,
                  float* __restrict__ factor) {
  // a CTA per token, those up to the next multiple of eight too (zeros): tokens lie side by side in each row of fragments, which
  // a load of eight tokens then reads as whole lines
  dep_launch();
  const int token = blockIdx.x, tokens = gridDim.x;
  w4_prepare<NG, 1024>(token < n ? X + (size_t)token * ldx : nullptr, token, in, norm, eps, blocks, 64 * tokens, 64,
                       (size_t)W4Order<NG>::BLOCK * tokens, factor);
}

template <int NB, int MT, int NG, int WK>
struct W4Tile {
  static constexpr int WR = W4_WARPS / WK;
  static constexpr int STAGES = 2;
  // A row's 128 bytes of codes lie in pieces of a group, piece p of row r at place p ^ (r % NG), so that the lanes of a fragment's
  // load (eight rows, one group) lie in distinct banks.
  static constexpr int PARAMS = 16 * MT * 128, STAGE = PARAMS + 16 * MT * NG * 4;
  static constexpr int RING = W4_WARPS * STAGES * STAGE;
  static constexpr int RED = W4_WARPS * MT * 16 * 4;                      // a token's [wk][wr][mt][row]
};

struct W4Mat { const char* codes; const uint32_t* params; };

// The line of steps: tiles x steps, cut into `ctas` pieces.  A share is [token][a tile's rows in the order wr, mt, row]; a CTA
// has at most two: 2 cta + 1 of a tile that begins in its piece, 2 cta of one that began before.
// With `whole` the cuts fall between tiles.
struct W4Line {
  int tiles, steps, ctas, whole;
  __device__ __forceinline__ long total() const { return (long)tiles * steps; }
  __device__ __forceinline__ long begin(int cta) const {
    return whole ? (long)steps * (int)((long)tiles * cta / ctas) : total() * cta / ctas;
  }
  __device__ __forceinline__ int cta_of(long x) const { return (int)(((x + 1) * ctas - 1) / total()); }
};

// where output r of a tile lies in a share (two matrices: the up row 16 behind the gate row)
template <int MT, bool TWO> __device__ __forceinline__ int w4_place(int r) {
  constexpr int WROWS = TWO ? 8 * MT : 16 * MT;
  const int w = r / WROWS, rw = r - w * WROWS;
  return w * MT * 16 + (TWO ? (rw >> 4) * 32 + (rw & 15) : rw);
}

template <int NB, int MT, int NG, bool TWO, int WK, bool LOCAL>
__global__ void __launch_bounds__(W4_WARPS * 32, NB > 2 ? 1 : 2)
w4_gemv_kernel(W4Mat m1, W4Mat m2, int out, int in, int n, W4Line line, const bf16* __restrict__ X, int64_t ldx, int norm, float eps,
               const unsigned char* blocks_g, float* factor_g, float* __restrict__ part, W4Out o) {
  using T = W4Tile<NB, MT, NG, WK>;
  using L = W4Order<NG>;
  constexpr int WR = T::WR, WROWS = TWO ? 8 * MT : 16 * MT, ROWS = WR * WROWS;      // output features of a warp, of a tile
  constexpr int RSTRIDE = WR * MT * 16;
  constexpr int GT = L::GT, GB = 128 / NG;                    // words of a lane in a group, bytes of a row's group
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ float sm_factor[8 * NB];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, cc = lane & 3;
  const int wk = warp % WK, wr = warp / WK;
  const int chunks = (in + W4_CHUNK - 1) / W4_CHUNK, groups = in / (W4_CHUNK / NG);
  const size_t row_bytes = in / 2;
  float* red = reinterpret_cast<float*>(smem + T::RING);
  unsigned char* x_local = smem + T::RING + n * T::RED;       // a block of zeros, then LOCAL's blocks
  unsigned char* ring = smem + warp * (T::STAGES * T::STAGE);
  const uint32_t ring_s = (uint32_t)__cvta_generic_to_shared(ring);
  const long u0 = line.begin(blockIdx.x), u1 = line.begin(blockIdx.x + 1);

  // the walk of the copies: tile, chunk, the lane's pointers in that tile.  Of the codes a lane copies piece lane % 8 of rows
  // lane / 8, lane / 8 + 4, ... of every 16; of the params those of row `lane` of the warp's 16 MT rows.
  const int f_row = lane >> 3, f_piece = lane & 7;
  const bool aligned = groups % (NG < 4 ? NG : 4) == 0;       // rows of params begin on the copies' boundaries
  uint32_t f_dst[2];                                          // by the parity of the row's number among its four
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int unit = f_piece * 16 / GB, within = f_piece * 16 % GB;
    f_dst[i] = ring_s + f_row * 128 + (unit ^ ((4 * i + f_row) % NG)) * GB + within;
  }
  int f_tile = (int)(u0 / line.steps), f_step = (int)(u0 - (long)f_tile * line.steps);
  long f_left = u1 - u0;                                      // steps from here on
  int f_chunk = 0, f_end = 0;
  bool fetching = true;
  const char* f_codes[MT];
  int f_rows[MT];                                             // how many of the 16 rows there are, less the lane's first
  const uint32_t* f_params = nullptr;
  uint32_t fetch_at = 0, use_at = 0;
  auto f_open = [&]() {                                       // settles on the next tile in which this warp has a chunk
    while (f_left > 0) {
      const int here = (int)min((long)(line.steps - f_step), f_left);
      const int tile = f_tile;
      f_chunk = f_step * WK + wk;
      f_end = min(chunks, (f_step + here) * WK);
      f_left -= here;
      ++f_tile;
      f_step = 0;
      if (f_chunk >= f_end) continue;
      const int r0 = tile * ROWS + wr * WROWS;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        const int rm = r0 + 16 * (TWO ? mt >> 1 : mt);
        f_rows[mt] = out - rm - f_row;
        f_codes[mt] = (TWO && (mt & 1) ? m2.codes : m1.codes) + (size_t)min(rm + f_row, out - 1) * row_bytes + (size_t)f_chunk * 128 + 16 * f_piece;
      }
      const int mt = lane >> 4;
      f_params = (TWO && (mt & 1) ? m2.params : m1.params) + (size_t)min(r0 + 16 * (TWO ? mt >> 1 : mt) + (lane & 15), out - 1) * groups;
      return;
    }
    fetching = false;
  };
  f_open();
  auto fetch_next = [&]() {
    if (fetching) {
      // rows and features that there are not: their codes stay what they are and meet x = 0 or are not written out
      if (f_chunk * W4_CHUNK + 32 * f_piece < in) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (4 * i < f_rows[mt]) cp_async16(f_dst[i & 1] + fetch_at + (16 * mt + 4 * i) * 128, f_codes[mt] + (size_t)(4 * i) * row_bytes);
      }
      if (lane < 16 * MT) {
        const uint32_t* p = f_params + f_chunk * NG;
        const uint32_t pd = ring_s + fetch_at + T::PARAMS + lane * NG * 4;
        if (aligned && (f_chunk + 1) * NG <= groups) {
          if (NG == 2) cp_async8(pd, p);
          else cp_async16(pd, p);
          if (NG == 8) cp_async16(pd + 16, p + 4);
        } else {
#pragma unroll
          for (int i = 0; i < NG; ++i) {
            const bool has = f_chunk * NG + i < groups;
            cp_async4(pd + 4 * i, has ? p + i : f_params, has);
          }
        }
      }
      f_chunk += WK;
      if (f_chunk < f_end) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) f_codes[mt] += 128 * WK;
      } else {
        f_open();
      }
    }
    cp_async_commit();
    fetch_at = fetch_at + T::STAGE == T::STAGES * T::STAGE ? 0 : fetch_at + T::STAGE;
  };
#pragma unroll
  for (int i = 0; i < T::STAGES - 1; ++i) fetch_next();
  if (LOCAL && threadIdx.x < L::BLOCK / 16) reinterpret_cast<uint4*>(x_local)[threadIdx.x] = make_uint4(0u, 0u, 0u, 0u);
  const unsigned char* blocks = blocks_g;
  if (LOCAL) {
    for (int t = 0; t < n; ++t)
      w4_prepare<NG, W4_WARPS * 32>(X + (size_t)t * ldx, t, in, norm, eps, x_local + L::BLOCK, 64, L::BLOCK, (size_t)n * L::BLOCK, sm_factor);
    blocks = x_local + L::BLOCK;
    __syncthreads();
    if (blockIdx.x == 0 && threadIdx.x < n) factor_g[threadIdx.x] = sm_factor[threadIdx.x];      // for the join
  } else {
    dep_wait();                                               // x is prepared
    if (threadIdx.x < n) sm_factor[threadIdx.x] = __ldcg(factor_g + threadIdx.x);
    __syncthreads();
  }
  dep_launch();

  int tile = (int)(u0 / line.steps), step = (int)(u0 - (long)tile * line.steps);
  for (long left = u1 - u0; left > 0;) {
    const int here = (int)min((long)(line.steps - step), left), c1 = min(chunks, (step + here) * WK);
    float y[NB][MT][4];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int i = 0; i < 4; ++i) y[nb][mt][i] = 0.f;
    // absent tokens are zeros: LOCAL's lanes read its block of them
    constexpr int XROW = LOCAL ? 64 : 64 * 8 * NB;
    const unsigned char* xp;
    const size_t x_stride = (size_t)(LOCAL ? n : 8 * NB) * L::BLOCK, x_step = LOCAL && g >= n ? 0 : WK * x_stride;
    if (LOCAL) xp = (g < n ? blocks + (step * WK + wk) * x_stride + g * L::BLOCK : x_local) + 16 * cc;
    else xp = blocks + (step * WK + wk) * x_stride + g * 64 + 16 * cc;
    for (int chunk = step * WK + wk; chunk < c1; chunk += WK) {
      fetch_next();
      cp_async_wait<T::STAGES - 1>();
      __syncwarp();
      const unsigned char* st = ring + use_at;
      use_at = use_at + T::STAGE == T::STAGES * T::STAGE ? 0 : use_at + T::STAGE;
      const unsigned char* row = st + g * 128 + 4 * GT * cc;
      const unsigned char* prm = st + T::PARAMS + g * NG * 4;
      // params words of groups that there are not meet zeros in x's sums (a NaN among them makes the row NaN, as it is)
#pragma unroll
      for (int p = 0; p < L::SUMS / 4; ++p) {
        uint4 xs[NB];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) xs[nb] = *reinterpret_cast<const uint4*>(xp + (8 + p) * XROW + 512 * nb);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          const uint32_t p0 = *reinterpret_cast<const uint32_t*>(prm + 16 * mt * NG * 4 + 4 * ((4 * p + cc) % NG));
          const uint32_t p1 = *reinterpret_cast<const uint32_t*>(prm + (16 * mt + 8) * NG * 4 + 4 * ((4 * p + cc) % NG));
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            mma16816(y[nb][mt], p0, p1, p0, p1, xs[nb].x, xs[nb].y);
            mma16816(y[nb][mt], p0, p1, 0u, 0u, xs[nb].z, 0u);
          }
        }
      }
#pragma unroll
      for (int gr = 0; gr < NG; ++gr) {
        uint4 xf[NB][GT];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int tt = 0; tt < GT; ++tt) xf[nb][tt] = *reinterpret_cast<const uint4*>(xp + (gr * GT + tt) * XROW + 512 * nb);
        uint32_t w[MT][2][GT], q[MT][2];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            load_words<GT>(row + (16 * mt + 8 * h) * 128 + (gr ^ (g % NG)) * GB, w[mt][h]);
            q[mt][h] = *reinterpret_cast<const uint32_t*>(prm + ((16 * mt + 8 * h) * NG + gr) * 4);
          }
        float acc[NB][MT][4];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[nb][mt][i] = 0.f;
        // the row tiles take turns, so that a product does not wait for the one before it
#pragma unroll
        for (int tt = 0; tt < GT; ++tt) {
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            const uint32_t a0 = code_pair<0>(w[mt][0][tt]), a1 = code_pair<0>(w[mt][1][tt]);
            const uint32_t a2 = code_pair<1>(w[mt][0][tt]), a3 = code_pair<1>(w[mt][1][tt]);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) mma_f16(acc[nb][mt], a0, a1, a2, a3, xf[nb][tt].x, xf[nb][tt].y);
          }
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            const uint32_t a0 = code_pair<2>(w[mt][0][tt]), a1 = code_pair<2>(w[mt][1][tt]);
            const uint32_t a2 = code_pair<3>(w[mt][0][tt]), a3 = code_pair<3>(w[mt][1][tt]);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) mma_f16(acc[nb][mt], a0, a1, a2, a3, xf[nb][tt].z, xf[nb][tt].w);
          }
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          const float s0 = lo_bf16(q[mt][0]), s1 = lo_bf16(q[mt][1]);
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              y[nb][mt][i] = fmaf(s0, acc[nb][mt][i], y[nb][mt][i]);
              y[nb][mt][2 + i] = fmaf(s1, acc[nb][mt][2 + i], y[nb][mt][2 + i]);
            }
        }
      }
      xp += x_step;
      __syncwarp();                                           // the stage may be filled again
    }
    // ---- the warps' shares meet: red[wk][token][wr][mt][row]
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int token = 8 * nb + 2 * cc + i;
        if (token < n) {
          float* r = red + (size_t)(wk * n + token) * RSTRIDE + wr * MT * 16 + g;
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) { r[16 * mt] = y[nb][mt][i]; r[16 * mt + 8] = y[nb][mt][2 + i]; }
        }
      }
    __syncthreads();
    auto sum_wk = [&](int t, int r) {
      float v = 0.f;
#pragma unroll
      for (int w = 0; w < WK; ++w) v += red[(size_t)(w * n + t) * RSTRIDE + r];
      return v;
    };
    if (here == line.steps) {
      for (int i = threadIdx.x; i < n * ROWS; i += W4_WARPS * 32) {
        const int t = i / ROWS, r = i - t * ROWS, row = tile * ROWS + r, at = w4_place<MT, TWO>(r);
        if (row >= out) continue;
        const float f = sm_factor[t], v = sum_wk(t, at) * CODE_UNIT_INV * f;
        w4_store<bf16>(o, t, row, TWO ? silu_mul(v, sum_wk(t, at + 16) * CODE_UNIT_INV * f) : v);
      }
    } else {
      float* mine = part + (size_t)(2 * blockIdx.x + (step == 0 ? 1 : 0)) * n * RSTRIDE;
      for (int i = threadIdx.x; i < n * RSTRIDE; i += W4_WARPS * 32) mine[i] = sum_wk(i / RSTRIDE, i % RSTRIDE);
    }
    left -= here;
    ++tile;
    step = 0;
    __syncthreads();
  }
  cp_async_wait<0>();
}

// Outputs of tiles that were cut between CTAs: the sum of their shares.
template <int MT, bool TWO, int WR>
__global__ void __launch_bounds__(128)
w4_join_kernel(int out, int n, W4Line line, const float* __restrict__ part, const float* __restrict__ factor, W4Out o) {
  constexpr int ROWS = WR * (TWO ? 8 * MT : 16 * MT), RSTRIDE = WR * MT * 16;
  const int row = blockIdx.x * 128 + threadIdx.x, t = blockIdx.y;
  const int tile = row / ROWS, at = w4_place<MT, TWO>(row - tile * ROWS);
  const int c0 = line.cta_of((long)tile * line.steps), c1 = line.cta_of((long)(tile + 1) * line.steps - 1);
  dep_wait();
  if (row >= out || c0 == c1) return;
  const size_t share = (size_t)n * RSTRIDE;
  const float* p = part + (size_t)t * RSTRIDE + at;
  float v = __ldcg(p + (2 * c0 + 1) * share), v2 = TWO ? __ldcg(p + (2 * c0 + 1) * share + 16) : 0.f;
#pragma unroll 8
  for (int c = c0 + 1; c <= c1; ++c) {
    v += __ldcg(p + 2 * c * share);
    if (TWO) v2 += __ldcg(p + 2 * c * share + 16);
  }
  const float f = __ldcg(factor + t);
  v *= CODE_UNIT_INV;
  v2 *= CODE_UNIT_INV;
  w4_store<bf16>(o, t, row, TWO ? silu_mul(v * f, v2 * f) : v * f);
}

template <typename... KArgs, typename... Args>
cudaError_t launch_dep_smem(void (*kernel)(KArgs...), dim3 grid, int threads, size_t smem, cudaStream_t st, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, KArgs(args)...);
}

template <int NB, int MT, int NG, bool TWO, int WK, bool LOCAL>
spts_status launch_tile(spts_ctx* ctx, const W4GemvArgs& a) {
  using T = W4Tile<NB, MT, NG, WK>;
  const W4Out o{a.residual, a.ldr, a.Y, a.ldy, a.fp32_out};
  const int rows = T::WR * (TWO ? 8 * MT : 16 * MT), chunks = ceil_div(a.in, W4_CHUNK);
  W4Line line;
  line.tiles = ceil_div(a.out, rows);
  line.steps = ceil_div(chunks, WK);
  constexpr int SEATS = NB > 2 ? 1 : 2;            // CTAs to an SM
  const int most = SEATS * (ctx->sm_count < W4_MAX_CTAS / 2 ? ctx->sm_count : W4_MAX_CTAS / 2);
  // what the workspace holds of shares (two to a CTA), and of x by W4_X_ELEMENTS
  static_assert((size_t)2 * SEATS * (W4_MAX_CTAS / 2) * 8 * NB * T::WR * MT * 16 <= W4_PART_FLOATS, "shares");
  static_assert(2 * W4Order<NG>::BLOCK <= 5 * W4_CHUNK && 8 * NB * sizeof(float) <= 256, "x");
  const long total = (long)line.tiles * line.steps;
  // Whole tiles where there are three for every resident CTA, or between one and two for every SM, or where tiles are too
  // short for two more launches to pay (8 steps take about 8 us); else equal pieces of the line, whose cut tiles are joined.
  line.whole = line.tiles >= 3 * most || (line.tiles <= most && (line.tiles >= ctx->sm_count || (LOCAL && line.steps <= 8)));
  line.ctas = line.whole ? (line.tiles < most ? line.tiles : most) : total < most ? (int)total : most;
  const bool cut = !line.whole;
  unsigned char* blocks = (unsigned char*)ctx->ws.w4_x;
  float* factor = (float*)(blocks + (size_t)chunks * 8 * NB * W4Order<NG>::BLOCK);
  if (!LOCAL) {
    w4_prepare_kernel<NG><<<8 * NB, 1024, 0, ctx->stream>>>((const bf16*)a.X, a.ldx, a.in, a.n, a.norm, ctx->desc.rms_eps, blocks, factor);
    SPTS_CUDA_OK(ctx);
  }
  auto kernel = w4_gemv_kernel<NB, MT, NG, TWO, WK, LOCAL>;
  const size_t smem = T::RING + (size_t)a.n * T::RED + (LOCAL ? ((size_t)chunks * a.n + 1) * W4Order<NG>::BLOCK : 0);
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return SPTS_ERR_CUDA;
  const W4Mat m1{(const char*)a.codes, (const uint32_t*)a.params}, m2{(const char*)a.codes2, (const uint32_t*)a.params2};
  const cudaError_t e = [&]() {
    if (!LOCAL)
      return launch_dep_smem(kernel, dim3(line.ctas), W4_WARPS * 32, smem, ctx->stream, m1, m2, a.out, a.in, a.n, line, (const bf16*)a.X, a.ldx,
                             a.norm, ctx->desc.rms_eps, (const unsigned char*)blocks, factor, ctx->ws.w4_part, o);
    kernel<<<line.ctas, W4_WARPS * 32, smem, ctx->stream>>>(m1, m2, a.out, a.in, a.n, line, (const bf16*)a.X, a.ldx, a.norm,
                                                            ctx->desc.rms_eps, blocks, factor, ctx->ws.w4_part, o);
    return cudaGetLastError();
  }();
  if (e != cudaSuccess) return SPTS_ERR_CUDA;
  SPTS_CUDA_OK(ctx);
  if (cut) {
    if (launch_dep_smem(w4_join_kernel<MT, TWO, T::WR>, dim3(ceil_div(a.out, 128), a.n), 128, 0, ctx->stream, a.out, a.n, line,
                        (const float*)ctx->ws.w4_part, (const float*)factor, o) != cudaSuccess)
      return SPTS_ERR_CUDA;
    SPTS_CUDA_OK(ctx);
  }
  return SPTS_OK;
}
template <int NB, int NG>
spts_status launch_rows(spts_ctx* ctx, const W4GemvArgs& a) {
  if constexpr (NB > 1) {
    if (a.codes2 != nullptr) return launch_tile<NB, 2, NG, true, 1, false>(ctx, a);
    // up to 16 tokens: 16 rows to a warp, whose registers let two CTAs onto an SM (9 x 4096 x 4096: 9.8 us instead of 11.7, 16 x
    // 28672 x 4096: 27.8 instead of 28.7); more tokens weigh more on x's loads (32 x 128256 x 4096: 164 us instead of 150)
    return launch_tile<NB, NB == 2 ? 1 : 2, NG, false, 1, false>(ctx, a);
  } else {
    // few elements of x are laid out in the kernel itself; few rows: all eight warps on one tile of 16
    const bool local = (long)a.n * align_up((size_t)a.in, W4_CHUNK) <= W4_LOCAL;
    // two matrices: tiles of 64 features and half the depth of a step where there are many (8 x 14336 x 4096: 20.2 us instead of 22.2, 8 x
    // 28672 x 8192: 55 instead of 61), of 32 where there are few (8 x 1024 x 4096: 7.6 instead of 9.0)
    if (a.codes2 != nullptr && ceil_div(a.out, 32) > 2 * ctx->sm_count)
      return local ? launch_tile<1, 2, NG, true, W4_WK / 2, true>(ctx, a) : launch_tile<1, 2, NG, true, W4_WK / 2, false>(ctx, a);
    if (a.codes2 != nullptr) return local ? launch_tile<1, 2, NG, true, W4_WK, true>(ctx, a) : launch_tile<1, 2, NG, true, W4_WK, false>(ctx, a);
    if (ceil_div(a.out, 16) <= 2 * ctx->sm_count)
      return local ? launch_tile<1, 1, NG, false, 8, true>(ctx, a) : launch_tile<1, 1, NG, false, 8, false>(ctx, a);
    return local ? launch_tile<1, 2, NG, false, W4_WK, true>(ctx, a) : launch_tile<1, 2, NG, false, W4_WK, false>(ctx, a);
  }
}
template <int NB>
spts_status launch_group(spts_ctx* ctx, const W4GemvArgs& a) {
  if (a.group == 128) return launch_rows<NB, 2>(ctx, a);
  return a.group == 64 ? launch_rows<NB, 4>(ctx, a) : launch_rows<NB, 8>(ctx, a);
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
