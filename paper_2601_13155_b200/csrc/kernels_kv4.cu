// The 4-bit KV cache: rows are quantised into it (kv4_append_kernel) and single tokens attend to it.
//
// kv4_attn_plain_kernel: one CTA per query head and sequence, CUDA cores, fp32 arithmetic, online softmax per warp.
// fp32 storage and SPTS_REFERENCE_KERNELS.
#include "q4_common.cuh"

namespace spts {

namespace {

using namespace q4;

struct Kv4Dev {
  char* k_codes; char* v_codes; uint32_t* k_params; uint32_t* v_params;
  int32_t* pos; int32_t* len;
  int n_seq, capacity, group, Hkv;
};

// One unit = one (row, KV head, K or V): D / 8 lanes, eight dims each; quantised, its words stored in the cache's order.
template <typename T, int D>
__global__ void __launch_bounds__(256)
kv4_append_kernel(Kv4Dev c, const T* __restrict__ K, int64_t ldk, const T* __restrict__ V, int64_t ldv,
                  const int32_t* __restrict__ pos, const int32_t* __restrict__ row_start, const int32_t* __restrict__ at,
                  int n_rows, T* __restrict__ K_read, T* __restrict__ V_read, int* status) {
  constexpr int LPR = D / 8;                       // lanes per unit
  const int sub = threadIdx.x % LPR;
  const int units = 2 * c.Hkv;
  const long total = (long)n_rows * units;
  const long u0 = ((long)blockIdx.x * 256 + threadIdx.x) / LPR, stride = (long)gridDim.x * 256 / LPR;
  const long first = ((long)blockIdx.x * 256 + (threadIdx.x & ~31)) / LPR;      // the warp's first unit
  for (long step = 0; first + step < total; step += stride) {
    const long u = u0 + step;
    const int row = u < total ? (int)(u / units) : 0;
    const int which = (int)(u % units);
    const int kvh = which >> 1;
    const bool is_v = which & 1;
    // the sequence that owns the row: the last b with row_start[b] <= row
    int b = row, first_row = row;
    bool in = u < total;
    if (row_start != nullptr) {
      int lo = 0, hi = c.n_seq;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (__ldg(&row_start[mid]) <= row) lo = mid; else hi = mid;
      }
      b = lo;
      first_row = __ldg(&row_start[b]);
      in = in && row >= first_row && row < __ldg(&row_start[b + 1]);
    }
    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (in) load8((is_v ? V + (size_t)row * ldv : K + (size_t)row * ldk) + kvh * D + 8 * sub, x);
    uint32_t p;
    bool bad;
    float read[8];
    const uint32_t w = quantize8(x, c.group / 8, p, read, bad);
    if (!in) continue;
    if (K_read != nullptr || V_read != nullptr) {
      T* dst = is_v ? V_read : K_read;
      if (dst != nullptr) store8(dst + ((size_t)row * c.Hkv + kvh) * D + 8 * sub, read);
    }
    const long slot = (long)(at != nullptr ? __ldg(&at[b]) : c.len[b]) + (row - first_row);
    if (bad) set_status(status, SPTS_ERR_NONFINITE);
    if (slot < 0 || slot >= c.capacity) {
      if (sub == 0) set_status(status, SPTS_ERR_WORKSPACE);
      continue;
    }
    const size_t r = ((size_t)b * c.Hkv + kvh) * c.capacity + slot;
    const int t = sub >> 2, q = sub & 3;           // dims 32 t + 8 q .. + 7
    if (!is_v) {
      reinterpret_cast<uint32_t*>(c.k_codes + r * (D / 2))[q * (D / 32) + t] = w;
    } else {
      uint16_t* v = reinterpret_cast<uint16_t*>(c.v_codes + r * (D / 2));
      v[2 * q * (D / 32) + t] = (uint16_t)w;
      v[(2 * q + 1) * (D / 32) + t] = (uint16_t)(w >> 16);
    }
    const int lanes = c.group / 8;
    if (sub % lanes == 0) (is_v ? c.v_params : c.k_params)[r * (D / c.group) + sub / lanes] = p;
    if (pos != nullptr && c.pos != nullptr && which == 0 && sub == 0) c.pos[(size_t)b * c.capacity + slot] = pos[row];
  }
}

// len[b] = at[b] + rows of b, clipped; a kernel of its own behind the append, whose blocks still read the old lengths
__global__ void kv4_len_kernel(int32_t* len, const int32_t* __restrict__ at, const int32_t* __restrict__ row_start, int n_seq,
                               int capacity) {
  const int b = blockIdx.x * blockDim.x + threadIdx.x;
  if (b >= n_seq) return;
  const long n = row_start != nullptr ? max(0, row_start[b + 1] - row_start[b]) : 1;
  const long v = (long)(at != nullptr ? at[b] : len[b]) + n;
  len[b] = (int32_t)(v < 0 ? 0 : v > capacity ? capacity : v);
}

constexpr int PLAIN_WARPS = 16;

template <typename T, int D>
__global__ void __launch_bounds__(PLAIN_WARPS * 32)
kv4_attn_plain_kernel(Kv4Dev c, const T* __restrict__ Q, int64_t ldq, int H, T* __restrict__ O, int64_t ldo) {
  constexpr int E = D / 32;                        // storage positions per lane
  __shared__ float sm_m[PLAIN_WARPS], sm_l[PLAIN_WARPS];
  __shared__ float sm_o[PLAIN_WARPS][D];
  const int h = blockIdx.x, b = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int kvh = h / (H / c.Hkv);
  const int len = max(0, min(c.len[b], c.capacity));
  T* out = O + (size_t)b * ldo + (size_t)h * D;
  float q[E], o[E];
  int gk[E], gv[E], dv[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int p = lane * E + e;
    const int dk = 32 * ((p / 8) % (D / 32)) + 8 * (p / (D / 4)) + p % 8;
    dv[e] = 32 * ((p / 4) % (D / 32)) + 4 * (p / (D / 8)) + p % 4;
    gk[e] = dk / c.group; gv[e] = dv[e] / c.group;
    q[e] = to_f32(Q[(size_t)b * ldq + (size_t)h * D + dk]) * rsqrtf((float)D);
    o[e] = 0.f;
  }
  float m = -INFINITY, l = 0.f;
  const size_t base = ((size_t)b * c.Hkv + kvh) * c.capacity;
  const int ng = D / c.group;
  for (int j = warp; j < len; j += PLAIN_WARPS) {
    const size_t r = base + j;
    uint32_t kw, vw;
    if (E == 4) {
      kw = reinterpret_cast<const uint16_t*>(c.k_codes + r * (D / 2))[lane];
      vw = reinterpret_cast<const uint16_t*>(c.v_codes + r * (D / 2))[lane];
    } else {
      kw = reinterpret_cast<const uint8_t*>(c.k_codes + r * (D / 2))[lane];
      vw = reinterpret_cast<const uint8_t*>(c.v_codes + r * (D / 2))[lane];
    }
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const uint32_t p = c.k_params[r * ng + gk[e]];
      s = fmaf(q[e], fmaf(lo_bf16(p), (float)((int)((kw >> (4 * e)) & 15) - 8), hi_bf16(p)), s);
    }
    s = warp_sum(s);
    const float mn = fmaxf(m, s);
    // a NaN score (non-finite rows in the cache) goes on as NaN
    const float corr = m == -INFINITY ? 0.f : expf(m - mn), pr = s == -INFINITY ? 0.f : expf(s - mn);
    l = l * corr + pr;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const uint32_t p = c.v_params[r * ng + gv[e]];
      o[e] = fmaf(pr, fmaf(lo_bf16(p), (float)((int)((vw >> (4 * e)) & 15) - 8), hi_bf16(p)), o[e] * corr);
    }
    m = mn;
  }
  if (lane == 0) { sm_m[warp] = m; sm_l[warp] = l; }
#pragma unroll
  for (int e = 0; e < E; ++e) sm_o[warp][dv[e]] = o[e];
  __syncthreads();
  for (int dim = threadIdx.x; dim < D; dim += PLAIN_WARPS * 32) {
    float M = -INFINITY, L = 0.f, a = 0.f;
    for (int w = 0; w < PLAIN_WARPS; ++w) M = fmaxf(M, sm_m[w]);
    for (int w = 0; w < PLAIN_WARPS; ++w) {
      const float f = sm_m[w] == -INFINITY ? 0.f : expf(sm_m[w] - M);
      L += sm_l[w] * f;
      a = fmaf(sm_o[w][dim], f, a);
    }
    out[dim] = from_f32<T>(len > 0 ? a / L : 0.f);
  }
}

Kv4Dev kv4_dev(const spts_ctx* ctx, const spts_kv4_cache* c) {
  return Kv4Dev{(char*)c->k_codes, (char*)c->v_codes, (uint32_t*)c->k_params, (uint32_t*)c->v_params, c->pos, c->len,
                c->n_seq, c->capacity, c->group, ctx->desc.n_kv_heads};
}

template <typename T, int D>
spts_status append_t(spts_ctx* ctx, const spts_kv4_cache* cache, const void* K, int64_t ldk, const void* V, int64_t ldv,
                     const int32_t* pos, const int32_t* row_start, const int32_t* at, int n_rows, void* K_read, void* V_read) {
  const Kv4Dev c = kv4_dev(ctx, cache);
  if (n_rows > 0) {
    long blocks = ((long)n_rows * 2 * c.Hkv * (D / 8) + 255) / 256;
    if (blocks > 8L * ctx->sm_count) blocks = 8L * ctx->sm_count;
    kv4_append_kernel<T, D><<<(int)blocks, 256, 0, ctx->stream>>>(c, (const T*)K, ldk, (const T*)V, ldv, pos, row_start, at, n_rows,
                                                                  (T*)K_read, (T*)V_read, ctx->ws.status);
    SPTS_CUDA_OK(ctx);
  }
  kv4_len_kernel<<<ceil_div(c.n_seq, 256), 256, 0, ctx->stream>>>(c.len, at, row_start, c.n_seq, c.capacity);
  SPTS_CUDA_OK(ctx);
  return SPTS_OK;
}

template <typename T, int D>
spts_status attn_plain_t(spts_ctx* ctx, const spts_kv4_cache* cache, const void* Q, int64_t ldq, void* O, int64_t ldo) {
  const Kv4Dev c = kv4_dev(ctx, cache);
  const int H = ctx->desc.n_q_heads;
  kv4_attn_plain_kernel<T, D><<<dim3(H, c.n_seq), PLAIN_WARPS * 32, 0, ctx->stream>>>(c, (const T*)Q, ldq, H, (T*)O, ldo);
  SPTS_CUDA_OK(ctx);
  return SPTS_OK;
}

}  // namespace

spts_status launch_kv4_append(spts_ctx* ctx, const spts_kv4_cache* cache, const void* K, int64_t ldk, const void* V,
                              int64_t ldv, const int32_t* pos, const int32_t* row_start, const int32_t* at, int n_rows,
                              void* K_read, void* V_read) {
  const bool wide = ctx->desc.head_dim == 128;
  if (ctx->desc.dtype == SPTS_BF16)
    return wide ? append_t<bf16, 128>(ctx, cache, K, ldk, V, ldv, pos, row_start, at, n_rows, K_read, V_read)
                : append_t<bf16, 64>(ctx, cache, K, ldk, V, ldv, pos, row_start, at, n_rows, K_read, V_read);
  return wide ? append_t<float, 128>(ctx, cache, K, ldk, V, ldv, pos, row_start, at, n_rows, K_read, V_read)
              : append_t<float, 64>(ctx, cache, K, ldk, V, ldv, pos, row_start, at, n_rows, K_read, V_read);
}

spts_status launch_kv4_attention(spts_ctx* ctx, const spts_kv4_cache* cache, const void* Q, int64_t ldq, void* O, int64_t ldo) {
  const bool wide = ctx->desc.head_dim == 128;
  if (ctx->desc.dtype == SPTS_BF16)
    return wide ? attn_plain_t<bf16, 128>(ctx, cache, Q, ldq, O, ldo) : attn_plain_t<bf16, 64>(ctx, cache, Q, ldq, O, ldo);
  return wide ? attn_plain_t<float, 128>(ctx, cache, Q, ldq, O, ldo) : attn_plain_t<float, 64>(ctx, cache, Q, ldq, O, ldo);
}

}  // namespace spts
