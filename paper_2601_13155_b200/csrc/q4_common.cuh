// 4-bit groups: value = scale * (code - 8) + mid, bf16 (scale, mid) per 32, 64 or 128 elements (include/spts.h has the
// quantiser's definition).  Shared by the weight and the KV-cache kernels.
#pragma once

#include <cuda_fp16.h>

#include "spts_common.cuh"

namespace spts {
namespace q4 {

__device__ __forceinline__ float lo_bf16(uint32_t w) { return __uint_as_float(w << 16); }            // scale of a params word
__device__ __forceinline__ float hi_bf16(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }    // mid

__device__ __forceinline__ void load8(const float* p, float* x) {
  const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
  x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
__device__ __forceinline__ void load8(const bf16* p, float* x) {
  const uint4 v = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[2 * i] = lo_bf16(w[i]); x[2 * i + 1] = hi_bf16(w[i]); }
}
__device__ __forceinline__ void store8(float* p, const float* x) {
  *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
  *reinterpret_cast<float4*>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ void store8(bf16* p, const float* x) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t*>(&v);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}

// ---- matrix instructions on codes
// A nibble in the low mantissa bits of an fp16 whose other bits are zero IS a number: code * 2^-24 in bits 0..3 and
// code * 2^-20 in bits 4..7 (subnormals, and exact; the matrix units take them as they are).  So the eight codes of a word
// become four registers of two fp16 with four masks and one shift, without a bias or a conversion.  J-th codes of the two
// 16-bit halves, times 2^-24 (J even) or 2^-20 (J odd):
template <int J> __device__ __forceinline__ uint32_t code_pair(uint32_t w) {
  const uint32_t s = J < 2 ? w : w >> 8;
  return s & ((J & 1) ? 0x00F000F0u : 0x000F000Fu);
}
constexpr float CODE_UNIT = 5.9604644775390625e-08f;        // 2^-24
constexpr float CODE_UNIT_INV = 16777216.f;                 // 2^24
constexpr float ODD = 0.0625f;                              // what a factor of an odd J is multiplied by to be in the same unit
// The power of two that brings `top` (>= 0) to [2^13, 2^14), held within 2^-100 .. 2^120; 1 for zero, infinity and NaN.
__device__ __forceinline__ float scale_to_2_13(float top) {
  const int e = (int)(__float_as_uint(top) >> 23);          // biased exponent
  if (e == 0 || e >= 255) return e == 0 && top > 0.f ? 1.329227995784916e36f : 1.f;
  return __uint_as_float((uint32_t)(127 + max(-100, min(120, 13 + 127 - e))) << 23);
}
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack2_f16(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ float round_bf16(float v) { return __bfloat162float(__float2bfloat16_rn(v)); }

// ---- asynchronous copies into shared memory
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async4(uint32_t dst, const void* src, bool in) {       // zero where not `in`
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(in ? 4 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Quantises the eight elements of this lane; the group is `lanes` (4, 8 or 16) neighbouring lanes of the warp, aligned
// to their number, and every lane of the warp calls.  Returns the eight codes, element i in bits 4i .. 4i + 3; `params`
// = scale | mid << 16; read (if not null) the values that the codes stand for.
// The code is the exact quotient's rounding: the fp32 quotient is off by less than 3 * 2^-24 * 9 = 1.7e-6 steps (three
// roundings, at most nine steps from the middle), so wherever it lies farther than 1e-5 from a border it gives the exact
// quotient's code, and the rest (about one in 50,000 of smooth data) is divided in 64 bits.
__device__ __forceinline__ uint32_t quantize8(const float* x, int lanes, uint32_t& params, float* read, bool& nonfinite) {
  float hi = x[0], lo = x[0];
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    hi = fmaxf(hi, x[i]); lo = fminf(lo, x[i]);
    bad = bad || !(fabsf(x[i]) <= 3.402823466e38f);
  }
  for (int o = 1; o < lanes; o <<= 1) {
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
  }
  const uint32_t votes = __ballot_sync(0xffffffffu, bad);
  const int lane = threadIdx.x & 31;
  const uint32_t mine = ((1u << lanes) - 1u) << (lane & ~(lanes - 1));
  nonfinite = (votes & mine) != 0;
  if (nonfinite) {
    params = 0x7FC00000u;                       // scale 0, mid NaN
    if (read)
#pragma unroll
      for (int i = 0; i < 8; ++i) read[i] = __uint_as_float(0x7FC00000u);
    return 0x88888888u;
  }
  const double dh = (double)hi, dl = (double)lo;
  const bf16 sb = __float2bfloat16_rn((float)((dh - dl) / 15.0));
  const float s = __bfloat162float(sb);
  const bf16 mb = __float2bfloat16_rn((float)(0.5 * (dh + dl) + 0.5 * (double)s));
  const float m = __bfloat162float(mb);
  params = (uint32_t)__bfloat16_as_ushort(sb) | ((uint32_t)__bfloat16_as_ushort(mb) << 16);
  uint32_t word = 0;
  const bool tiny = s < 1e-30f;                 // 1 / s would overflow
  const float inv = tiny ? 0.f : 1.0f / s;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float t = (x[i] - m) * inv;
    float r = rintf(t);
    if (tiny || fabsf(fabsf(t - r) - 0.5f) < 1e-5f) {
      if (s == 0.f) r = 0.f;
      else r = (float)fmin(8.0, fmax(-9.0, rint(((double)x[i] - (double)m) / (double)s)));
    }
    const int c = (int)fminf(7.f, fmaxf(-8.f, r));
    word |= (uint32_t)(c + 8) << (4 * i);
    if (read) read[i] = fmaf(s, (float)c, m);
  }
  return word;
}

}  // namespace q4
}  // namespace spts
