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
// Eight elements as they lie in memory.
template <typename T> struct Raw8;
template <> struct Raw8<float> {
  float4 a, b;
  __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ void load(const float* p) { a = *reinterpret_cast<const float4*>(p); b = *reinterpret_cast<const float4*>(p + 4); }
  __device__ __forceinline__ void get(float* x) const { x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w; }
};
template <> struct Raw8<bf16> {
  uint4 v;
  __device__ __forceinline__ void zero() { v = make_uint4(0u, 0u, 0u, 0u); }
  __device__ __forceinline__ void load(const bf16* p) { v = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void get(float* x) const {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = lo_bf16(w[i]); x[2 * i + 1] = hi_bf16(w[i]); }
  }
};
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

// code i of a word, less 8, by a mask and an exact subtraction (a conversion instruction has a quarter of their rate)
__device__ __forceinline__ float code_less_8(uint32_t w, int i) {
  return __uint_as_float(((w >> (4 * i)) & 15u) | 0x4B000000u) - 8388616.f;
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
// The power of two that brings `top` (>= 0) to [2^13, 2^14), 2^120 at most (2^-114 at least, by what fp32 holds); 1 for zero,
// infinity and NaN.  Times CODE_UNIT it may leave fp32's normal range, so its inverse and CODE_UNIT_INV are applied one by one.
__device__ __forceinline__ float scale_to_2_13(float top) {
  const int e = (int)(__float_as_uint(top) >> 23);          // biased exponent
  if (e == 0 || e >= 255) return e == 0 && top > 0.f ? 1.329227995784916e36f : 1.f;
  return __uint_as_float((uint32_t)(127 + min(120, 13 + 127 - e)) << 23);
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

// N = 1, 2 or 4 neighbouring words as one load
template <int N> __device__ __forceinline__ void load_words(const unsigned char* p, uint32_t (&w)[N]) {
  if (N == 4) *reinterpret_cast<uint4*>(w) = *reinterpret_cast<const uint4*>(p);
  else if (N == 2) *reinterpret_cast<uint2*>(w) = *reinterpret_cast<const uint2*>(p);
  else w[0] = *reinterpret_cast<const uint32_t*>(p);
}

// ---- asynchronous copies into shared memory
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async8(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async4(uint32_t dst, const void* src, bool in) {       // zero where not `in`
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(in ? 4 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Quantises the eight elements of this lane; the group is LANES (4, 8 or 16) neighbouring lanes of the warp, aligned
// to their number, and every lane of the warp calls.  Returns the eight codes, element i in bits 4i .. 4i + 3; `params`
// = scale | mid << 16; read (if not null) the values that the codes stand for.
// The stored numbers are those of 64-bit arithmetic (scale and mid rounded to bf16 by way of fp32), at the price of 32-bit
// arithmetic: each is computed in fp32 with a bound on its error, and only where the bound reaches a border between two results the
// border is decided exactly.  Borders
// are common, not rare: differences of bf16 numbers have few bits, so a quotient that ends in exactly one half turns up in
// every other warp, and a mid that needs nine bits in every group; both are decided in fp32 with error-free sums.
//   scale  three roundings, off by less than 4 in the 16 bits that bf16 drops: near their middle, 64 bits (rare)
//   mid    fp32 sums with their errors: without error it is exact; with one it is off by less than 2^-22 (|hi| + |lo| + scale),
//          and where that reaches a border, 64 bits (rare)
//   code   the quotient has error below 4 * 2^-23 * 9 steps = 4.3e-6; within 1e-5 of a border the residual d - border * scale
//          decides, which a fused multiply-add gives exactly there (d = x - mid with its own error)
__device__ __forceinline__ __nv_bfloat162 as_bf162(uint32_t w) { return *reinterpret_cast<const __nv_bfloat162*>(&w); }
__device__ __forceinline__ uint32_t as_word(__nv_bfloat162 v) { return *reinterpret_cast<const uint32_t*>(&v); }

// Largest and smallest of the group; a NaN in it makes `hi` NaN.
template <int LANES> __device__ __forceinline__ void group_range(const float* p, const float* x, float& hi, float& lo) {
  hi = lo = x[0];
  bool nan = x[0] != x[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) {
    hi = fmaxf(hi, x[i]); lo = fminf(lo, x[i]);
    nan = nan || x[i] != x[i];
  }
  if (nan) hi = __uint_as_float(0x7FFFFFFFu);
#pragma unroll
  for (int o = 1; o < LANES; o <<= 1) {
    const float h = __shfl_xor_sync(0xffffffffu, hi, o);
    hi = hi != hi || h != h ? __uint_as_float(0x7FFFFFFFu) : fmaxf(hi, h);
    lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
  }
}
// The same for bf16, on pairs as they lie in memory: (largest, largest of the negatives) travel in one register.
template <int LANES> __device__ __forceinline__ void group_range(const bf16* p, const float* x, float& hi, float& lo) {
  const uint32_t w[4] = {__byte_perm(__float_as_uint(x[0]), __float_as_uint(x[1]), 0x7632), __byte_perm(__float_as_uint(x[2]), __float_as_uint(x[3]), 0x7632),
                         __byte_perm(__float_as_uint(x[4]), __float_as_uint(x[5]), 0x7632), __byte_perm(__float_as_uint(x[6]), __float_as_uint(x[7]), 0x7632)};
  const __nv_bfloat162 h = __hmax2_nan(__hmax2_nan(as_bf162(w[0]), as_bf162(w[1])), __hmax2_nan(as_bf162(w[2]), as_bf162(w[3])));
  const __nv_bfloat162 l = __hmin2_nan(__hmin2_nan(as_bf162(w[0]), as_bf162(w[1])), __hmin2_nan(as_bf162(w[2]), as_bf162(w[3])));
  const uint32_t hw = as_word(h), lw = as_word(l) ^ 0x80008000u;
  uint32_t v = as_word(__hmax2_nan(as_bf162(__byte_perm(hw, lw, 0x5410)), as_bf162(__byte_perm(hw, lw, 0x7632))));
#pragma unroll
  for (int o = 1; o < LANES; o <<= 1) v = as_word(__hmax2_nan(as_bf162(v), as_bf162(__shfl_xor_sync(0xffffffffu, v, o))));
  hi = lo_bf16(v);
  lo = -hi_bf16(v);
}

// a + b - s, exactly, where s is the rounded sum
__device__ __forceinline__ float sum_error(float a, float b, float s) {
  const float bb = __fsub_rn(s, a);
  return __fadd_rn(__fsub_rn(a, __fsub_rn(s, bb)), __fsub_rn(b, bb));
}

template <int LANES, typename T>
__device__ __forceinline__ uint32_t quantize8(const T* type, const float* x, uint32_t& params, float* read, bool& nonfinite) {
  float hi, lo;
  group_range<LANES>(type, x, hi, lo);
  const float big = fmaxf(fabsf(hi), fabsf(lo));
  nonfinite = hi != hi || !(big <= 3.402823466e38f);
  if (nonfinite) {
    params = 0x7FC00000u;                       // scale 0, mid NaN
    if (read)
#pragma unroll
      for (int i = 0; i < 8; ++i) read[i] = __uint_as_float(0x7FC00000u);
    return 0x88888888u;
  }
  // (small ranges, where fp32 loses bits to underflow, and ranges that overflow it go the long way)
  float sf = (hi - lo) * (1.0f / 15.0f);
  const uint32_t low = __float_as_uint(sf) & 0xFFFFu;
  bf16 sb = __float2bfloat16_rn(sf);
  if (!(sf > 1e-30f && sf < 1e37f) || (low - 0x7FFCu) <= 8u) sb = __float2bfloat16_rn((float)(((double)hi - (double)lo) / 15.0));
  const float s = __bfloat162float(sb);
  const float sum = hi + lo, m2 = sum + s;      // twice the mid
  const bool exact = sum - hi == lo && sum - lo == hi && m2 - sum == s && m2 - s == sum;
  const float mf = 0.5f * m2;
  bf16 mb = __float2bfloat16_rn(mf);
  if (!(big < 1e37f && s > 1e-30f)) mb = __float2bfloat16_rn((float)(0.5 * ((double)hi + (double)lo) + 0.5 * (double)s));
  else if (!exact) {
    const float me = 2.4e-7f * (fabsf(hi) + fabsf(lo) + s);
    if (__bfloat16_as_ushort(__float2bfloat16_rn(mf - me)) != __bfloat16_as_ushort(__float2bfloat16_rn(mf + me)))
      mb = __float2bfloat16_rn((float)(0.5 * ((double)hi + (double)lo) + 0.5 * (double)s));
  }
  const float m = __bfloat162float(mb);
  params = (uint32_t)__bfloat16_as_ushort(sb) | ((uint32_t)__bfloat16_as_ushort(mb) << 16);
  float xs[8], ss = s, ms = m;
#pragma unroll
  for (int i = 0; i < 8; ++i) xs[i] = x[i];
  if (s < 1e-37f) {                             // a scale near the end of fp32's range (all elements lie below 2^-90 then)
    const float up = s == 0.f ? 0.f : 1.8446744073709552e19f;
#pragma unroll
    for (int i = 0; i < 8; ++i) xs[i] = s == 0.f ? 0.f : x[i] * up;
    ss = s == 0.f ? 1.f : s * up;
    ms = m * up;
  }
  float inv;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(ss));
  // adding 1.5 * 2^23 + 8 leaves the code in a float's last bits (round to nearest, ties to even) under a constant, which
  // the sum of all eight carries off at once
  constexpr float MAGIC = 12582920.f;
  constexpr uint32_t MAGIC_BITS = 0x4B400000u;
  uint32_t word = 0;
  float r[8], far = 0.f;                        // far: the largest distance of an element from its code's value
#pragma unroll
  for (int i = 7; i >= 0; --i) {
    const float d = xs[i] - ms, y = fminf(fmaxf(fmaf(d, inv, MAGIC), MAGIC - 8.f), MAGIC + 7.f);
    r[i] = y - MAGIC;
    far = fmaxf(far, fabsf(fmaf(-r[i], ss, d)));
    word = word * 16u + __float_as_uint(y);
  }
  word -= MAGIC_BITS * 0x11111111u;
  if (far > 0.49999f * ss) {
    word = 0;
#pragma unroll
    for (int i = 7; i >= 0; --i) {
      const float d = xs[i] - ms, off = fmaf(-r[i], ss, d);
      if (fabsf(off) > 0.49999f * ss) {
        const float border = r[i] + copysignf(0.5f, off);
        const float side = fmaf(-border, ss, d) + sum_error(xs[i], -ms, d);
        const float below = border - 0.5f, even = (__float_as_uint(below + MAGIC) & 1u) ? below + 1.f : below;
        const float c = side > 0.f ? below + 1.f : side < 0.f ? below : even;
        r[i] = fminf(fmaxf(c, -8.f), 7.f);
      }
      word = word * 16u + (__float_as_uint(r[i] + MAGIC) & 15u);
    }
  }
  if (read)
#pragma unroll
    for (int i = 0; i < 8; ++i) read[i] = fmaf(s, r[i], m);
  return word;
}

}  // namespace q4
}  // namespace spts
