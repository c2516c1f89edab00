// One-byte codes to 16-bit operands, exactly.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "cache.cuh"
#include "softmax_rows.cuh"

namespace crisp {
namespace {

__device__ __forceinline__ uint32_t half2_bits(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// Four codes (bytes 0, 1 and 2, 3 of w) to two pairs of fp16.
template <int kFormat>
__device__ __forceinline__ void decode4(uint32_t w, uint32_t& lo, uint32_t& hi) {
  if (kFormat == CRISP_CACHE_E4M3) {
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\t"
        "cvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}"
        : "=r"(lo), "=r"(hi)
        : "r"(w));
  } else {
    // 0x6400 + u is the fp16 number 1024 + u for a byte u; with u = code + 128, subtracting 1152 leaves the code
    const uint32_t u = w ^ 0x80808080u;
    const __half2 bias = __half2half2(__ushort_as_half(0x6480));  // 1152
    const uint32_t a = __byte_perm(u, 0x64646464u, 0x4140), b = __byte_perm(u, 0x64646464u, 0x4342);
    const __half2 x = __hsub2(*reinterpret_cast<const __half2*>(&a), bias);
    const __half2 y = __hsub2(*reinterpret_cast<const __half2*>(&b), bias);
    lo = *reinterpret_cast<const uint32_t*>(&x);
    hi = *reinterpret_cast<const uint32_t*>(&y);
  }
}

// Two fp32 values to bf16, clamped to the largest finite one; NaN stays NaN.
__device__ __forceinline__ uint32_t pack_bf16_finite(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.satfinite.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// Four codes times their block's scale (a power of two) to two pairs of bf16, exactly.  The one exception: a value above
// 255/256 of 2^128 may have been rounded to the code for 2^128, which is clamped, so that a weight of zero hides it.
template <int kFormat>
__device__ __forceinline__ void decode_values4(uint32_t w, float scale, uint32_t& lo, uint32_t& hi) {
  float f[4];
  if (kFormat == CRISP_CACHE_E4M3) {
    uint32_t h[2];
    decode4<kFormat>(w, h[0], h[1]);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&h[k]));
      f[2 * k] = v.x * scale;
      f[2 * k + 1] = v.y * scale;
    }
  } else {
    // 0x4b000000 + u is the fp32 number 2^23 + u; with u = code + 128, subtracting 2^23 + 128 leaves the code.  (The scale
    // comes after: (2^23 + 128) scale would overflow from 2^105 on.  In pairs: eight pieces of
    // 1 to 700 tokens over up to 20000, 28/4 heads, take 293 us; one by one 297, through decode4 308.)
    const uint32_t u = w ^ 0x80808080u;
    auto number = [&](int k) { return __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7440 + k)); };
#pragma unroll
    for (int k = 0; k < 4; k += 2)
      unpack2(mul2(add2(pack2(number(k), number(k + 1)), pack2(-8388736.0f, -8388736.0f)), pack2(scale, scale)), f[k], f[k + 1]);
  }
  lo = pack_bf16_finite(f[0], f[1]);
  hi = pack_bf16_finite(f[2], f[3]);
}

}  // namespace
}  // namespace crisp
