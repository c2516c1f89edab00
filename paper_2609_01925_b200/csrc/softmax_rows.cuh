// Row-wise softmax pieces of the tcgen05 attention kernels (prefill.cu, cache_prefill.cu): one thread per query row, 64
// logits at a time in registers, base 2; packed fp32x2 arithmetic; register budgets.
#pragma once
#include "sm100_ptx.cuh"

namespace crisp {
using namespace sm100;
namespace {

template <int N>
__device__ __forceinline__ void reg_alloc() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
}
template <int N>
__device__ __forceinline__ void reg_dealloc() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}

// ---- packed fp32x2 arithmetic (two lanes per instruction on the FMA pipe)
__device__ __forceinline__ uint64_t pack2(float lo, float hi) {
  uint64_t v;
  asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(lo), "f"(hi));
  return v;
}
__device__ __forceinline__ void unpack2(uint64_t v, float& lo, float& hi) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

// 2^t for a pair of values on the FMA pipe instead of the MUFU: t = n + f with n = round(t),
// f in [-0.5, 0.5]; 2^f by a degree-4 minimax polynomial (max relative error 2.6e-6, far below the
// bf16 rounding of P); 2^n by adding n to the exponent field.  t is clamped at -125.
__device__ __forceinline__ void exp2_poly2(uint64_t t2, float& p0, float& p1) {
  float t0, t1;
  unpack2(t2, t0, t1);
  t0 = fmaxf(t0, -125.0f);
  t1 = fmaxf(t1, -125.0f);
  t2 = pack2(t0, t1);
  const uint64_t magic = pack2(12582912.0f, 12582912.0f);      // 1.5 * 2^23: rounds to an integer
  const uint64_t neg_magic = pack2(-12582912.0f, -12582912.0f);
  const uint64_t neg_one = pack2(-1.0f, -1.0f);
  const uint64_t r2 = add2(t2, magic);
  const uint64_t n2 = add2(r2, neg_magic);
  const uint64_t f2 = fma2(n2, neg_one, t2);
  uint64_t q2 = fma2(f2, pack2(0.009570101276040077f, 0.009570101276040077f),
                     pack2(0.05591785907745361f, 0.05591785907745361f));
  q2 = fma2(q2, f2, pack2(0.240247443318367f, 0.240247443318367f));
  q2 = fma2(q2, f2, pack2(0.6931217908859253f, 0.6931217908859253f));
  q2 = fma2(q2, f2, pack2(0.9999992847442627f, 0.9999992847442627f));
  float r0, r1, q0, q1;
  unpack2(r2, r0, r1);
  unpack2(q2, q0, q1);
  p0 = __int_as_float(__float_as_int(q0) + (__float_as_int(r0) << 23));
  p1 = __int_as_float(__float_as_int(q1) + (__float_as_int(r1) << 23));
}

// Maximum of 64 raw logits of one row (keys key0 .. key0 + 63 of the block); on the diagonal block only
// keys j <= r are visible.
template <bool kDiag>
__device__ __forceinline__ float row_max(const uint32_t (&x)[2][32], int r, int key0) {
  float m0 = -INFINITY, m1 = -INFINITY, m2 = -INFINITY, m3 = -INFINITY;
#pragma unroll
  for (int c = 0; c < 2; ++c)
#pragma unroll
    for (int i = 0; i < 32; i += 8) {
      float a[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        a[u] = __uint_as_float(x[c][i + u]);
        if (kDiag && (key0 + c * 32 + i + u) > r) a[u] = -INFINITY;
      }
      m0 = max3(m0, a[0], a[1]);
      m1 = max3(m1, a[2], a[3]);
      m2 = max3(m2, a[4], a[5]);
      m3 = max3(m3, a[6], a[7]);
    }
  return fmaxf(fmaxf(m0, m1), fmaxf(m2, m3));
}

// P = 2^(x * scale - m) for 64 keys as bf16 pairs (two keys per 32-bit word); returns the fp32 row sum.
// With kPolyEvery > 0 one pair in every kPolyEvery goes through exp2_poly2 (FMA pipe) instead of the MUFU.
#ifndef CRISP_POLY_EVERY
#define CRISP_POLY_EVERY 0
#endif
constexpr int kPolyEvery = CRISP_POLY_EVERY;
// `release` is called once, after kPaceRelease of the 32 pairs (see the pacing of the two tiles in the kernel).
constexpr int kPaceRelease = 12;
template <bool kDiag, class Release>
__device__ __forceinline__ float exp_pack(const uint32_t (&x)[2][32], int r, int key0, float scale_log2, float m_used,
                                          uint32_t (&pk)[2][16], Release release) {
  const uint64_t scale2 = pack2(scale_log2, scale_log2);
  const uint64_t negm2 = pack2(-m_used, -m_used);
  uint64_t sum_a = pack2(0.f, 0.f), sum_b = pack2(0.f, 0.f);
#pragma unroll
  for (int c = 0; c < 2; ++c) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const uint64_t t2 = fma2(pack2(__uint_as_float(x[c][2 * i]), __uint_as_float(x[c][2 * i + 1])), scale2, negm2);
      float p0, p1;
      if (kPolyEvery > 0 && (i % (kPolyEvery > 0 ? kPolyEvery : 1)) == kPolyEvery - 1) {
        exp2_poly2(t2, p0, p1);
      } else {
        float t0, t1;
        unpack2(t2, t0, t1);
        p0 = ex2(t0);
        p1 = ex2(t1);
      }
      if (kDiag) {
        if (key0 + c * 32 + 2 * i > r) p0 = 0.f;
        if (key0 + c * 32 + 2 * i + 1 > r) p1 = 0.f;
      }
      if (i & 1) {
        sum_a = add2(sum_a, pack2(p0, p1));
      } else {
        sum_b = add2(sum_b, pack2(p0, p1));
      }
      pk[c][i] = pack_bf16(p0, p1);
      if (c * 16 + i == kPaceRelease - 1) release(pk[c][i]);
    }
  }
  float s0, s1, s2, s3;
  unpack2(sum_a, s0, s1);
  unpack2(sum_b, s2, s3);
  return (s0 + s1) + (s2 + s3);
}

}  // namespace
}  // namespace crisp
