// Operands of the 8-bit product: e4m3 codes with one scale byte for each row and block of 128 columns.
// A byte b stands for 2^(b - 127); the scale is the smallest power of two >= 2^-126 that brings the block's largest finite
// magnitude within 448 = 1.75 * 2^8 (as in the cache), so that a division by it is exact and a code is rounded once.
#pragma once
#include <cstdint>
#include "common.cuh"
#include "softmax_rows.cuh"

namespace crisp {

constexpr int kScaleBlock = 128;   // columns per scale
constexpr int kScaleWord = 512;    // columns per 32-bit word of scales: rows of scales are whole words
constexpr uint8_t kScaleOne = 127;

inline int scale_words(int n_cols) { return (n_cols + kScaleWord - 1) / kScaleWord; }

#ifdef __CUDACC__
// The scale byte of a block with this largest finite magnitude, and one over the scale.
__device__ __forceinline__ uint32_t scale_byte(float amax, float& inverse) {
  const uint32_t bits = __float_as_uint(amax);
  int e = static_cast<int>(bits >> 23) - 135;         // amax in [2^(e + 8), 2^(e + 9))
  e += (bits & 0x7fffffu) > 0x600000u ? 1 : 0;        // above 1.75 * 2^(e + 8)
  e = max(e, -126);
  inverse = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
  return static_cast<uint32_t>(e + 127);
}
// Two values to two codes: nearest, ties to even, infinities to the largest, NaN to NaN.
__device__ __forceinline__ uint32_t pack_e4m3(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
// Largest finite magnitude of a block's 128 values, eight in each of 16 neighbouring lanes; NaN counts as nothing.
// Every lane of the warp calls it.
__device__ __forceinline__ float block_amax(const float (&y)[8]) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 8; i += 2) m = max3(m, fabsf(y[i]), fabsf(y[i + 1]));
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (__any_sync(0xffffffffu, m == INFINITY)) {   // rare: once more without the infinities
    m = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(y[i]) == INFINITY ? 0.f : fabsf(y[i]));
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  }
  return m;
}
__device__ __forceinline__ uint2 pack_codes(const float (&y)[8], float inverse) {
  float z[8];
#pragma unroll
  for (int i = 0; i < 8; i += 2) unpack2(mul2(pack2(y[i], y[i + 1]), pack2(inverse, inverse)), z[i], z[i + 1]);
  return make_uint2(pack_e4m3(z[0], z[1]) | pack_e4m3(z[2], z[3]) << 16, pack_e4m3(z[4], z[5]) | pack_e4m3(z[6], z[7]) << 16);
}
__device__ __forceinline__ void unpack_bf16(const uint4& w, float (&f)[8]) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(u[i] << 16);
    f[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
  }
}
#endif

int launch_quantize(const void* x, int n_rows, int n_cols, void* codes, uint8_t* scales, cudaStream_t stream);
int launch_rms_norm(const void* x, const void* residual, const void* weight, int n_rows, int n_cols, float eps, void* sum,
                    void* y, void* codes, uint8_t* scales, cudaStream_t stream);
int launch_rotary(const crisp_rotary_plan& plan, int n_tokens, const int32_t* positions, int first_position, int n_q_heads,
                  int n_kv_heads, const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                  int64_t v_stride, void* q_out, void* k_out, void* v_out, cudaStream_t stream);
int launch_matmul(const void* codes, const uint8_t* scales, const void* w_codes, const uint8_t* w_scales, int n_rows,
                  int n_out, int n_cols, void* out, void* ws, cudaStream_t stream);

constexpr int kMaxNormCols = 32768;      // a row is held in the registers of one CTA
constexpr int kMaxOperandSize = 1 << 28;  // rows and columns of an operand

// Tensor map of codes [rows][cols] with a {128, box_rows} box and 128-byte swizzle; what lies outside reads as zero.
int make_tmap_operand(CUtensorMap* out, const void* base, int rows, int cols, int box_rows);
// Tensor map of bf16 [rows][cols], cols a multiple of 8, with a {128, box_rows} box.
int make_tmap_product(CUtensorMap* out, void* base, int rows, int cols, int box_rows);

}  // namespace crisp
