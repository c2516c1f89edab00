// Shared declarations of the two kernels of the product (matmul.cu, matmul_pair.cu).
#pragma once
#include "cache.cuh"
#include "matmul_wait.h"
#include "operand.cuh"

namespace crisp {

struct MatmulArgs {
  const uint8_t *scales, *w_scales;
  __nv_bfloat16* out;
  int* status;
  int n_rows, n_out, n_cols;
  int tile_tokens;       // tokens of a tile
  int n_feature_tiles, split, stages, tmem_cols;
  long long n_tiles;
  unsigned long long wait_ns;   // for a whole tile
};

constexpr int kPairTokens = 224;   // most tokens of a pair's tile: two accumulators and the scales fit TMEM's 512 columns

inline int ceil_div(int a, int b) { return (a + b - 1) / b; }

#ifdef __CUDACC__
// Four words of a row's scales, from word `at`; ones behind the end.
__device__ __forceinline__ void load_words(const uint8_t* scales, long long row, int rows, int words, int at, uint32_t (&w)[4]) {
  const uint32_t* p = reinterpret_cast<const uint32_t*>(scales) + row * words + at;
  if (row < rows && ((words | at) & 3) == 0 && (reinterpret_cast<uintptr_t>(scales) & 15) == 0) {
    const uint4 v = *reinterpret_cast<const uint4*>(p);
    w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = row < rows && at + i < words ? p[i] : 0x7f7f7f7fu;
  }
}
#endif

int launch_matmul_pair(MatmulArgs a, const void* codes, const void* w_codes, int tile_tokens, int n_sm, cudaStream_t stream);

}  // namespace crisp
