// Shared declarations of the two kernels of the product (matmul.cu, matmul_pair.cu).
#pragma once
#include "cache.cuh"
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
};

inline int ceil_div(int a, int b) { return (a + b - 1) / b; }

int launch_matmul_pair(MatmulArgs a, const void* codes, const void* w_codes, int tile_tokens, int n_sm, cudaStream_t stream);

}  // namespace crisp
