// Joins the partial results of the cache attention kernels (cache_split.cuh).
//
// O = sum_j 2^(m_j - M) O_j / sum_j 2^(m_j - M) l_j over the partials j of a row, M = max_j m_j.  A few hundred KB to a few
// MB in all: what counts is the length of the chain of dependent loads and how many warps an SM holds.  So a warp takes
// four partials of a row at a time, maxima and values in flight together (each batch is one step of an online softmax), and
// with more than four, four warps share a row, take every fourth partial each, and meet in shared memory.  (Eight at a time
// cost registers and with them two thirds of the warps: 1.7 us more in the smallest call, 10 us more in a call of 285 us.)
#include "cache_split.cuh"

namespace crisp {
namespace {

constexpr int kWarps = 16, kBatch = 4;

struct Row {
  float m = -INFINITY, l = 0.f;
  float4 acc = {0.f, 0.f, 0.f, 0.f};
  __device__ __forceinline__ void scale(float top) {
    const float f = m == -INFINITY ? 0.f : ex2(m - top);
    m = top;
    l *= f;
    acc = make_float4(acc.x * f, acc.y * f, acc.z * f, acc.w * f);
  }
  __device__ __forceinline__ void add(float m_in, float l_in, const float4& x) {
    if (m_in == -INFINITY) return;  // saw nothing, or is not there
    const float f = ex2(m_in - m);
    l = fmaf(l_in, f, l);
    acc.x = fmaf(x.x, f, acc.x);
    acc.y = fmaf(x.y, f, acc.y);
    acc.z = fmaf(x.z, f, acc.z);
    acc.w = fmaf(x.w, f, acc.w);
  }
};

// kRowWarps warps per row; the CTA takes 16 / kRowWarps rows at a time.
template <int kRowWarps>
__device__ __forceinline__ void join_rows(const Partials& w, const Output& out, const JoinDesc& d, float4 (*s_acc)[32],
                                          float2* s_ml) {
  constexpr int kRows = kWarps / kRowWarps;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, part = warp % kRowWarps, row_at = warp / kRowWarps;
  for (int r0 = blockIdx.y * kRows; r0 < d.rows; r0 += gridDim.y * kRows) {
    const int r = r0 + row_at;
    Row row;
    if (r < d.rows) {
      for (int j0 = part; j0 < d.count; j0 += kRowWarps * kBatch) {
        float4 x[kBatch];
        float2 ml[kBatch];
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
          const int j = j0 + k * kRowWarps;
          ml[k] = make_float2(-INFINITY, 0.f);
          if (j < d.count) {
            const size_t at = static_cast<size_t>(j == 0 ? d.first : 2 * (blockIdx.x + j)) * w.rows + r;
            ml[k] = __ldg(&w.ml[at]);
            x[k] = __ldg(reinterpret_cast<const float4*>(w.o + at * kHeadDim) + lane);
          }
        }
        float top = row.m;
#pragma unroll
        for (int k = 0; k < kBatch; ++k) top = fmaxf(top, ml[k].x);
        row.scale(top);
#pragma unroll
        for (int k = 0; k < kBatch; ++k) row.add(ml[k].x, ml[k].y, x[k]);
      }
    }
    if (kRowWarps > 1) {
      s_acc[warp][lane] = row.acc;
      if (lane == 0) s_ml[warp] = make_float2(row.m, row.l);
      __syncthreads();
      if (part == 0) {
        float top = row.m;
#pragma unroll
        for (int i = 1; i < kRowWarps; ++i) top = fmaxf(top, s_ml[warp + i].x);
        row.scale(top);
#pragma unroll
        for (int i = 1; i < kRowWarps; ++i) row.add(s_ml[warp + i].x, s_ml[warp + i].y, s_acc[warp + i][lane]);
      }
    }
    if (part == 0 && r < d.rows) write_row(out, d.t0, d.head, d.row0 + r, lane, row.acc, row.m, row.l);
    if (kRowWarps > 1) __syncthreads();
  }
}

__global__ void __launch_bounds__(32 * kWarps, 3)
cache_join_kernel(const Partials w, const Output out) {
  pdl_enter();
  __shared__ float4 s_acc[kWarps][32];
  __shared__ float2 s_ml[kWarps];
  const JoinDesc d = w.desc[blockIdx.x];
  if (d.count <= kBatch)
    join_rows<1>(w, out, d, s_acc, s_ml);
  else
    join_rows<4>(w, out, d, s_acc, s_ml);
}

}  // namespace

int launch_cache_join(const Partials& w, const Output& out, int max_rows, int ctas, cudaStream_t stream) {
  const int chunks = (max_rows + 3) / 4;  // rows are few, or the partials of a row are
  CRISP_KERNEL("cache_join", stream, launch_pdl(cache_join_kernel, dim3(ctas, chunks < 16 ? chunks : 16), dim3(32 * kWarps),
                                                0, stream, w, out));
  CRISP_CUDA_TRY(cudaGetLastError(), "cache_attention: launch of the join");
  return CRISP_OK;
}

}  // namespace crisp
