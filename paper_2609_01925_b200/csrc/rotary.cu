// Rotary positions: token t's pairs of elements turn by position * frequency; bound by HBM (each element is read and written
// once; the cosines are computed once per token and pair and shared by the heads).
//
// Angles.  position * frequency in fp32 would be off by 2^-24 of up to 10^6 radians.  A frequency is held in turns per
// position as a 64-bit fraction instead: position * fraction modulo 2^64 is the angle modulo a whole turn, exactly, and its upper
// 32 bits go to sincospi within 2^-25 turns.
#include <cmath>

#include "cache.cuh"
#include "operand.cuh"

namespace crisp {
namespace {

constexpr int kItems = kHeadDim / 16;   // a thread's item: two vectors of 8 elements of a head
constexpr int kMaxRotaryThreads = 512;

struct Part {
  const char* in;
  char* out;
  int64_t in_stride;    // bytes per token
  int64_t out_stride;
  int heads;
};

struct RotaryArgs {
  crisp_rotary_plan plan;
  Part part[3];         // q, k, v
  const int32_t* positions;
  int n_tokens, first, items;   // items: of one token
};

template <int kTokens>
__global__ void __launch_bounds__(kMaxRotaryThreads) rotary_kernel(const __grid_constant__ RotaryArgs a) {
  __shared__ __align__(16) float2 turn[kTokens][kHeadDim / 2];   // (cosine, sine) of the CTA's tokens and pairs
  pdl_enter();
  const int pairs = a.plan.rotary_dim / 2;
  const int t0 = blockIdx.x * kTokens;
  for (int i = threadIdx.x; i < kTokens * (kHeadDim / 2); i += blockDim.x) {
    const int t = t0 + i / (kHeadDim / 2), p = i % (kHeadDim / 2);
    if (t >= a.n_tokens || p >= pairs) continue;
    const long long position = a.positions ? a.positions[t] : static_cast<long long>(a.first) + t;
    const uint64_t angle = a.plan.turns[p] * static_cast<uint64_t>(position);
    float s, c;
    sincospif(static_cast<float>(static_cast<int32_t>(angle >> 32)) * 0x1p-31f, &s, &c);
    turn[i / (kHeadDim / 2)][p] = make_float2(c * a.plan.magnitude, s * a.plan.magnitude);
  }
  __syncthreads();

  for (int item = threadIdx.x; item < a.items; item += blockDim.x) {
    const int j = item % kItems;
    int head = item / kItems, which = 0;
    while (which < 2 && head >= a.part[which].heads) head -= a.part[which++].heads;
    const Part part = a.part[which];
    const bool rotate = which < 2 && 16 * j < a.plan.rotary_dim;
    const bool half = rotate && a.plan.layout == CRISP_ROTARY_HALF;
    // byte offsets of the item's two vectors in the head
    const int at0 = half ? 16 * j : 32 * j, at1 = half ? 16 * j + 2 * pairs : 32 * j + 16;
    const char* in = part.in + t0 * part.in_stride + head * (kHeadDim * 2);
    char* out = part.out + t0 * part.out_stride + head * (kHeadDim * 2);
    uint4 x[kTokens], y[kTokens];
#pragma unroll
    for (int t = 0; t < kTokens; ++t) {
      if (t0 + t >= a.n_tokens) continue;
      x[t] = *reinterpret_cast<const uint4*>(in + t * part.in_stride + at0);
      y[t] = *reinterpret_cast<const uint4*>(in + t * part.in_stride + at1);
    }
#pragma unroll
    for (int t = 0; t < kTokens; ++t) {
      if (t0 + t >= a.n_tokens) continue;
      if (rotate) {
        float u[8], v[8], p[8], q[8];
        unpack_bf16(x[t], u);
        unpack_bf16(y[t], v);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float2 cs = turn[t][8 * j + i];
          const float first = half ? u[i] : (i < 4 ? u[2 * (i & 3)] : v[2 * (i & 3)]);
          const float second = half ? v[i] : (i < 4 ? u[2 * (i & 3) + 1] : v[2 * (i & 3) + 1]);
          p[i] = first * cs.x - second * cs.y;
          q[i] = second * cs.x + first * cs.y;
        }
        uint32_t lo[4], hi[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const __nv_bfloat162 l = half ? __floats2bfloat162_rn(p[2 * i], p[2 * i + 1]) : __floats2bfloat162_rn(p[i], q[i]);
          const __nv_bfloat162 h = half ? __floats2bfloat162_rn(q[2 * i], q[2 * i + 1]) : __floats2bfloat162_rn(p[4 + i], q[4 + i]);
          lo[i] = *reinterpret_cast<const uint32_t*>(&l);
          hi[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
        x[t] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
        y[t] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
      }
      *reinterpret_cast<uint4*>(out + t * part.out_stride + at0) = x[t];
      *reinterpret_cast<uint4*>(out + t * part.out_stride + at1) = y[t];
    }
  }
}

}  // namespace

int launch_rotary(const crisp_rotary_plan& plan, int n_tokens, const int32_t* positions, int first_position, int n_q_heads,
                  int n_kv_heads, const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                  int64_t v_stride, void* q_out, void* k_out, void* v_out, cudaStream_t stream) {
  RotaryArgs a;
  a.plan = plan;
  auto part = [](const void* in, int64_t stride, void* out, int heads) {
    return Part{static_cast<const char*>(in), static_cast<char*>(out), stride * 2, static_cast<int64_t>(heads) * kHeadDim * 2,
                in ? heads : 0};
  };
  a.part[0] = part(q, q_stride, q_out, n_q_heads);
  a.part[1] = part(k, k_stride, k_out, n_kv_heads);
  a.part[2] = part(v, v_stride, v_out, n_kv_heads);
  a.positions = positions;
  a.n_tokens = n_tokens;
  a.first = first_position;
  a.items = kItems * (a.part[0].heads + a.part[1].heads + a.part[2].heads);
  const int passes = (a.items + kMaxRotaryThreads - 1) / kMaxRotaryThreads;
  const int threads = ((a.items + passes - 1) / passes + 31) / 32 * 32;
  int n_sm = 0;
  const int rc = current_sm_count(&n_sm);
  if (rc != CRISP_OK) return rc;
  // four tokens per CTA share the search for an item's place and keep eight loads of a thread in flight; a few tokens are
  // spread over the SMs instead
  if (n_tokens > 4 * n_sm) {
    CRISP_KERNEL("rotary", stream, launch_pdl(rotary_kernel<4>, dim3((n_tokens - 1) / 4 + 1), dim3(threads), 0, stream, a));
  } else {
    CRISP_KERNEL("rotary", stream, launch_pdl(rotary_kernel<1>, dim3(n_tokens), dim3(threads), 0, stream, a));
  }
  CRISP_CUDA_TRY(cudaGetLastError(), "rotary: launch");
  return CRISP_OK;
}

}  // namespace crisp
