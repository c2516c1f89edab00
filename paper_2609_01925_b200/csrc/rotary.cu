// Rotary positions: token t's pairs of elements turn by position * frequency; bound by HBM (each element is read and written
// once; the cosines are computed once per token and pair and shared by the heads).
//
// 131072 tokens of 32/8 heads, 3.2 GB: 462 us, 7.0 TB/s; 5003 of 28/4 heads, a half of each rotated, 92 MB: 12.1 us.
//
// Angles.  position * frequency in fp32 would be off by 2^-24 of up to 10^6 radians.  A frequency is held in turns per
// position as a 64-bit fraction instead: position * fraction modulo 2^64 is the angle modulo a whole turn, exactly, and its upper
// 32 bits go to sincospi within 2^-25 turns.
#include <cmath>

#include "cache.cuh"
#include "operand.cuh"
#include "sm100_ptx.cuh"

namespace crisp {
namespace {

constexpr int kItems = kHeadDim / 16;   // a thread's item: two vectors of 8 elements of a head
constexpr int kMaxRotaryThreads = 512;
constexpr int kTurnRow = 82;            // (cosine, sine) of a token's 64 pairs, two places free behind eight (see turn_place), and two
constexpr int kMaxGroups = 16;          // groups of tokens of a CTA, where a token has few heads

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

// Where pair p's cosine and sine are in a token's row.  The eight items of a head read eight pairs each, 64 bytes apart, which would
// be four to a bank; 80 bytes apart they meet no other.
__device__ __forceinline__ int turn_place(int p) { return p + p / 8 * 2; }

// Two elements (8 bytes of bf16 pairs make a vector of 16) turned by (cosine, sine).
__device__ __forceinline__ uint32_t turn_pair(uint32_t w, float2 cs) {
  const float a = __uint_as_float(w << 16), b = __uint_as_float(w & 0xffff0000u);
  return sm100::pack_bf16(a * cs.x - b * cs.y, b * cs.x + a * cs.y);
}
__device__ __forceinline__ uint4 turn_vector(const uint4& w, const float2* cs) {
  const float4 a = reinterpret_cast<const float4*>(cs)[0], b = reinterpret_cast<const float4*>(cs)[1];
  return make_uint4(turn_pair(w.x, make_float2(a.x, a.y)), turn_pair(w.y, make_float2(a.z, a.w)),
                    turn_pair(w.z, make_float2(b.x, b.y)), turn_pair(w.w, make_float2(b.z, b.w)));
}

// A CTA has blockDim.y groups of kTokens tokens; a thread takes items of its group's tokens, kTokens at a time.  kOnce: the input is
// read with a hint that it will not be read again.
template <int kTokens, bool kOnce>
__global__ void __launch_bounds__(kMaxRotaryThreads, kTokens == 4 ? 2 : 3) rotary_kernel(const __grid_constant__ RotaryArgs a) {
  extern __shared__ __align__(16) float2 turns[];   // [group][kTokens][kTurnRow]
  pdl_enter();
  const int pairs = a.plan.rotary_dim / 2;
  const int cta_tokens = kTokens * static_cast<int>(blockDim.y);
  const long long first_token = static_cast<long long>(blockIdx.x) * cta_tokens;
  const long long t0 = first_token + static_cast<long long>(threadIdx.y) * kTokens;
  const int here = static_cast<int>(min(static_cast<long long>(kTokens), a.n_tokens - t0));   // of the group's tokens; may be < 1

  // The item's two vectors of the head's 16: those whose elements are pairs (both), or j and j + 8, so that neighbouring threads
  // have neighbouring vectors (interleaved, and what is copied).
  bool both, turn0, turn1;
  int v0, v1;
  char* out;
  int64_t out_stride;
  uint4 x[kTokens], y[kTokens];
  auto fetch = [&](int item) {
    const int j = item % kItems;
    int head = item / kItems, which = 0;
    while (which < 2 && head >= a.part[which].heads) head -= a.part[which++].heads;
    const Part& part = a.part[which];
    const bool half = a.plan.layout == CRISP_ROTARY_HALF && which < 2;
    both = half && 16 * j < a.plan.rotary_dim;
    v0 = both ? j : half ? 2 * j : j;
    v1 = both ? j + pairs / 8 : half ? 2 * j + 1 : j + 8;
    turn0 = !half && which < 2 && 8 * v0 < a.plan.rotary_dim;
    turn1 = !half && which < 2 && 8 * v1 < a.plan.rotary_dim;
    out = part.out + t0 * part.out_stride + head * (kHeadDim * 2);
    out_stride = part.out_stride;
    const char* in = part.in + t0 * part.in_stride + head * (kHeadDim * 2);
    auto load = [](const char* p) {
      const uint4* v = reinterpret_cast<const uint4*>(p);
      return kOnce ? __ldcs(v) : *v;
    };
#pragma unroll
    for (int t = 0; t < kTokens; ++t) {
      if (t >= here) continue;
      x[t] = load(in + t * part.in_stride + 16 * v0);
      y[t] = load(in + t * part.in_stride + 16 * v1);
    }
  };
  // the first items are on their way while the cosines are computed
  if (static_cast<int>(threadIdx.x) < a.items) fetch(threadIdx.x);
  // (neighbouring threads have the same pair where they can: the table is in constant memory, which reads one place at a time)
  for (int i = threadIdx.y * blockDim.x + threadIdx.x; i < cta_tokens * pairs; i += blockDim.x * blockDim.y) {
    const int p = i / cta_tokens, token = i - p * cta_tokens;
    const long long t = first_token + token;
    if (t >= a.n_tokens) continue;
    const long long position = a.positions ? a.positions[t] : static_cast<long long>(a.first) + t;
    const uint64_t angle = a.plan.turns[p] * static_cast<uint64_t>(position);
    float s, c;
    sincospif(static_cast<float>(static_cast<int32_t>(angle >> 32)) * 0x1p-31f, &s, &c);
    turns[token * kTurnRow + turn_place(p)] = make_float2(c * a.plan.magnitude, s * a.plan.magnitude);
  }
  __syncthreads();

  const float2* turn = turns + threadIdx.y * (kTokens * kTurnRow);
  for (int item = threadIdx.x; item < a.items; item += blockDim.x) {
    if (item != static_cast<int>(threadIdx.x)) fetch(item);
#pragma unroll
    for (int t = 0; t < kTokens; ++t) {
      if (t >= here) continue;
      const float2* cs = turn + t * kTurnRow;
      if (both) {
        float u[8], v[8], p[8], q[8];
        unpack_bf16(x[t], u);
        unpack_bf16(y[t], v);
        const float4* c4 = reinterpret_cast<const float4*>(cs + turn_place(8 * v0));   // two pairs each
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float4 two = c4[i / 2];
          const float2 c = i & 1 ? make_float2(two.z, two.w) : make_float2(two.x, two.y);
          p[i] = u[i] * c.x - v[i] * c.y;
          q[i] = v[i] * c.x + u[i] * c.y;
        }
        x[t] = make_uint4(sm100::pack_bf16(p[0], p[1]), sm100::pack_bf16(p[2], p[3]), sm100::pack_bf16(p[4], p[5]),
                          sm100::pack_bf16(p[6], p[7]));
        y[t] = make_uint4(sm100::pack_bf16(q[0], q[1]), sm100::pack_bf16(q[2], q[3]), sm100::pack_bf16(q[4], q[5]),
                          sm100::pack_bf16(q[6], q[7]));
      }
      if (turn0) x[t] = turn_vector(x[t], cs + turn_place(4 * v0));
      if (turn1) y[t] = turn_vector(y[t], cs + turn_place(4 * v1));
      *reinterpret_cast<uint4*>(out + t * out_stride + 16 * v0) = x[t];
      *reinterpret_cast<uint4*>(out + t * out_stride + 16 * v1) = y[t];
    }
  }
}

template <int kTokens, bool kOnce>
void launch_tokens(const RotaryArgs& a, cudaStream_t stream) {
  const int passes = (a.items + kMaxRotaryThreads - 1) / kMaxRotaryThreads;
  const int across = (a.items + passes - 1) / passes;
  int groups = kTokens == 1 ? 1 : 384 / across;   // CTAs of some 384 threads
  groups = groups < 1 ? 1 : groups > kMaxGroups ? kMaxGroups : groups;
  const long long tokens = static_cast<long long>(kTokens) * groups;
  const dim3 grid(static_cast<unsigned>((a.n_tokens + tokens - 1) / tokens));
  const dim3 block(groups == 1 ? (across + 31) / 32 * 32 : across, groups);
  CRISP_KERNEL("rotary", stream, launch_pdl(rotary_kernel<kTokens, kOnce>, grid, block, tokens * kTurnRow * sizeof(float2),
                                            stream, a));
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
  int n_sm = 0;
  const int rc = current_sm_count(&n_sm);
  if (rc != CRISP_OK) return rc;
  // Four tokens at a time keep eight loads of a thread in flight (131072 tokens of 32/8 heads: 462 us; two: 509 in an earlier build
  // whose four took 490).  Where input and output fit L2, two at a time, read once, are ahead (5003 tokens of 28/4 heads: 12.1 us; in
  // that build 14.6, and 15.9 with four, kept), and a few tokens are spread over the SMs.
  const long long bytes = static_cast<long long>(n_tokens) * a.items * 64;
  if (n_tokens <= 4 * n_sm) {
    launch_tokens<1, false>(a, stream);
  } else if (bytes <= 120ll << 20) {
    launch_tokens<2, true>(a, stream);
  } else {
    launch_tokens<4, false>(a, stream);
  }
  CRISP_CUDA_TRY(cudaGetLastError(), "rotary: launch");
  return CRISP_OK;
}

}  // namespace crisp
