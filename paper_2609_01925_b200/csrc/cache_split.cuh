// What the two cache attention kernels share: the cut of all work into equal runs, one per CTA, and the joining of the
// partial results that a run leaves where it begins or ends inside a group.
//
// A unit is one page for one group (item, KV head, tile of rows); groups follow each other in one sequence, which is cut
// into runs of equal length (to one unit).  A group that lies in several CTAs is joined by the CTA that completes it: first
// within sets of kSet CTAs, then the sets' results, so a single long sequence is not joined by one CTA alone.  Which
// partials are added in which order depends on the sizes alone, so the same call gives the same bits.
#pragma once
#include "cache.cuh"
#include "sm100_ptx.cuh"

namespace crisp {
using namespace sm100;
namespace {

constexpr int kSet = 16;

struct Cut {
  int units, ctas, each, extra;  // the first `extra` CTAs run each + 1 units, the others `each`
  __device__ __forceinline__ Cut(int units_, int most) {
    units = units_;
    ctas = units_ < most ? units_ : most;
    each = ctas > 0 ? units_ / ctas : 0;
    extra = units_ - each * ctas;
  }
  __device__ __forceinline__ int first(int cta) const { return cta * each + min(cta, extra); }
  __device__ __forceinline__ int cta_of(int u) const {
    const int big = extra * (each + 1);
    return u < big ? u / (each + 1) : extra + (u - big) / each;
  }
};

// A run of pages [p0, p1) of one group of `pages` pages; g0 is the unit of the group's first page.
struct Segment {
  int item, head, tile, p0, p1, pages, g0;
};

// Partial results: two slots per CTA (2 c for a run that begins at the CTA's first unit, 2 c + 1 for one that begins
// later), each with `rows` rows of 128 and their maximum (log2 units) and sum.
struct Partials {
  int* counters;  // [2][2 * ctas]: arrivals within a set, and of sets; zero between calls
  int n_slots;    // 2 * ctas
  float2* ml;
  float* o;
  int rows;
};

// Where the result goes.
struct Output {
  __nv_bfloat16* o;
  float* lse;
  int n_q_heads, group, n_tokens;
};
__device__ __forceinline__ void write_row(const Output& out, int t0, int head, int row, int lane, const float4& acc,
                                          float top, float sum) {
  const size_t token = static_cast<size_t>(t0) + row / out.group;
  const int h = head * out.group + row % out.group;
  const float inv = sum == 0.f ? 0.f : 1.0f / sum;
  uint2 v;
  v.x = pack_bf16(acc.x * inv, acc.y * inv);
  v.y = pack_bf16(acc.z * inv, acc.w * inv);
  reinterpret_cast<uint2*>(out.o + (token * out.n_q_heads + h) * kHeadDim)[lane] = v;
  if (out.lse && lane == 0)
    out.lse[static_cast<size_t>(h) * out.n_tokens + token] = sum == 0.f ? -INFINITY : top * 0.6931471805599453f + logf(sum);
}

// Joins `count` <= 32 partial results, row by row: a warp per row, four dims per lane.  Partial 0 lies in first_slot,
// partial j in slot 2 * (next + (j - 1) * stride).  final_: writes the output; otherwise first_slot gets the result.
template <int kWarps>
__device__ void join(const Partials& w, const Output& out, int t0, int head, int row0, int rows, int first_slot, int next,
                     int stride, int count, bool final_) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  auto slot_of = [&](int j) { return j == 0 ? first_slot : 2 * (next + (j - 1) * stride); };
  const int my_slot = slot_of(lane < count ? lane : 0);
  for (int r = warp; r < rows; r += kWarps) {
    const float2 ml = __ldcg(&w.ml[static_cast<size_t>(my_slot) * w.rows + r]);
    const float m = lane < count ? ml.x : -INFINITY;
    float top = m;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const float f = m == -INFINITY ? 0.f : ex2(m - top);
    float sum = f == 0.f ? 0.f : ml.y * f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    const float4* base = reinterpret_cast<const float4*>(w.o + static_cast<size_t>(r) * kHeadDim) + lane;
    const size_t slot_stride = static_cast<size_t>(w.rows) * (kHeadDim / 4);
#pragma unroll 1
    for (int j0 = 0; j0 < count; j0 += 8) {
      float4 x[8];
      float fj[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int at = min(j0 + j, count - 1);
        fj[j] = __shfl_sync(0xffffffffu, f, at);
        if (j0 + j >= count) fj[j] = 0.f;
        x[j] = __ldcg(base + slot_of(at) * slot_stride);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        acc.x = fmaf(fj[j], x[j].x, acc.x);
        acc.y = fmaf(fj[j], x[j].y, acc.y);
        acc.z = fmaf(fj[j], x[j].z, acc.z);
        acc.w = fmaf(fj[j], x[j].w, acc.w);
      }
    }
    if (final_) {
      write_row(out, t0, head, row0 + r, lane, acc, top, sum);
    } else {
      reinterpret_cast<float4*>(w.o + (static_cast<size_t>(first_slot) * w.rows + r) * kHeadDim)[lane] = acc;
      if (lane == 0) w.ml[static_cast<size_t>(first_slot) * w.rows + r] = make_float2(top, sum);
    }
  }
}

// One more of `count` arrivals at a counter; true, for all threads of the group, at the last one, which resets it.
template <int kGroupThreads>
__device__ __forceinline__ bool arrive_last(int* shared_flag, int* counter, int count) {
  __threadfence();
  named_bar_sync(1, kGroupThreads);
  if (threadIdx.x == 0) {
    const bool last = atomicAdd(counter, 1) == count - 1;
    if (last) *counter = 0;
    *shared_flag = last;
  }
  named_bar_sync(1, kGroupThreads);
  const bool last = *shared_flag != 0;
  if (last) __threadfence();
  return last;
}

// slot of CTA c's partial result of the group whose first unit is g0 and first CTA is cf
__device__ __forceinline__ int partial_slot(const Cut& cut, int g0, int cf, int c) {
  return 2 * c + (c == cf && cut.first(c) < g0 ? 1 : 0);
}

// Called by the threads of a group of kWarps warps (threads 0 ..) once this CTA's partial of the group is written.
template <int kWarps>
__device__ void finish_partial(const Cut& cut, const Segment& g, int cta, const Partials& w, const Output& out, int t0,
                               int row0, int rows, int* shared_flag) {
  const int cf = cut.cta_of(g.g0), cl = cut.cta_of(g.g0 + g.pages - 1);
  const int set0 = cta / kSet * kSet;
  const int f = max(cf, set0), e = min(cl, set0 + kSet - 1);
  const int sets = cl / kSet - cf / kSet + 1;
  if (e > f) {
    const int slot = partial_slot(cut, g.g0, cf, f);
    if (!arrive_last<32 * kWarps>(shared_flag, w.counters + slot, e - f + 1)) return;
    join<kWarps>(w, out, t0, g.head, row0, rows, slot, f + 1, 1, e - f + 1, sets == 1);
  }
  if (sets > 1) {
    const int slot = partial_slot(cut, g.g0, cf, cf);
    if (!arrive_last<32 * kWarps>(shared_flag, w.counters + w.n_slots + slot, sets)) return;
    join<kWarps>(w, out, t0, g.head, row0, rows, slot, (cf / kSet + 1) * kSet, kSet, sets, true);
  }
}

}  // namespace
}  // namespace crisp
