// What the two cache attention kernels share: the cut of all work into equal runs, one per CTA, and the joining of the
// partial results that a run leaves where it begins or ends inside a group.
//
// A unit is one page for one group (item, KV head, tile of rows); groups follow each other in one sequence, which is cut
// into runs of equal length (to one unit).  A run that begins or ends inside a group leaves a partial result, and a second
// small kernel (cache_join_kernel) joins them; launched behind the first one's start, it costs about 2 us.  (Joining in the
// kernel, by the CTA that arrives last, needs a fence, an atomic and two dependent loads per level, each a round trip
// through a loaded memory system: up to 16 us at the end of a 45 us kernel, measured.)  Which partials are added in which
// order depends on the sizes alone, so the same call gives the same bits.
#pragma once
#include "cache.cuh"
#include "sm100_ptx.cuh"

namespace crisp {
using namespace sm100;

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

// What the join kernel has to do for the group whose first partial CTA c holds (a CTA holds the first partial of at most
// one group: it lies behind the CTA's other groups, or the group is all that the CTA works on).
struct JoinDesc {
  int rows;        // 0: nothing
  int count;       // partials: slot `first`, then the slots 2 (c + 1), 2 (c + 2), ...
  int first;
  int t0, head, row0;
};

// Partial results: two slots per CTA (2 c for a run that begins at the CTA's first unit, 2 c + 1 for one that begins
// later), each with `rows` rows of 128 and their maximum (log2; short of Output's unit_bits) and sum.
struct Partials {
  JoinDesc* desc;  // [ctas]
  float2* ml;
  float* o;
  int ctas, rows;
};
inline Partials carve_partials(void* ws, size_t* off, int ctas, int rows) {
  uint8_t* base = static_cast<uint8_t*>(ws);
  Partials w;
  w.ctas = ctas;
  w.rows = rows;
  w.desc = reinterpret_cast<JoinDesc*>(base + *off);
  *off += align_up(sizeof(JoinDesc) * static_cast<size_t>(ctas), 256);
  w.ml = reinterpret_cast<float2*>(base + *off);
  *off += align_up(sizeof(float2) * 2 * static_cast<size_t>(ctas) * rows, 256);
  w.o = reinterpret_cast<float*>(base + *off);
  *off += align_up(sizeof(float) * 2 * static_cast<size_t>(ctas) * rows * kHeadDim, 256);
  return w;
}

// Where the result goes.
struct Output {
  __nv_bfloat16* o;
  float* lse;
  int n_q_heads, group, n_tokens;
  float unit_bits;  // values and sums stand in units of 2^(maximum + unit_bits)
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
    out.lse[static_cast<size_t>(h) * out.n_tokens + token] = sum == 0.f ? -INFINITY : (top + out.unit_bits) * 0.6931471805599453f + logf(sum);
}

namespace {

// slot of CTA c's partial result of the group whose first unit is g0 and first CTA is cf
__device__ __forceinline__ int partial_slot(const Cut& cut, int g0, int cf, int c) {
  return 2 * c + (c == cf && cut.first(c) < g0 ? 1 : 0);
}

// The join kernel's work for a group of which this CTA holds the first partial; rows = 0 in any other case.
__device__ __forceinline__ JoinDesc join_desc(const Cut& cut, const Segment& g, int cta, int t0, int row0, int rows) {
  JoinDesc d = {0, 0, 0, 0, 0, 0};
  const int cf = cut.cta_of(g.g0);
  if (cf == cta && !(g.p0 == 0 && g.p1 == g.pages))
    d = JoinDesc{rows, cut.cta_of(g.g0 + g.pages - 1) - cf + 1, partial_slot(cut, g.g0, cf, cf), t0, g.head, row0};
  return d;
}

}  // namespace

int launch_cache_join(const Partials& w, const Output& out, int max_rows, int ctas, cudaStream_t stream);

}  // namespace crisp
