// Causal attention of a few new tokens over the 8-bit paged cache (answering token by token, verifying a draft).
//
// Every cached byte is needed once per (item, KV head), for the G = H_q / H_kv query heads and the item's new tokens
// together (the rows of a group), so the kernel is bound by reading the codes from HBM.  What follows from that:
//  * One unit of work is one page of one KV head (16 KB of K codes, 16 KB of V codes, by TMA into a ring of slots).
//    The units of all items and heads form one sequence that is cut into equal runs, one per CTA, whatever the
//    lengths are; a run that begins or ends inside a group leaves a partial result (maximum, sum, O) in the workspace,
//    and the CTA that completes a set of partials joins them: first within sets of 16 CTAs, then the sets' results, so
//    a single long sequence is not joined by one CTA alone.  The order of every sum is fixed by the sizes.
//  * Codes are not converted in bulk: a warp takes its fragments from shared memory, converts them in registers and
//    multiplies with m16n8k16 (fp16 in, fp32 out).  Products are computed transposed, S^T = K Q^T and O^T = V^T P^T, so
//    that the padded dimension, N = 8, is the few query rows.  (tcgen05 has no shape for so few rows without
//    the codes going through shared memory a second time, and the tensor pipe is not what bounds this kernel.)
//    fp16 holds every code of both formats exactly; Q is brought to fp16 by a power of two per row (exact but for
//    elements 2^-29 below the row's largest), P in [0, 1] is rounded to fp16's 11 bits, everything else is fp32.
//  * The order of the dims inside a dot product and of the keys inside P V is free.  A thread therefore reads whole
//    16-byte chunks, and which chunk belongs to which fragment row is chosen so that the eight threads of a
//    shared-memory phase always touch eight different 16-byte banks of the 128-byte-swizzled tile.
//  * Scales are one per page and head: K's multiplies the logits, V's the page's P V product (O is accumulated in
//    fp32 per page, which also applies the running maximum's correction).
#include <cuda_fp16.h>

#include "cache.cuh"
#include "sm100_ptx.cuh"

namespace crisp {
using namespace sm100;

namespace {

constexpr int kSlots = 4;            // ring slots of one K or V tile
constexpr int kWarps = 4;            // consumer warps: 32 tokens of a page each
constexpr int kThreads = kWarps * 32 + 32;
constexpr int kMaxCtas = 512;        // bound on the grid; sizes the workspace
constexpr int kMaxRows = 16;         // rows of a partial result
constexpr int kSet = 16;             // CTAs whose partials are joined first

struct AttnWs {
  int* status;
  int* counters;   // [2][2 * kMaxCtas]: arrivals within a set, and of sets
  float2* part_ml; // [2 * kMaxCtas][kMaxRows] running maximum (log2 units) and sum
  float* part_o;   // [2 * kMaxCtas][kMaxRows][128]
};
AttnWs carve(void* ws, size_t* total) {
  uint8_t* base = static_cast<uint8_t*>(ws);
  AttnWs w;
  w.status = reinterpret_cast<int*>(base);
  size_t off = kWsHeader;
  w.counters = reinterpret_cast<int*>(base + off);
  off += sizeof(int) * 4 * kMaxCtas;
  w.part_ml = reinterpret_cast<float2*>(base + off);
  off += sizeof(float2) * 2 * kMaxCtas * kMaxRows;
  w.part_o = reinterpret_cast<float*>(base + off);
  off += sizeof(float) * 2 * kMaxCtas * kMaxRows * kHeadDim;
  *total = off;
  return w;
}

struct AttnArgs {
  CacheView c;
  CacheBatch b;
  int layer, n_q_heads, group;
  float scale_log2;
  const __nv_bfloat16* q;
  __nv_bfloat16* o;
  float* lse;
  AttnWs w;
};

struct DecodeSmem {
  alignas(1024) uint8_t ring[kSlots][kPageTileBytes];
  float red[kWarps][8][kHeadDim];  // the warps' O of eight rows
  float red_m[kWarps][kMaxRows], red_l[kWarps][kMaxRows];
  float scale[kSlots];
  uint64_t full[kSlots], empty[kSlots];
  int4 items[kMaxCacheBatch];      // seq, len, t0, n
  int start[kMaxCacheBatch + 1];   // units of one head before item i
  long long scratch[33];
  int abort_flag;
  int last;
};

__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
// Four codes (bytes 0, 1 and 2, 3 of w) to two pairs of fp16, exactly.
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

// A run of pages of one group (item, KV head, tile of rows), and where its neighbours are.
struct Segment {
  int item, head, tile;
  int p0, p1;            // pages [p0, p1) of the group's `pages`
  int pages;
  long long g0;          // first unit of the group
};

struct Cut {
  long long units;
  int ctas;
  __device__ __forceinline__ long long first(int cta) const { return cta * units / ctas; }
  __device__ __forceinline__ int cta_of(long long u) const { return static_cast<int>(((u + 1) * ctas - 1) / units); }
};

template <int kRowTile>
__device__ __forceinline__ int row_tiles(int n, int group) { return (n * group + kRowTile - 1) / kRowTile; }

template <int kRowTile>
__device__ __forceinline__ Segment segment_at(const DecodeSmem& s, const AttnArgs& a, long long u, long long end) {
  Segment g;
  const int heads = a.c.heads;
  int lo = 0, hi = a.b.batch;
  const int key = static_cast<int>(u / heads);
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (s.start[mid] <= key) lo = mid; else hi = mid;
  }
  g.item = lo;
  const int4 it = s.items[lo];
  g.pages = max(1, pages_of(it.y));  // an empty sequence still has rows to write
  const int tiles = row_tiles<kRowTile>(it.w, a.group);
  const int rem = static_cast<int>(u - static_cast<long long>(s.start[lo]) * heads);  // < 2^31: see the check of the total
  g.head = rem / (g.pages * tiles);
  const int in_head = rem - g.head * g.pages * tiles;
  g.tile = in_head / g.pages;
  g.p0 = in_head - g.tile * g.pages;
  g.g0 = u - g.p0;
  const long long left = end - u;
  g.p1 = g.pages - g.p0 <= left ? g.pages : g.p0 + static_cast<int>(left);
  return g;
}

// Joins `count` partial results (slots first_slot, then 2 * (next + j * stride) ..) row by row: a warp per row, four
// dims per lane.  final: writes O and lse; otherwise the joined partial goes to first_slot.
template <int kRowTile>
__device__ void join(const AttnArgs& a, const CacheItem& it, const Segment& g, int first_slot, int next, int stride,
                     int count, bool final_) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rows = min(kRowTile, it.n * a.group - g.tile * kRowTile);
  auto slot_of = [&](int j) { return j == 0 ? first_slot : 2 * (next + (j - 1) * stride); };
  for (int r = warp; r < rows; r += kWarps) {
    float m = -INFINITY, l = 0.f;
    if (lane < count) {
      const float2 ml = __ldcg(&a.w.part_ml[slot_of(lane) * kMaxRows + r]);
      m = ml.x;
      l = ml.y;
    }
    float top = m;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const float w = m == -INFINITY ? 0.f : exp2f(m - top);
    float sum = l * w;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
    for (int j = 0; j < count; ++j) {
      const float wj = __shfl_sync(0xffffffffu, w, j);
      const float4 x = __ldcg(reinterpret_cast<const float4*>(
                                  a.w.part_o + (static_cast<size_t>(slot_of(j)) * kMaxRows + r) * kHeadDim) + lane);
      acc.x = fmaf(wj, x.x, acc.x);
      acc.y = fmaf(wj, x.y, acc.y);
      acc.z = fmaf(wj, x.z, acc.z);
      acc.w = fmaf(wj, x.w, acc.w);
    }
    if (final_) {
      const int row = g.tile * kRowTile + r;
      const size_t token = static_cast<size_t>(it.t0) + row / a.group;
      const int h = g.head * a.group + row % a.group;
      const float inv = top == -INFINITY ? 0.f : 1.0f / sum;
      uint2 v;
      v.x = pack_bf16(acc.x * inv, acc.y * inv);
      v.y = pack_bf16(acc.z * inv, acc.w * inv);
      reinterpret_cast<uint2*>(a.o + (token * a.n_q_heads + h) * kHeadDim)[lane] = v;
      if (a.lse && lane == 0)
        a.lse[static_cast<size_t>(h) * a.b.n_tokens + token] =
            top == -INFINITY ? -INFINITY : top * 0.6931471805599453f + logf(sum);
    } else {
      reinterpret_cast<float4*>(a.w.part_o + (static_cast<size_t>(first_slot) * kMaxRows + r) * kHeadDim)[lane] = acc;
      if (lane == 0) a.w.part_ml[first_slot * kMaxRows + r] = make_float2(top, sum);
    }
  }
}

// One more of `count` arrivals at a counter; true (for the whole consumer group) for the last, which resets it.
__device__ __forceinline__ bool arrive_last(DecodeSmem& s, int* counter, int count) {
  __threadfence();
  named_bar_sync(1, kWarps * 32);
  if (threadIdx.x == 0) {
    const bool last = atomicAdd(counter, 1) == count - 1;
    if (last) *counter = 0;
    s.last = last;
  }
  named_bar_sync(1, kWarps * 32);
  const bool last = s.last != 0;
  if (last) __threadfence();
  return last;
}

template <int kFormat, int kTilesN>
__global__ void __launch_bounds__(kThreads, 2)
cache_decode_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v, const AttnArgs a) {
  constexpr int kRowTile = 8 * kTilesN;
  pdl_enter();
  extern __shared__ uint8_t smem_raw[];
  DecodeSmem& s = *reinterpret_cast<DecodeSmem*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int heads = a.c.heads, batch = a.b.batch;
  if (tid == 0) {
    s.abort_flag = 0;
    for (int i = 0; i < kSlots; ++i) {
      mbar_init(&s.full[i], 1);
      mbar_init(&s.empty[i], kWarps);
    }
    fence_mbar_init();
  }
  // ---- every CTA reads the batch and counts the units before each item
  long long carry = 0;
  for (int base = 0; base < batch; base += kThreads) {
    const int i = base + tid;
    int units = 0;
    if (i < batch) {
      const CacheItem it = load_item(a.c, a.b, i, a.w.status);
      s.items[i] = make_int4(it.seq, it.len, it.t0, it.seq < 0 ? 0 : it.n);
      if (it.seq >= 0) units = max(1, pages_of(it.len)) * row_tiles<kRowTile>(it.n, a.group);
    }
    long long total;
    const long long before = block_exclusive_scan<kThreads>(units, s.scratch, &total);
    if (i < batch) s.start[i] = static_cast<int>(min(carry + before, 0x7fffffffLL));
    carry += total;
  }
  __syncthreads();
  if (carry * heads > 0x7fffffffLL) {  // an item's units are counted in 32 bits
    if (tid == 0) cache_fail(a.w.status, CRISP_ERR_BAD_CACHE);
    return;
  }
  Cut cut;
  cut.units = carry * heads;
  cut.ctas = static_cast<int>(min(static_cast<long long>(gridDim.x), cut.units));
  const int cta = blockIdx.x;
  if (cta >= cut.ctas) return;
  const long long u0 = cut.first(cta), u1 = cut.first(cta + 1);
  volatile int* abort_flag = &s.abort_flag;

  if (warp == kWarps) {
    // =============================================================== producer: pages in order, K then V
    uint32_t load = 0;
    bool ok = true;
    for (long long u = u0; u < u1;) {
      const Segment g = segment_at<kRowTile>(s, a, u, u1);
      const int4 it = s.items[g.item];
      const int* row = a.c.page_table + static_cast<size_t>(it.x) * a.c.max_pages;
      for (int p = g.p0; p < g.p1; p += 32) {  // 32 table entries and scales at a time, one per lane
        int page = 0;
        if (p + lane < g.p1 && p + lane < pages_of(it.y)) {
          page = row[p + lane];
          if (page < 0 || page >= a.c.pages) {
            cache_fail(a.w.status, CRISP_ERR_BAD_CACHE);
            page = 0;
          }
        }
        const int block = (a.layer * a.c.pages + page) * heads + g.head;  // < 2^24
        const float ks = a.c.k_scale[block], vs = a.c.v_scale[block];
        const int n = min(32, g.p1 - p);
        for (int j = 0; j < n; ++j) {
          const int blk = __shfl_sync(0xffffffffu, block, j);
          const float sc[2] = {__shfl_sync(0xffffffffu, ks, j), __shfl_sync(0xffffffffu, vs, j)};
          if (lane == 0 && ok) {
#pragma unroll
            for (int kind = 0; kind < 2; ++kind, ++load) {
              const int slot = load % kSlots;
              if (load >= kSlots) ok = ok && mbar_wait(&s.empty[slot], (load / kSlots - 1) & 1, abort_flag);
              if (!ok) break;
              s.scale[slot] = sc[kind];
              mbar_arrive_expect_tx(&s.full[slot], kPageTileBytes);
              tma_load_2d(s.ring[slot], kind == 0 ? &tmap_k : &tmap_v, &s.full[slot], 0, blk * kPage);
            }
          }
        }
      }
      u += g.p1 - g.p0;
    }
    if (lane == 0 && !ok) {
      // given up: the copies in flight still write to this CTA's shared memory, so see them in (bounded)
      const unsigned long long t0 = global_timer_ns();
      for (uint32_t i = load >= kSlots ? load - kSlots : 0; i < load; ++i)
        while (!mbar_try_wait(&s.full[i % kSlots], (i / kSlots) & 1) && global_timer_ns() - t0 < kWaitLimitNs) {
        }
    }
    __syncwarp();
  } else {
    // =============================================================== consumers: 32 tokens of every page
    const int gid = lane >> 2, t = lane & 3;
    const int perm = (gid >> 1) | ((gid & 1) << 2);  // token of fragment row gid for K, chunk of fragment row gid for V
    uint32_t load = 0;
    bool ok = true;  // after a wait that gave up, the loops and barriers run on without waiting
    for (long long u = u0; u < u1;) {
      const Segment g = segment_at<kRowTile>(s, a, u, u1);
      CacheItem it;
      {
        const int4 v = s.items[g.item];
        it.seq = v.x;
        it.len = v.y;
        it.t0 = v.z;
        it.n = v.w;
      }
      const int all_rows = it.n * a.group;
      // ---- Q fragments: row gid of each N tile, dims 16 t .. and 64 + 16 t ..
      uint32_t qf[kTilesN][8][2];
      float col_scale[kTilesN][2];
      int col_last[kTilesN][2];  // last position that the column's row may see
#pragma unroll
      for (int nt = 0; nt < kTilesN; ++nt) {
        const int row = g.tile * kRowTile + nt * 8 + gid;
        uint4 x[4];
        if (row < all_rows) {
          const size_t token = static_cast<size_t>(it.t0) + row / a.group;
          const uint4* p = reinterpret_cast<const uint4*>(
              a.q + (token * a.n_q_heads + g.head * a.group + row % a.group) * kHeadDim);
          x[0] = __ldg(p + 2 * t);
          x[1] = __ldg(p + 2 * t + 1);
          x[2] = __ldg(p + 8 + 2 * t);
          x[3] = __ldg(p + 8 + 2 * t + 1);
        } else {
          x[0] = x[1] = x[2] = x[3] = make_uint4(0, 0, 0, 0);
        }
        uint32_t amax = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t wd[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
          for (int k = 0; k < 4; ++k) amax = max(amax, max(wd[k] & 0x7fffu, (wd[k] >> 16) & 0x7fffu));
        }
        amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
        amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
        const int ex = static_cast<int>(amax >> 7);  // 255: the row holds an infinity or NaN and stays one
        const int e = ex == 255 ? 0 : min(141 - ex, 126);  // the row's largest element lands in [2^14, 2^15)
        const float f = pow2i(e);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t wd[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const __half2 h = __floats2half2_rn(__uint_as_float(wd[k] << 16) * f, __uint_as_float(wd[k] & 0xffff0000u) * f);
            // chunk i / 2, elements 8 (i % 2) + 2 k: K step 4 (i / 2) + 2 (i % 2) + k / 2, pair k % 2
            qf[nt][4 * (i >> 1) + 2 * (i & 1) + (k >> 1)][k & 1] = *reinterpret_cast<const uint32_t*>(&h);
          }
        }
        const float back = a.scale_log2 * pow2i(-e);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          col_scale[nt][k] = __shfl_sync(0xffffffffu, back, (2 * t + k) * 4);
          col_last[nt][k] = it.len - it.n + (g.tile * kRowTile + nt * 8 + 2 * t + k) / a.group;
        }
      }
      const int all_see = it.len - it.n + (g.tile * kRowTile) / a.group;  // every row sees the keys up to here

      float o[kTilesN][8][4];
      float m[kTilesN][2], l[kTilesN][2];
#pragma unroll
      for (int nt = 0; nt < kTilesN; ++nt) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int k = 0; k < 4; ++k) o[nt][j][k] = 0.f;
        m[nt][0] = m[nt][1] = -INFINITY;
        l[nt][0] = l[nt][1] = 0.f;
      }

      for (int p = g.p0; p < g.p1; ++p) {
        const int tok0 = warp * 32;            // the warp's tokens in the page
        const int pos0 = p * kPage + tok0;     // and their first position
        // ---- S^T = K Q^T: two tiles of 16 tokens
        float x[kTilesN][2][4];
#pragma unroll
        for (int nt = 0; nt < kTilesN; ++nt)
#pragma unroll
          for (int mt = 0; mt < 2; ++mt)
#pragma unroll
            for (int k = 0; k < 4; ++k) x[nt][mt][k] = 0.f;
        int slot = load % kSlots;
        ok = ok && mbar_wait_warp(&s.full[slot], (load / kSlots) & 1, abort_flag);
        const float ks = s.scale[slot];
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
          const int tok = tok0 + 16 * mt + perm;   // rows gid and gid + 8: tokens tok and tok + 8 (same swizzle)
          const uint8_t* base = s.ring[slot] + tok * kHeadDim;
          uint4 w[2][2];  // [row half][chunk t, t + 4]
#pragma unroll
          for (int ch = 0; ch < 2; ++ch) {
            const int off = ((t + 4 * ch) ^ (tok & 7)) << 4;
            w[0][ch] = *reinterpret_cast<const uint4*>(base + off);
            w[1][ch] = *reinterpret_cast<const uint4*>(base + 8 * kHeadDim + off);
          }
#pragma unroll
          for (int ch = 0; ch < 2; ++ch) {
            const uint32_t up[4] = {w[0][ch].x, w[0][ch].y, w[0][ch].z, w[0][ch].w};
            const uint32_t dn[4] = {w[1][ch].x, w[1][ch].y, w[1][ch].z, w[1][ch].w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              uint32_t f[4];
              decode4<kFormat>(up[k], f[0], f[2]);
              decode4<kFormat>(dn[k], f[1], f[3]);
#pragma unroll
              for (int nt = 0; nt < kTilesN; ++nt) mma_f16(x[nt][mt], f, qf[nt][4 * ch + k][0], qf[nt][4 * ch + k][1]);
            }
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&s.empty[slot]);
        ++load;
        // ---- online softmax of the columns (the query rows) over the warp's 32 tokens
        const bool masked = pos0 + 31 > all_see;
        uint32_t pf[kTilesN][2][2];
        float alpha[kTilesN][2];
#pragma unroll
        for (int nt = 0; nt < kTilesN; ++nt) {
          float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
          for (int mt = 0; mt < 2; ++mt)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              float v = x[nt][mt][k] * (col_scale[nt][k & 1] * ks);
              if (masked && pos0 + 16 * mt + perm + 8 * (k >> 1) > col_last[nt][k & 1]) v = -INFINITY;
              x[nt][mt][k] = v;
              mx[k & 1] = fmaxf(mx[k & 1], v);
            }
#pragma unroll
          for (int k = 0; k < 2; ++k) {
#pragma unroll
            for (int sh = 4; sh <= 16; sh <<= 1) mx[k] = fmaxf(mx[k], __shfl_xor_sync(0xffffffffu, mx[k], sh));
            const float m_new = fmaxf(m[nt][k], mx[k]);
            const float ref = m_new == -INFINITY ? 0.f : m_new;
            alpha[nt][k] = ex2(m[nt][k] - ref);  // 0 while nothing has been seen
            m[nt][k] = m_new;
            l[nt][k] *= alpha[nt][k];
            mx[k] = ref;
          }
#pragma unroll
          for (int mt = 0; mt < 2; ++mt) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              x[nt][mt][k] = ex2(x[nt][mt][k] - mx[k & 1]);
              l[nt][k & 1] += x[nt][mt][k];
            }
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              const __half2 h = __floats2half2_rn(x[nt][mt][2 * half], x[nt][mt][2 * half + 1]);
              pf[nt][mt][half] = transpose8x8(*reinterpret_cast<const uint32_t*>(&h));
            }
          }
        }
        // ---- O^T += V^T P^T: eight tiles of 16 dims, two steps of 16 tokens
        slot = load % kSlots;
        ok = ok && mbar_wait_warp(&s.full[slot], (load / kSlots) & 1, abort_flag);
        const float vs = s.scale[slot];
        uint4 w[2][4];
        const bool tail = pos0 + 31 >= it.len;  // rows behind the last token may hold anything, NaN among it
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int tok = tok0 + 16 * mt + t + 4 * k;  // k of the product: 2 t, 2 t + 1, 2 t + 8, 2 t + 9
            w[mt][k] = *reinterpret_cast<const uint4*>(s.ring[slot] + tok * kHeadDim + ((perm ^ (tok & 7)) << 4));
            if (tail && p * kPage + tok >= it.len) w[mt][k] = make_uint4(0, 0, 0, 0);
          }
        __syncwarp();
        if (lane == 0) mbar_arrive(&s.empty[slot]);
        ++load;
#pragma unroll
        for (int j = 0; j < 8; ++j) {  // fragment rows gid, gid + 8: dims 16 perm + 2 j, + 1
          uint32_t f[2][4];
#pragma unroll
          for (int mt = 0; mt < 2; ++mt) {
            auto word = [&](int k) {
              const uint4& v = w[mt][k];
              return (j >> 1) == 0 ? v.x : (j >> 1) == 1 ? v.y : (j >> 1) == 2 ? v.z : v.w;
            };
            const uint32_t sel = (j & 1) ? 0x7362u : 0x5140u;
            decode4<kFormat>(__byte_perm(word(0), word(1), sel), f[mt][0], f[mt][1]);
            decode4<kFormat>(__byte_perm(word(2), word(3), sel), f[mt][2], f[mt][3]);
          }
#pragma unroll
          for (int nt = 0; nt < kTilesN; ++nt) {
            float acc[4] = {0.f, 0.f, 0.f, 0.f};
            mma_f16(acc, f[0], pf[nt][0][0], pf[nt][0][1]);
            mma_f16(acc, f[1], pf[nt][1][0], pf[nt][1][1]);
#pragma unroll
            for (int k = 0; k < 4; ++k) o[nt][j][k] = fmaf(acc[k], vs, o[nt][j][k] * alpha[nt][k & 1]);
          }
        }
      }

      // ---- join the four warps: common maximum, weighted sums
#pragma unroll
      for (int nt = 0; nt < kTilesN; ++nt)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
#pragma unroll
          for (int sh = 4; sh <= 16; sh <<= 1) l[nt][k] += __shfl_xor_sync(0xffffffffu, l[nt][k], sh);
          if (gid == 0) {
            s.red_m[warp][nt * 8 + 2 * t + k] = m[nt][k];
            s.red_l[warp][nt * 8 + 2 * t + k] = l[nt][k];
          }
        }
      const bool whole = g.p0 == 0 && g.p1 == g.pages;
      const int cf = cut.cta_of(g.g0), cl = cut.cta_of(g.g0 + g.pages - 1);
      auto slot_of = [&](int c) { return 2 * c + (c == cf && cut.first(c) < g.g0 ? 1 : 0); };
      const int my_slot = slot_of(cta);
#pragma unroll
      for (int nt = 0; nt < kTilesN; ++nt) {
        named_bar_sync(1, kWarps * 32);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int r = nt * 8 + 2 * t + k;
          const float top = fmaxf(fmaxf(s.red_m[0][r], s.red_m[1][r]), fmaxf(s.red_m[2][r], s.red_m[3][r]));
          // a warp that saw nothing for this row adds nothing, whatever its masked places held
          const bool none = m[nt][k] == -INFINITY;
          const float sc = exp2f(m[nt][k] - top);
          auto val = [&](int j, int c) { return none ? 0.f : o[nt][j][c] * sc; };
#pragma unroll
          for (int jj = 0; jj < 4; ++jj)
            *reinterpret_cast<float4*>(&s.red[warp][2 * t + k][16 * perm + 4 * jj]) =
                make_float4(val(2 * jj, k), val(2 * jj, k + 2), val(2 * jj + 1, k), val(2 * jj + 1, k + 2));
        }
        named_bar_sync(1, kWarps * 32);
        // a warp per row, four dims per lane
        for (int r8 = warp; r8 < 8; r8 += kWarps) {
          const int r = nt * 8 + r8, row = g.tile * kRowTile + r;
          if (row >= all_rows) break;
          float top = -INFINITY, sum = 0.f;
#pragma unroll
          for (int w = 0; w < kWarps; ++w) top = fmaxf(top, s.red_m[w][r]);
          float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
          for (int w = 0; w < kWarps; ++w) {
            const float mw = s.red_m[w][r];
            if (mw != -INFINITY) sum += s.red_l[w][r] * exp2f(mw - top);
            const float4 v = *reinterpret_cast<const float4*>(&s.red[w][r8][4 * lane]);
            acc.x += v.x;
            acc.y += v.y;
            acc.z += v.z;
            acc.w += v.w;
          }
          if (whole) {
            const size_t token = static_cast<size_t>(it.t0) + row / a.group;
            const int h = g.head * a.group + row % a.group;
            const float inv = top == -INFINITY ? 0.f : 1.0f / sum;
            uint2 v;
            v.x = pack_bf16(acc.x * inv, acc.y * inv);
            v.y = pack_bf16(acc.z * inv, acc.w * inv);
            reinterpret_cast<uint2*>(a.o + (token * a.n_q_heads + h) * kHeadDim)[lane] = v;
            if (a.lse && lane == 0)
              a.lse[static_cast<size_t>(h) * a.b.n_tokens + token] =
                  top == -INFINITY ? -INFINITY : top * 0.6931471805599453f + logf(sum);
          } else {
            reinterpret_cast<float4*>(a.w.part_o + (static_cast<size_t>(my_slot) * kMaxRows + r) * kHeadDim)[lane] = acc;
            if (lane == 0) a.w.part_ml[my_slot * kMaxRows + r] = make_float2(top, sum);
          }
        }
      }
      if (!whole) {
        // sets of kSet CTAs first; the result of a set lies in the slot of its first CTA
        const int set0 = cta / kSet * kSet;
        const int f = max(cf, set0), e = min(cl, set0 + kSet - 1);
        const int sets = cl / kSet - cf / kSet + 1;
        bool last = true;
        if (e > f) {
          last = arrive_last(s, a.w.counters + slot_of(f), e - f + 1);
          if (last) join<kRowTile>(a, it, g, slot_of(f), f + 1, 1, e - f + 1, sets == 1);
        }
        if (last && sets > 1) {
          last = arrive_last(s, a.w.counters + 2 * kMaxCtas + slot_of(cf), sets);
          if (last) join<kRowTile>(a, it, g, slot_of(cf), (cf / kSet + 1) * kSet, kSet, sets, true);
        }
      }
      named_bar_sync(1, kWarps * 32);  // the exchange buffers are free again
      u += g.p1 - g.p0;
    }
  }
  __syncthreads();
  if (tid == 0 && s.abort_flag) cache_fail(a.w.status, CRISP_ERR_DEVICE_TIMEOUT);
}

template <int kFormat, int kTilesN>
int launch_decode(const CUtensorMap& tk, const CUtensorMap& tv, const AttnArgs& a, int n_sm, cudaStream_t stream) {
  const size_t smem = sizeof(DecodeSmem) + 1024;
  CRISP_CUDA_TRY(cudaFuncSetAttribute(cache_decode_kernel<kFormat, kTilesN>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                      static_cast<int>(smem)),
                 "cache_attention: smem attribute");
  const int grid = 2 * n_sm < kMaxCtas ? 2 * n_sm : kMaxCtas;
  CRISP_KERNEL("cache_decode", stream, launch_pdl(cache_decode_kernel<kFormat, kTilesN>, dim3(grid), dim3(kThreads), smem,
                                                  stream, tk, tv, a));
  CRISP_CUDA_TRY(cudaGetLastError(), "cache_attention: launch");
  return CRISP_OK;
}

}  // namespace

size_t cache_attention_ws_bytes() {
  size_t total;
  carve(nullptr, &total);
  return total;
}

int launch_cache_attention(const CacheView& v, int layer, const CacheBatch& b, int n_q_heads, float scale, const void* q,
                           void* o, float* lse, void* ws, cudaStream_t stream) {
  size_t total;
  AttnArgs a;
  a.c = v;
  a.b = b;
  a.layer = layer;
  a.n_q_heads = n_q_heads;
  a.group = n_q_heads / v.heads;
  a.scale_log2 = scale * kLog2e;
  a.q = static_cast<const __nv_bfloat16*>(q);
  a.o = static_cast<__nv_bfloat16*>(o);
  a.lse = lse;
  a.w = carve(ws, &total);
  CUtensorMap tk, tv;
  const size_t rows = static_cast<size_t>(v.layers) * v.pages * v.heads * kPage;
  int rc = make_tmap_codes(&tk, v.k_codes, rows);
  if (rc == CRISP_OK) rc = make_tmap_codes(&tv, v.v_codes, rows);
  if (rc != CRISP_OK) return rc;
  int dev = 0, n_sm = 0;
  CRISP_CUDA_TRY(cudaGetDevice(&dev), "cache_attention: device");
  CRISP_CUDA_TRY(cudaDeviceGetAttribute(&n_sm, cudaDevAttrMultiProcessorCount, dev), "cache_attention: SM count");
  const bool narrow = static_cast<long long>(b.max_new) * a.group <= 8;
  if (v.format == CRISP_CACHE_E4M3)
    return narrow ? launch_decode<CRISP_CACHE_E4M3, 1>(tk, tv, a, n_sm, stream)
                  : launch_decode<CRISP_CACHE_E4M3, 2>(tk, tv, a, n_sm, stream);
  return narrow ? launch_decode<CRISP_CACHE_INT8, 1>(tk, tv, a, n_sm, stream)
                : launch_decode<CRISP_CACHE_INT8, 2>(tk, tv, a, n_sm, stream);
}

}  // namespace crisp
