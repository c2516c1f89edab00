// Causal attention of a few new tokens over the 8-bit paged cache (answering token by token, verifying a draft).
//
// Every cached byte is needed once per (item, KV head), for the G = H_q / H_kv query heads and the item's new tokens
// together (the rows of a group), so the kernel is bound by reading the codes from HBM.  What follows from that:
//  * One unit of work is one page of one KV head (16 KB of K codes, 16 KB of V codes, by TMA into a ring of slots).
//    The units of all items and heads form one sequence that is cut into equal runs, one per CTA, whatever the
//    lengths are; a run that begins or ends inside a group leaves a partial result (maximum, sum, O) in the workspace,
//    and a second small kernel joins them (cache_split.cuh).  The order of every sum is fixed by the sizes.
//  * Codes are not converted in bulk: a warp takes its fragments from shared memory, converts them in registers and
//    multiplies with m16n8k16 (fp16 in, fp32 out).  Products are computed transposed, S^T = K Q^T and O^T = V^T P^T, so
//    that the padded dimension, N = 8, is the few query rows.  (tcgen05 has no shape for so few rows without
//    the codes going through shared memory a second time, and the tensor pipe is not what bounds this kernel.)
//    fp16 holds every code of both formats exactly; Q is brought to fp16 by a power of two per row (exact but for
//    elements 2^-29 below the row's largest), the weights are rounded to fp16's 11 bits, everything else is fp32.
//  * A weight is computed in a unit of its page: 2^-15 of the largest among the 32 tokens that a warp takes from the page.
//    So none loses bits down to 2^-29 of that one, however much other tokens of the row weigh (a sink, say) and however far
//    apart the pages' scales of V are.  A row's sums stand in the largest of its units so far; one factor per page and row
//    brings either the sums or the page there, in fp32.
//  * The order of the dims inside a dot product and of the keys inside P V is free.  A thread therefore reads whole
//    16-byte chunks, and which chunk belongs to which fragment row is chosen so that the eight threads of a
//    shared-memory phase always touch eight different 16-byte banks of the 128-byte-swizzled tile.
//  * Scales are one per page and head: K's multiplies the logits, V's the page's P V product (O is accumulated in
//    fp32 per page, which also applies the running maximum's correction).
// Measured: 4 sequences of 65k to 131k tokens, 32/8 heads, int8: 134 us, 5.9 TB/s (151 us, 5.3 TB/s, once the board has settled
// at its power cap's clock); 262144 tokens, 28/4 heads, e4m3: 57 us, of which about 10 are the start and the join; 32 sequences
// of 1 to 8192 tokens: 22.5 us for 82 MB (24.7 settled); 300 tokens, 4/1 heads: 7 us.  With 24 rows (five tokens, groups of
// four) a page costs three times the products and softmax, and the latency of its chain bounds the kernel: 98 us for 224 MB.
// The weights' units cost 1 to 5 % (one exponential, one directed subtraction and four more instructions per row and page);
// two exponentials, for both factors, instead of one cost 13 % with 24 rows.
#include <cuda_fp16.h>

#include "cache_codes.cuh"
#include "cache_split.cuh"

namespace crisp {
using namespace sm100;

namespace {

constexpr int kWarps = 4;            // consumer warps, which share a page: 32 tokens each
constexpr int kThreads = kWarps * 32 + 32;
constexpr int kMaxCtas = 512;        // bound on the grid; sizes the workspace
constexpr int kMaxRows = kDecodeRows;  // rows of a partial result
constexpr float kWeightBits = 15.f, kWeightUnit = 1.f / 32768.f;
constexpr int kGroupUnits = 1;       // what beginning and ending a group costs, in pages

// Rows come in tiles of eight; a CTA computes kTiles of them at once, which share the loads and conversions of a page.
// One tile: three CTAs share an SM, and a ring of one K and one V slot each is enough: 96 KB under way per SM (three slots:
// 2 us more on 82 MB spread over 32 sequences; two CTAs with five slots: 4 % less bandwidth on long sequences).  Two or
// three tiles need 168 registers: two CTAs.
__host__ __device__ constexpr int ctas_per_sm(int tiles) { return tiles == 1 ? 3 : 2; }
__host__ __device__ constexpr int slots_of(int tiles) { return tiles == 1 ? 2 : 4; }

struct AttnArgs {
  CacheView c;
  CacheBatch b;
  Partials w;
  Output out;
  int layer, group;
  float scale_log2;
  const __nv_bfloat16* q;
  int* status;
};

template <int kTiles>
struct DecodeSmem {
  alignas(1024) uint8_t ring[slots_of(kTiles)][kPageTileBytes];
  float4 red[kWarps][8][kHeadDim / 4];      // the warps' O of eight rows
  alignas(16) uint8_t q[2][8 * kTiles][kHeadDim * 2];
  uint2 q_frag[kTiles][8][32];              // Q as fp16 fragments: [tile][K step][lane]
  float2 col_scale[kTiles][4];              // logit scales of rows 2 t, 2 t + 1
  float red_m[kWarps][8], red_l[kWarps][8];
  float scale[slots_of(kTiles)];
  uint64_t full[slots_of(kTiles)], empty[slots_of(kTiles)], q_full[2], q_empty[2];
  long long scratch[33];
  int abort_flag;
  int start[kMaxCacheBatch + 1];   // units of one head before item i
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
__device__ __forceinline__ int row_tiles(int rows, int row_tile) { return (rows + row_tile - 1) / row_tile; }

// Walks the groups of a CTA's run in order.  A group is kGroupUnits units without work, then its pages.
template <int kRowTile>
struct Walk {
  Segment g;
  CacheItem it;
  int rows, tiles;  // of the item
  int g_end;        // unit behind the group

  __device__ __forceinline__ void load(const AttnArgs& a) {
    it = load_item(a.c, a.b, g.item, a.status);
    rows = it.n * a.group;
    tiles = row_tiles(rows, kRowTile);
    g.pages = max(1, pages_of(it.len));  // an empty sequence still has rows to write
  }
  // the group that holds unit u
  __device__ __forceinline__ void seek(const int* start, const AttnArgs& a, int u) {
    int lo = 0, hi = a.b.batch;
    const int key = u / a.c.heads;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (start[mid] <= key) lo = mid; else hi = mid;
    }
    g.item = lo;
    load(a);
    const int per_group = g.pages + kGroupUnits;
    const int rem = u - start[lo] * a.c.heads, group = rem / per_group;
    g.head = group / tiles;
    g.tile = group - g.head * tiles;
    g.g0 = u - (rem - group * per_group) + kGroupUnits;
    g_end = g.g0 + g.pages;
  }
  __device__ __forceinline__ void next(const int* start, const AttnArgs& a) {
    if (++g.tile == tiles) {
      g.tile = 0;
      if (++g.head == a.c.heads) {
        g.head = 0;
        do ++g.item; while (start[g.item + 1] == start[g.item]);  // items without work
        load(a);
      }
    }
    g.g0 = g_end + kGroupUnits;
    g_end = g.g0 + g.pages;
  }
  // the part of the group within units [u0, u1); false when none of its pages is
  __device__ __forceinline__ bool clip(int u0, int u1) {
    g.p0 = max(u0 - g.g0, 0);
    g.p1 = min(u1 - g.g0, g.pages);
    return g.p0 < g.p1;
  }
};

template <int kFormat, int kTiles>
__global__ void __launch_bounds__(kThreads, ctas_per_sm(kTiles))
cache_decode_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v, const AttnArgs a) {
  constexpr int kRowTile = 8 * kTiles, kSlots = slots_of(kTiles);
  pdl_enter();
  extern __shared__ uint8_t smem_raw[];
  auto& s = *reinterpret_cast<DecodeSmem<kTiles>*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int heads = a.c.heads, batch = a.b.batch;
  if (tid == 0) {
    prefetch_tmap(&tmap_k);
    prefetch_tmap(&tmap_v);
    s.abort_flag = 0;
    for (int i = 0; i < kSlots; ++i) {
      mbar_init(&s.full[i], 2);  // the copy's bytes, and its scale
      mbar_init(&s.empty[i], kWarps);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&s.q_full[i], 1);
      mbar_init(&s.q_empty[i], kWarps);
    }
    fence_mbar_init();
  }
  // ---- every CTA reads the batch and counts the units before each item
  long long carry = 0;
  for (int base = 0; base < batch; base += kThreads) {
    const int i = base + tid;
    int units = 0;
    if (i < batch) {
      const CacheItem it = load_item(a.c, a.b, i, a.status);
      if (it.seq >= 0) units = (max(1, pages_of(it.len)) + kGroupUnits) * row_tiles(it.n * a.group, kRowTile);
    }
    long long total;
    const long long before = block_exclusive_scan<kThreads>(units, s.scratch, &total);
    if (i < batch) s.start[i] = static_cast<int>(min(carry + before, 0x7fffffffLL));
    carry += total;
  }
  if (tid == 0) s.start[batch] = static_cast<int>(min(carry, 0x7fffffffLL));
  __syncthreads();
  const bool too_many = carry * heads >= 0x7fffffffLL;  // units are counted in 32 bits
  if (too_many && tid == 0) cache_fail(a.status, CRISP_ERR_UNSUPPORTED);
  const Cut cut(too_many ? 0 : static_cast<int>(carry) * heads, gridDim.x);
  const int cta = blockIdx.x;
  if (cta >= cut.ctas) {
    if (tid == 0) a.w.desc[cta].rows = 0;  // nothing to join
    return;
  }
  const int u0 = cut.first(cta), u1 = cut.first(cta + 1);
  volatile int* abort_flag = &s.abort_flag;
  Walk<kRowTile> w;

  if (warp == kWarps) {
    // =============================================================== producer: a group's Q rows, then its pages, K and V
    uint32_t slot = 0, phase = 0, segs = 0;  // phase: parity of the ring's current round
    bool ok = true, round0 = true;           // the first round finds the slots empty
    for (w.seek(s.start, a, u0);; w.next(s.start, a)) {
      if (w.clip(u0, u1)) {
        const Segment& g = w.g;
        const int* row = a.c.page_table + static_cast<size_t>(w.it.seq) * a.c.max_pages;
        const int have = pages_of(w.it.len);
        int page0 = 0;
        if (g.p0 + lane < g.p1 && g.p0 + lane < have) page0 = row[g.p0 + lane];  // on its way while Q is fetched
        {
          const int qb = segs & 1;
          if (segs >= 2) ok = ok && mbar_wait_warp(&s.q_empty[qb], ((segs >> 1) - 1) & 1, abort_flag);
          const int n = min(kRowTile, w.rows - g.tile * kRowTile);
          if (ok && lane == 0) mbar_arrive_expect_tx(&s.q_full[qb], n * kHeadDim * 2);
          __syncwarp();
          if (ok && lane < n) {
            const int r = g.tile * kRowTile + lane;
            const size_t token = static_cast<size_t>(w.it.t0) + r / a.group;
            bulk_load(s.q[qb][lane], a.q + (token * a.out.n_q_heads + g.head * a.group + r % a.group) * kHeadDim,
                      kHeadDim * 2, &s.q_full[qb]);
          }
          ++segs;
        }
        for (int p = g.p0; p < g.p1; p += 32) {  // 32 table entries and scales at a time, one per lane
          const bool exists = p + lane < g.p1 && p + lane < have;  // (an empty sequence has one page of work)
          int page = p == g.p0 ? page0 : (exists ? row[p + lane] : 0);
          if (exists && (page < 0 || page >= a.c.pages)) {
            cache_fail(a.status, CRISP_ERR_BAD_CACHE);
            page = 0;
          }
          const int block = (a.layer * a.c.pages + page) * heads + g.head;  // < 2^24
          const float ks = exists ? a.c.k_scale[block] : 1.f, vs = exists ? a.c.v_scale[block] : 1.f;
          const int n = min(32, g.p1 - p);
          for (int j = 0; j < n; ++j) {
            const int blk = __shfl_sync(0xffffffffu, block, j);
            const uint32_t slot_k = slot;
            if (lane == 0 && ok) {
#pragma unroll
              for (int kind = 0; kind < 2; ++kind) {
                if (!round0) ok = ok && mbar_wait(&s.empty[slot], phase ^ 1u, abort_flag);
                if (!ok) break;
                mbar_arrive_expect_tx(&s.full[slot], kPageTileBytes);
                tma_load_2d(s.ring[slot], kind == 0 ? &tmap_k : &tmap_v, &s.full[slot], 0, blk * kPage);
                if (++slot == kSlots) {
                  slot = 0;
                  phase ^= 1u;
                  round0 = false;
                }
              }
            }
            // the scales are a load behind the table's: they follow the copies that need not wait for them
            const float sk = __shfl_sync(0xffffffffu, ks, j), sv = __shfl_sync(0xffffffffu, vs, j);
            if (lane == 0 && ok) {
              const uint32_t slot_v = slot_k + 1 == kSlots ? 0 : slot_k + 1;
              s.scale[slot_k] = sk;
              mbar_arrive(&s.full[slot_k]);
              s.scale[slot_v] = sv;
              mbar_arrive(&s.full[slot_v]);
            }
          }
        }
      }
      if (w.g_end >= u1) break;
    }
    __syncwarp();
  } else {
    // =============================================================== consumers
    const int gid = lane >> 2, t = lane & 3;
    const int perm = (gid >> 1) | ((gid & 1) << 2);  // token of fragment row gid for K, chunk of fragment row gid for V
    uint32_t slot = 0, phase = 0, segs = 0;
    auto next_slot = [&]() {
      if (++slot == kSlots) {
        slot = 0;
        phase ^= 1u;
      }
    };
    bool ok = true;  // after a wait that gave up, the loops and barriers run on without waiting
    JoinDesc todo = {0, 0, 0, 0, 0, 0};
    for (w.seek(s.start, a, u0);; w.next(s.start, a)) {
      if (w.clip(u0, u1)) {
        const Segment& g = w.g;
        const CacheItem& it = w.it;
        const int first_row = g.tile * kRowTile;
        // ---- Q fragments, one tile per warp: row gid, dims 16 t .. and 64 + 16 t ..
        {
          const int qb = segs & 1;
          ok = ok && mbar_wait_warp(&s.q_full[qb], (segs >> 1) & 1, abort_flag);
          if (warp < kTiles) {
            uint4 x[4];
            const uint4* p = reinterpret_cast<const uint4*>(s.q[qb][8 * warp + gid]);
            const bool have = first_row + 8 * warp + gid < w.rows;
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = have ? p[(i & 1) + 2 * t + 8 * (i >> 1)] : make_uint4(0, 0, 0, 0);
            uint32_t amax = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t wd[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
              for (int k = 0; k < 4; ++k) amax = __vmaxu2(amax, wd[k] & 0x7fff7fffu);
            }
            amax = __vmaxu2(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
            amax = __vmaxu2(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
            amax = max(amax & 0xffffu, amax >> 16);
            const int ex = static_cast<int>(amax >> 7);  // 255: the row holds an infinity or NaN and stays one
            const int e = ex == 255 ? 0 : min(141 - ex, 126);  // the row's largest element lands in [2^14, 2^15)
            const float f = pow2i(e);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t wd[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
              for (int k = 0; k < 4; k += 2)
                // chunk i / 2, elements 8 (i % 2) + 2 k: K step 4 (i / 2) + 2 (i % 2) + k / 2
                s.q_frag[warp][4 * (i >> 1) + 2 * (i & 1) + (k >> 1)][lane] = make_uint2(
                    half2_bits(__uint_as_float(wd[k] << 16) * f, __uint_as_float(wd[k] & 0xffff0000u) * f),
                    half2_bits(__uint_as_float(wd[k + 1] << 16) * f, __uint_as_float(wd[k + 1] & 0xffff0000u) * f));
            }
            if (t == 0) reinterpret_cast<float*>(s.col_scale[warp])[gid] = a.scale_log2 * pow2i(-e);
          }
          named_bar_sync(1, kWarps * 32);
          if (lane == 0) mbar_arrive(&s.q_empty[qb]);
          ++segs;
        }
        const int all_see = it.len - it.n + first_row / a.group;  // every row sees the keys up to here

        float o[kTiles][8][4];
        float m[kTiles][2], l[kTiles][2];  // o: sums of weight x V, times 2^-15; m: log2 of their unit; l: sums of weights
#pragma unroll
        for (int nt = 0; nt < kTiles; ++nt) {
          m[nt][0] = m[nt][1] = -INFINITY;
          l[nt][0] = l[nt][1] = 0.f;
#pragma unroll
          for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k) o[nt][j][k] = 0.f;
        }

#pragma unroll 1
        for (int p = g.p0; p < g.p1; ++p) {
          const int tok0 = warp * 32;            // the warp's tokens in the page
          const int pos0 = p * kPage + tok0;     // and their first position
          // ---- S^T = K Q^T: two tiles of 16 tokens
          float x[kTiles][2][4];
#pragma unroll
          for (int nt = 0; nt < kTiles; ++nt)
#pragma unroll
            for (int mt = 0; mt < 2; ++mt)
#pragma unroll
              for (int k = 0; k < 4; ++k) x[nt][mt][k] = 0.f;
          ok = ok && mbar_wait_warp(&s.full[slot], phase, abort_flag);
          const float ks = s.scale[slot];
#pragma unroll
          for (int ch = 0; ch < 2; ++ch) {
            uint4 kw[2][2];  // [tile of tokens][row half]: rows gid and gid + 8 are tokens perm and perm + 8 (same swizzle)
#pragma unroll
            for (int mt = 0; mt < 2; ++mt) {
              const int tok = tok0 + 16 * mt + perm;
              const uint8_t* base = s.ring[slot] + tok * kHeadDim + (((t + 4 * ch) ^ (tok & 7)) << 4);
              kw[mt][0] = *reinterpret_cast<const uint4*>(base);
              kw[mt][1] = *reinterpret_cast<const uint4*>(base + 8 * kHeadDim);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              uint2 qf[kTiles];
#pragma unroll
              for (int nt = 0; nt < kTiles; ++nt) qf[nt] = s.q_frag[nt][4 * ch + k][lane];
#pragma unroll
              for (int mt = 0; mt < 2; ++mt) {
                auto word = [&](const uint4& v) { return k == 0 ? v.x : k == 1 ? v.y : k == 2 ? v.z : v.w; };
                uint32_t f[4];
                decode4<kFormat>(word(kw[mt][0]), f[0], f[2]);
                decode4<kFormat>(word(kw[mt][1]), f[1], f[3]);
#pragma unroll
                for (int nt = 0; nt < kTiles; ++nt) mma_f16(x[nt][mt], f, qf[nt].x, qf[nt].y);
              }
            }
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(&s.empty[slot]);
          next_slot();
          // ---- online softmax of the columns (the query rows) over the warp's 32 tokens
          const bool masked = pos0 + 31 > all_see;
          uint32_t pf[kTiles][2][2];
          float alpha[kTiles][2], beta[kTiles][2];
#pragma unroll
          for (int nt = 0; nt < kTiles; ++nt) {
            const float2 cs = s.col_scale[nt][t];
            const float sc[2] = {cs.x * ks, cs.y * ks};
            float ref[2] = {-INFINITY, -INFINITY};
#pragma unroll
            for (int mt = 0; mt < 2; ++mt)
#pragma unroll
              for (int k = 0; k < 4; ++k) x[nt][mt][k] *= sc[k & 1];
            if (masked) {
              int last[2];  // last position that the column's row may see
#pragma unroll
              for (int k = 0; k < 2; ++k) last[k] = it.len - it.n + (first_row + 8 * nt + 2 * t + k) / a.group;
#pragma unroll
              for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                  if (pos0 + 16 * mt + perm + 8 * (k >> 1) > last[k & 1]) x[nt][mt][k] = -INFINITY;
            }
#pragma unroll
            for (int mt = 0; mt < 2; ++mt)
#pragma unroll
              for (int k = 0; k < 4; ++k) ref[k & 1] = fmaxf(ref[k & 1], x[nt][mt][k]);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
#pragma unroll
              for (int sh = 4; sh <= 16; sh <<= 1) ref[k] = fmaxf(ref[k], __shfl_xor_sync(0xffffffffu, ref[k], sh));
              const float low = __fsub_ru(ref[k], kWeightBits);  // rounded upwards: no weight comes above 2^15
              const float d = low == m[nt][k] ? 0.f : low - m[nt][k], f = ex2(-fabsf(d));  // 0 beside a unit of -infinity
              alpha[nt][k] = d > 0.f ? f : 1.f;
              beta[nt][k] = d > 0.f ? 1.f : f;
              m[nt][k] = fmaxf(m[nt][k], low);
              ref[k] = low == -INFINITY ? 0.f : low;
            }
            float sum[2] = {0.f, 0.f};
#pragma unroll
            for (int mt = 0; mt < 2; ++mt) {
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                x[nt][mt][k] = ex2(x[nt][mt][k] - ref[k & 1]);
                sum[k & 1] += x[nt][mt][k];
              }
#pragma unroll
              for (int half = 0; half < 2; ++half)
                pf[nt][mt][half] = transpose8x8(half2_bits(x[nt][mt][2 * half], x[nt][mt][2 * half + 1]));
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) l[nt][k] = fmaf(sum[k], beta[nt][k], l[nt][k] * alpha[nt][k]);
          }
          // ---- O^T += V^T P^T: eight tiles of 16 dims, two steps of 16 tokens
          ok = ok && mbar_wait_warp(&s.full[slot], phase, abort_flag);
          const float vs = s.scale[slot] * kWeightUnit;
          uint4 vw[2][4];
          const bool tail = pos0 + 31 >= it.len;  // rows behind the last token may hold anything, NaN among it
#pragma unroll
          for (int mt = 0; mt < 2; ++mt)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const int tok = tok0 + 16 * mt + t + 4 * k;  // k of the product: 2 t, 2 t + 1, 2 t + 8, 2 t + 9
              vw[mt][k] = *reinterpret_cast<const uint4*>(s.ring[slot] + tok * kHeadDim + ((perm ^ (tok & 7)) << 4));
              if (tail && p * kPage + tok >= it.len) vw[mt][k] = make_uint4(0, 0, 0, 0);
            }
          __syncwarp();
          if (lane == 0) mbar_arrive(&s.empty[slot]);
          next_slot();
#pragma unroll
          for (int nt = 0; nt < kTiles; ++nt)
#pragma unroll
            for (int k = 0; k < 2; ++k) beta[nt][k] *= vs;
#pragma unroll
          for (int j = 0; j < 8; ++j) {  // fragment rows gid, gid + 8: dims 16 perm + 2 j, + 1
            uint32_t f[2][4];
#pragma unroll
            for (int mt = 0; mt < 2; ++mt) {
              auto word = [&](int k) {
                const uint4& v = vw[mt][k];
                return (j >> 1) == 0 ? v.x : (j >> 1) == 1 ? v.y : (j >> 1) == 2 ? v.z : v.w;
              };
              const uint32_t sel = (j & 1) ? 0x7362u : 0x5140u;
              decode4<kFormat>(__byte_perm(word(0), word(1), sel), f[mt][0], f[mt][1]);
              decode4<kFormat>(__byte_perm(word(2), word(3), sel), f[mt][2], f[mt][3]);
            }
#pragma unroll
            for (int nt = 0; nt < kTiles; ++nt) {
              float acc[4] = {0.f, 0.f, 0.f, 0.f};
              mma_f16(acc, f[0], pf[nt][0][0], pf[nt][0][1]);
              mma_f16(acc, f[1], pf[nt][1][0], pf[nt][1][1]);
#pragma unroll
              for (int k = 0; k < 4; ++k) o[nt][j][k] = fmaf(acc[k], beta[nt][k & 1], o[nt][j][k] * alpha[nt][k & 1]);
            }
          }
        }

        // ---- join the four warps, eight rows at a time.  A row's 32 chunks of four dims lie permuted, so that neither the
        // writers (rows 2 t + k, chunks 4 perm + jj) nor the readers (one row, all chunks) meet in a bank.
        const bool whole = g.p0 == 0 && g.p1 == g.pages;
        const int my_slot = whole ? 0 : partial_slot(cut, g.g0, cut.cta_of(g.g0), cta);
#pragma unroll
        for (int nt = 0; nt < kTiles; ++nt) {
#pragma unroll
          for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int sh = 4; sh <= 16; sh <<= 1) l[nt][k] += __shfl_xor_sync(0xffffffffu, l[nt][k], sh);
          named_bar_sync(1, kWarps * 32);  // the readers of the rows before are done
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            if (gid == 0) {
              l[nt][k] *= kWeightUnit;
              if (l[nt][k] != l[nt][k]) m[nt][k] = 0.f;  // NaN among the row's logits: its maximum may be none, but it has been seen
              s.red_m[warp][2 * t + k] = m[nt][k];
              s.red_l[warp][2 * t + k] = l[nt][k];
            }
#pragma unroll
            for (int jj = 0; jj < 4; ++jj)
              s.red[warp][2 * t + k][(4 * perm + jj) ^ (t + 4 * (perm >> 2))] =
                  make_float4(o[nt][2 * jj][k], o[nt][2 * jj][k + 2], o[nt][2 * jj + 1][k], o[nt][2 * jj + 1][k + 2]);
          }
          named_bar_sync(1, kWarps * 32);
          for (int r = warp; r < 8; r += kWarps) {  // a warp per row, four dims per lane
            const int row = first_row + 8 * nt + r;
            if (row >= w.rows) break;
            float mw[kWarps], top = -INFINITY, sum = 0.f;
#pragma unroll
            for (int i = 0; i < kWarps; ++i) top = fmaxf(top, mw[i] = s.red_m[i][r]);
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int i = 0; i < kWarps; ++i) {
              if (mw[i] == -INFINITY) continue;  // saw nothing for this row: adds nothing, whatever its masked places held
              const float f = ex2(mw[i] - top);
              sum = fmaf(s.red_l[i][r], f, sum);
              const float4 v = s.red[i][r][lane ^ ((r >> 1) + 4 * (lane >> 4))];
              acc.x = fmaf(v.x, f, acc.x);
              acc.y = fmaf(v.y, f, acc.y);
              acc.z = fmaf(v.z, f, acc.z);
              acc.w = fmaf(v.w, f, acc.w);
            }
            if (whole) {
              write_row(a.out, it.t0, g.head, row, lane, acc, top, sum);
            } else {
              const int at = my_slot * kMaxRows + 8 * nt + r;
              reinterpret_cast<float4*>(a.w.o + static_cast<size_t>(at) * kHeadDim)[lane] = acc;
              if (lane == 0) a.w.ml[at] = make_float2(top, sum);
            }
          }
        }
        const JoinDesc d = join_desc(cut, g, cta, it.t0, first_row, min(kRowTile, w.rows - first_row));
        if (d.rows > 0) todo = d;
      }
      if (w.g_end >= u1) break;
    }
    if (tid == 0) a.w.desc[cta] = todo;
  }
  __syncthreads();
  if (tid == 0 && s.abort_flag) {
    // given up: copies in flight still write to this CTA's shared memory, so give them time to land (bounded)
    const unsigned long long t0 = global_timer_ns();
    while (global_timer_ns() - t0 < kWaitLimitNs / 4) {
    }
    cache_fail(a.status, CRISP_ERR_DEVICE_TIMEOUT);
  }
  __syncthreads();
}

template <int kFormat, int kTiles>
int launch_decode(const CUtensorMap& tk, const CUtensorMap& tv, const AttnArgs& a, int n_sm, cudaStream_t stream) {
  const size_t smem = sizeof(DecodeSmem<kTiles>) + 1024;
  static_assert((sizeof(DecodeSmem<kTiles>) + 2048) * ctas_per_sm(kTiles) <= 228 * 1024, "shared memory of an SM");
  static std::atomic<unsigned long long> done{0};
  const int rc = allow_smem(reinterpret_cast<const void*>(&cache_decode_kernel<kFormat, kTiles>), smem, &done);
  if (rc != CRISP_OK) return rc;
  const int grid = ctas_per_sm(kTiles) * n_sm < kMaxCtas ? ctas_per_sm(kTiles) * n_sm : kMaxCtas;
  CRISP_KERNEL("cache_decode", stream, launch_pdl(cache_decode_kernel<kFormat, kTiles>, dim3(grid), dim3(kThreads), smem,
                                                  stream, tk, tv, a));
  CRISP_CUDA_TRY(cudaGetLastError(), "cache_attention: launch");
  return launch_cache_join(a.w, a.out, 8 * kTiles, grid, stream);
}

template <int kFormat>
int launch_format(const CUtensorMap& tk, const CUtensorMap& tv, const AttnArgs& a, int n_sm, cudaStream_t stream) {
  const long long rows = static_cast<long long>(a.b.max_new < a.b.hi ? a.b.max_new : a.b.hi) * a.group;
  if (rows <= 8) return launch_decode<kFormat, 1>(tk, tv, a, n_sm, stream);
  if (rows <= 16) return launch_decode<kFormat, 2>(tk, tv, a, n_sm, stream);
  return launch_decode<kFormat, 3>(tk, tv, a, n_sm, stream);
}

}  // namespace

size_t cache_decode_ws(void* ws, size_t off) {
  carve_partials(ws, &off, kMaxCtas, kMaxRows);
  return off;
}

int launch_cache_decode(const CacheView& v, int layer, const CacheBatch& b, int n_q_heads, float scale, const void* q,
                        void* o, float* lse, void* ws, size_t ws_off, const CUtensorMap& tk, const CUtensorMap& tv, int n_sm,
                        cudaStream_t stream) {
  AttnArgs a;
  a.c = v;
  a.b = b;
  a.layer = layer;
  a.group = n_q_heads / v.heads;
  a.scale_log2 = scale * kLog2e;
  a.q = static_cast<const __nv_bfloat16*>(q);
  a.out = Output{static_cast<__nv_bfloat16*>(o), lse, n_q_heads, a.group, b.n_tokens, kWeightBits};
  a.status = static_cast<int*>(ws);
  a.w = carve_partials(ws, &ws_off, kMaxCtas, kMaxRows);
  return v.format == CRISP_CACHE_E4M3 ? launch_format<CRISP_CACHE_E4M3>(tk, tv, a, n_sm, stream)
                                      : launch_format<CRISP_CACHE_INT8>(tk, tv, a, n_sm, stream);
}

}  // namespace crisp
