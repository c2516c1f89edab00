// Causal attention of longer pieces (many rows per KV head) over the 8-bit paged cache, on tcgen05 tensor cores.
//
// Rows are packed: the new tokens of an item times the G = H_q / H_kv query heads of a KV head, 256 rows (two tiles of
// 128) per group, so that every page that is brought in and converted serves all of them.  The products run as in the
// prompt kernel (prefill.cu): S = Q K^T in two halves of 64 keys, P over the columns of S, O += P V from TMEM, one
// issuing thread per tile.  What differs is where K and V come from:
//  * TMA brings half a page's codes (64 tokens, 8 KB) into a ring; four converter warps turn them into 16-bit operands
//    in a second ring, in the 128-byte-swizzled layout the descriptors want.  Conversion is exact: K's codes become fp16 (a single
//    instruction per pair for e4m3), V's values, code * scale, become bf16, whose exponent range holds every scale.
//    Two pairs of warps share the halves by the slots of the rings (cache_ring.h).
//    Rows of V behind the sequence's end become zero (their codes may be anything, NaN among it).
//  * Q K^T is fp16: Q is brought to fp16 by a power of two per row (exact but for elements 2^-29 below the row's
//    largest); that power and the page's K scale multiply the logits.  P V is bf16, P rounded to bf16 as in prefill.cu.
// The work is cut into equal runs of pages, one per CTA, and partial results are joined (cache_split.cuh).
//
// P's 8 bits are the prompt kernel's, so that a piece answers like the prompt it continues; V is exact in bf16 in both formats.
// (The kernel for few rows has 11 bits: fp16 P would want V's codes as fp16 and its scale elsewhere.)
//
// What bounds it: 4850 cycles per page of 256 rows (2048 new tokens over 32768, 32/8 heads, e4m3: 1.15 ms, 0.92 PFLOP/s; once
// the board has settled at its power cap's clock 1.22 ms, 0.88 PFLOP/s).  Of 4650 in an earlier version the softmax warps were
// busy for 4200; the tensor pipe needs 2880 (its N = 64 products are bound by operand fetch) and the shared memory port about
// 3100 (256 KB of operands, 96 KB of conversion, 32 KB of codes).  Tried and slower, in that version (1.10 ms): two
// warpgroups per tile, one for each half of the keys, with a shared running maximum (1180 us); Q K^T of whole pages behind
// P V, with either (1360 to 1410 us: the chain from S to S is what it lengthens); pacing the two tiles' exponentials or
// computing part of them on the FMA pipe (1125 to 1195 us).  Code size matters more than any of these: with the converters'
// loops unrolled eight and four times the same kernel takes 1480 us, because the roles' code misses the instruction caches.
//
// Warps (512 threads): 0-3, 4-7 softmax of tile 0, 1 (a thread per row); 8 TMA producer; 9, 10 issuers; 11 idle;
// 12-15 converters.  TMEM: S_0 | S_1 | O_0 | O_1, 128 columns each.
#include <cmath>
#include <cuda_fp16.h>

#include "cache_split.cuh"
#include "cache_codes.cuh"
#include "cache_ring.h"
#include "softmax_rows.cuh"

namespace crisp {
namespace {

// K and V move in halves of a page, 64 tokens, in the order in which the products use them:
//   K_A(0) K_B(0) | V_A(0) K_A(1) V_B(0) K_B(1) | V_A(1) K_A(2) V_B(1) K_B(2) | ... | V_A(n-1) V_B(n-1)
constexpr int kHalf = kPage / 2;
constexpr int kInfo = 16;          // words per load or page under way; more than there can be
constexpr int kIsK = -0x40000000;  // marks a load of K where V's has the number of its tokens that exist
constexpr int kTileRows = 256;     // rows of a group of work
constexpr int kGroupUnits = 4;     // what beginning and ending a group costs, in pages
constexpr int kMaxTileCtas = 160;  // bound on the grid; sizes the workspace
constexpr int kPrefillThreads = 512;
constexpr float kNothing = -3.402823466e38f;  // running maximum of a row that has seen nothing: the least finite number
// A weight's exponent, x scale - m in one FMA, is off by half a unit of m in its last place, the same for all of a row: up to
// |m| = 2^30 that is a factor of at most 2^32 on weights and sums alike.  Beyond, two fp32 logits that differ at all differ by 64
// or more, so that the row's weights are its ties for the maximum; there the product with a power of two, which is exact, gives
// the same weights.  It is the power above the scale, so that such logits stay beyond all others; the maximum is brought
// back at the end (true_max).  (Scaling the logits first instead, or multiplying the difference: 2 to 10 % of the kernel.)
constexpr float kFar = 1073741824.0f;
constexpr float kRescaleAt = 8.0f;  // log2 units (as in prefill.cu)

constexpr int kRegsSoft = 176, kRegsMisc = 72, kRegsConv = 88;
static_assert(256 * kRegsSoft + 128 * kRegsMisc + 128 * kRegsConv <= kPrefillThreads * 128, "setmaxnreg budgets exceed the CTA's pool");

struct TileArgs {
  CacheView c;
  CacheBatch b;
  Partials w;
  Output out;
  int layer, group, tile_tokens;  // tile_tokens: 256 / group, the new tokens of a group of work
  float scale_pow2, scale_rest;  // softmax scale x log2(e) = 2 scale_pow2 x scale_rest, a power of two and 1/2 to 1
  const __nv_bfloat16* q;
  int* status;
};

struct TileSmem {
  alignas(1024) uint8_t q[2][2][16384];        // [tile][64-dim half]
  alignas(1024) uint8_t conv[kConv][2][8192];  // [slot][64-dim half]
  alignas(1024) uint8_t raw[kRaw][kPageTileBytes / 2];
  uint64_t raw_full[kRaw], raw_empty[kRaw], conv_full[kConv], conv_empty[kConv];
  uint64_t q_full[2], s_full[2][2], p_ready[2][2], o_done[2][2];
  float load_scale[kInfo], page_scale[kInfo];  // V's scale by load, K's by page
  int load_rows[kInfo];
  long long scratch[33];
  int start[kMaxCacheBatch + 1];  // units of one head before item i
  uint32_t tmem_base;
  int abort_flag;
};

// Pages that tile `tile` of an item (n new tokens, length len) can see; at least one, so that its rows are written.
__device__ __forceinline__ int tile_pages(int len, int n, int tile, int tile_tokens) {
  const int last = len - n + min((tile + 1) * tile_tokens, n) - 1;  // position of the tile's last token
  return last < 0 ? 1 : last / kPage + 1;
}
__device__ __forceinline__ int tiles_of(int n, int tile_tokens) { return (n + tile_tokens - 1) / tile_tokens; }

// Units of one head of an item, summed by a whole warp (at most 2^31 - 1: the caller refuses that many).
__device__ __forceinline__ int item_units(int len, int n, int tile_tokens, int lane) {
  long long sum = 0;
  for (int t = lane; t < tiles_of(n, tile_tokens); t += 32) sum += tile_pages(len, n, t, tile_tokens) + kGroupUnits;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  return static_cast<int>(min(sum, 0x7fffffffLL));
}

// Walks the groups of a CTA's run in order.  A group is kGroupUnits units without work, then its pages.
struct TileWalk {
  Segment g;
  CacheItem it;
  int tiles;  // of the item
  int rows;   // of the group: up to 256
  int g_end;  // unit behind the group

  __device__ __forceinline__ void load(const TileArgs& a) {
    it = load_item(a.c, a.b, g.item, a.status);
    tiles = tiles_of(it.n, a.tile_tokens);
  }
  __device__ __forceinline__ void place(const TileArgs& a, int first_unit) {
    g.pages = tile_pages(it.len, it.n, g.tile, a.tile_tokens);
    rows = min(a.tile_tokens, it.n - g.tile * a.tile_tokens) * a.group;
    g.g0 = first_unit + kGroupUnits;
    g_end = g.g0 + g.pages;
  }
  // the group that holds unit u; a whole warp searches
  __device__ __forceinline__ void seek(const int* start, const TileArgs& a, int u, int lane) {
    int lo = 0, hi = a.b.batch;
    const int key = u / a.c.heads;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (start[mid] <= key) lo = mid; else hi = mid;
    }
    g.item = lo;
    load(a);
    const int per_head = start[lo + 1] - start[lo];
    int rem = u - start[lo] * a.c.heads;
    g.head = rem / per_head;
    rem -= g.head * per_head;
    g.tile = 0;
    for (int t0 = 0; t0 < tiles; t0 += 32) {
      int incl = t0 + lane < tiles ? tile_pages(it.len, it.n, t0 + lane, a.tile_tokens) + kGroupUnits : 0;
      const int mine = incl;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += x;
      }
      const uint32_t past = __ballot_sync(0xffffffffu, incl > rem);
      if (past) {
        const int src = __ffs(past) - 1;
        g.tile = t0 + src;
        rem -= __shfl_sync(0xffffffffu, incl - mine, src);
        break;
      }
      rem -= __shfl_sync(0xffffffffu, incl, 31);
    }
    place(a, u - rem);
  }
  __device__ __forceinline__ void next(const int* start, const TileArgs& a) {
    if (++g.tile == tiles) {
      g.tile = 0;
      if (++g.head == a.c.heads) {
        g.head = 0;
        do ++g.item; while (start[g.item + 1] == start[g.item]);  // items without work
        load(a);
      }
    }
    place(a, g_end);
  }
  // the part of the group within units [u0, u1); false when none of its pages is
  __device__ __forceinline__ bool clip(int u0, int u1) {
    g.p0 = max(u0 - g.g0, 0);
    g.p1 = min(u1 - g.g0, g.pages);
    return g.p0 < g.p1;
  }
};

__host__ __device__ constexpr uint32_t umma_idesc_f16(int M, int N) {
  return (1u << 4) | (static_cast<uint32_t>(N >> 3) << 17) | (static_cast<uint32_t>(M >> 4) << 24);  // f16 x f16 -> f32
}

template <int kFormat>
__global__ void __launch_bounds__(kPrefillThreads, 1)
cache_prefill_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v, const TileArgs a) {
  pdl_enter();
  extern __shared__ uint8_t smem_raw[];
  TileSmem& s = *reinterpret_cast<TileSmem*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int heads = a.c.heads, batch = a.b.batch;
  if (tid == 0) {
    s.abort_flag = 0;
    for (int i = 0; i < kRaw; ++i) {
      mbar_init(&s.raw_full[i], 1);
      mbar_init(&s.raw_empty[i], 2);
    }
    for (int i = 0; i < kConv; ++i) {
      mbar_init(&s.conv_full[i], 2);
      mbar_init(&s.conv_empty[i], 2);  // one arrival per issuer, whether or not its tile has rows
    }
    for (int t = 0; t < 2; ++t) {
      mbar_init(&s.q_full[t], 128);
      for (int h = 0; h < 2; ++h) {
        mbar_init(&s.s_full[t][h], 1);
        mbar_init(&s.p_ready[t][h], 128);
        mbar_init(&s.o_done[t][h], 1);
      }
    }
    fence_mbar_init();
  }
  // ---- units of every item: a warp per item, then their scan (in place)
  for (int i = warp; i < batch; i += kPrefillThreads / 32) {
    const CacheItem it = load_item(a.c, a.b, i, a.status);
    const int units = it.seq < 0 ? 0 : item_units(it.len, it.n, a.tile_tokens, lane);
    if (lane == 0) s.start[i] = units;
  }
  __syncthreads();
  long long carry = 0;
  for (int base = 0; base < batch; base += kPrefillThreads) {
    const int i = base + tid;
    const int units = i < batch ? s.start[i] : 0;
    long long total;
    const long long before = block_exclusive_scan<kPrefillThreads>(units, s.scratch, &total);
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

  if (warp == 8) {
    tmem_alloc(&s.tmem_base, 512);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tm = s.tmem_base;
  volatile int* abort_flag = &s.abort_flag;
  TileWalk w;

  if (warp < 8) {
    // =============================================================== softmax / epilogue, one row per thread
    reg_alloc<kRegsSoft>();
    const int t = warp >> 2, r = tid & 127;
    const uint32_t lane_addr = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t s_addr = tm + lane_addr + t * 128;
    const uint32_t o_addr = tm + lane_addr + 256 + t * 128;
    uint32_t step_count = 0;  // steps of this tile so far: phase of s_full / p_ready / o_done
    uint32_t page_count = 0;  // pages so far
    bool ok = true;           // after a wait that gave up, the loops run on without waiting
    JoinDesc todo = {0, 0, 0, 0, 0, 0};
    auto rescale_o = [&](float f) {
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        uint32_t ov[32];
        tmem_ld_x32(o_addr + c * 32, ov);
        tmem_ld_wait();
#pragma unroll
        for (int i = 0; i < 32; ++i) ov[i] = __float_as_uint(__uint_as_float(ov[i]) * f);
        tmem_st_x32(o_addr + c * 32, ov);
      }
    };
    for (w.seek(s.start, a, u0, lane);; w.next(s.start, a)) {
      if (!w.clip(u0, u1)) {
        if (w.g_end >= u1) break;
        continue;
      }
      const Segment& g = w.g;
      const CacheItem& it = w.it;
      const int row0 = g.tile * a.tile_tokens * a.group;               // first row of the pair of tiles
      const int rows = w.rows;
      const int my_row = t * 128 + r;
      const bool active = t * 128 < rows;                               // the tile has rows
      const bool whole = g.p0 == 0 && g.p1 == g.pages;
      const int slot = partial_slot(cut, g.g0, cut.cta_of(g.g0), cta);
      if (active) {
        // ---- Q: this thread's row to fp16, into the swizzled operand tile
        float row_scale;
        {
          const int row = row0 + my_row;
          const uint4* src = reinterpret_cast<const uint4*>(
              a.q + ((static_cast<size_t>(it.t0) + row / a.group) * a.out.n_q_heads + g.head * a.group + row % a.group) * kHeadDim);
          uint4 x[16];
#pragma unroll
          for (int c = 0; c < 16; ++c) x[c] = my_row < rows ? __ldg(src + c) : make_uint4(0, 0, 0, 0);
          uint32_t amax = 0;
#pragma unroll
          for (int c = 0; c < 16; ++c) {
            const uint32_t wd[4] = {x[c].x, x[c].y, x[c].z, x[c].w};
#pragma unroll
            for (int k = 0; k < 4; ++k) amax = max(amax, max(wd[k] & 0x7fffu, (wd[k] >> 16) & 0x7fffu));
          }
          const int ex = static_cast<int>(amax >> 7);        // 255: the row holds an infinity or NaN and stays one
          const int e = ex == 255 ? 0 : min(141 - ex, 126);  // the row's largest element lands in [2^14, 2^15)
          const float f = pow2i(e);
          row_scale = a.scale_pow2 * pow2i(1 - e);
#pragma unroll
          for (int c = 0; c < 16; ++c) {
            const uint32_t wd[4] = {x[c].x, x[c].y, x[c].z, x[c].w};
            uint32_t h[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) h[k] = half2_bits(__uint_as_float(wd[k] << 16) * f, __uint_as_float(wd[k] & 0xffff0000u) * f);
            *reinterpret_cast<uint4*>(s.q[t][c >> 3] + r * 128 + (((c & 7) ^ (r & 7)) << 4)) = make_uint4(h[0], h[1], h[2], h[3]);
          }
          fence_proxy_async_smem();
          mbar_arrive(&s.q_full[t]);
        }
        // position of the last key this row sees, and of the last one that all rows of the warp see
        const int last_key = min(it.len - it.n + g.tile * a.tile_tokens + my_row / a.group, it.len - 1);
        const int all_see = it.len - it.n + g.tile * a.tile_tokens + (my_row - lane) / a.group;
        float m_used = kNothing, l_run = 0.f;
        auto no_pacing = [](uint32_t&) {};
        float scale = 0.f;
        // one step of the online softmax per half page; both halves run the same code (two copies of it, beside the
        // converters', do not fit the instruction caches: a third of all stalls were fetches)
        const int n_halves = 2 * (g.p1 - g.p0);
#pragma unroll 1
        for (int i = 0; i < n_halves; ++i) {
          const int h = i & 1;
          const uint32_t ph = step_count & 1;
          const int key0 = (2 * g.p0 + i) * kHalf;                       // position of the half's first key
          const bool masked = key0 + kHalf - 1 > all_see;
          const int lim = max(last_key - key0, -1);
          ok = ok && mbar_wait_warp(&s.s_full[t][h], ph, abort_flag);
          if (!ok) break;
          tc_fence_after_sync();
          uint32_t x[2][32];
          const uint32_t half_addr = s_addr + h * kHalf;
          tmem_ld_x32(half_addr, x[0]);
          tmem_ld_x32(half_addr + 32, x[1]);
          if (h == 0) scale = row_scale * *reinterpret_cast<volatile float*>(&s.page_scale[page_count % kInfo]);
          tmem_ld_wait();
          const float top = masked ? row_max<true>(x, lim, 0) : row_max<false>(x, lim, 0);
          const float near = scale * a.scale_rest;
          const bool far = fabsf(top * near) > kFar;
          const float logit_scale = far ? scale : near, mx = top * logit_scale;
          if (i == 0) {
            m_used = fmaxf(mx, kNothing);
          } else if (__any_sync(0xffffffffu, mx > m_used + kRescaleAt)) {
            // the latest P V issued is that of the half before this one
            ok = mbar_wait_warp(&s.o_done[t][h ^ 1], h == 0 ? ph ^ 1u : ph, abort_flag);
            if (!ok) break;
            tc_fence_after_sync();
            const float m_new = fmaxf(m_used, mx);
            const float f = ex2(m_used - m_new);
            rescale_o(f);
            l_run *= f;
            m_used = m_new;
          }
          uint32_t pk[2][16];
          l_run += masked ? exp_pack<true>(x, lim, 0, logit_scale, m_used, pk, no_pacing)
                          : exp_pack<false>(x, lim, 0, logit_scale, m_used, pk, no_pacing);
          asm volatile("" : "+f"(l_run)::"memory");  // the run of exponentials ends here
          tmem_st_x16(half_addr, pk[0]);       // P over the columns of its own S, which this warp has read
          tmem_st_x16(half_addr + 16, pk[1]);
          tmem_st_wait();
          tc_fence_before_sync();
          mbar_arrive(&s.p_ready[t][h]);
          step_count += h;
          page_count += h;
        }
        // ---- epilogue: the row leaves TMEM as output, or as a partial result
        ok = ok && mbar_wait_warp(&s.o_done[t][1], (step_count - 1) & 1, abort_flag);
        if (ok) {
          tc_fence_after_sync();
          const int row = row0 + my_row;
          const size_t token = static_cast<size_t>(it.t0) + row / a.group;
          const int h = g.head * a.group + row % a.group;
          const float inv = l_run == 0.f ? 0.f : 1.0f / l_run;
          const float true_max = fabsf(m_used) > kFar ? m_used * a.scale_rest : m_used;
          __nv_bfloat16* orow = a.out.o + (token * a.out.n_q_heads + h) * kHeadDim;
          float* prow = a.w.o + (static_cast<size_t>(slot) * kTileRows + my_row) * kHeadDim;
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            uint32_t ov[32];
            tmem_ld_x32(o_addr + c * 32, ov);
            tmem_ld_wait();
            if (my_row < rows) {
              if (whole) {
                uint4* dst = reinterpret_cast<uint4*>(orow + c * 32);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                  auto two = [&](int j) {
                    return pack_bf16(__uint_as_float(ov[8 * k + j]) * inv, __uint_as_float(ov[8 * k + j + 1]) * inv);
                  };
                  dst[k] = make_uint4(two(0), two(2), two(4), two(6));
                }
              } else {
                uint4* dst = reinterpret_cast<uint4*>(prow + c * 32);
#pragma unroll
                for (int k = 0; k < 8; ++k) dst[k] = make_uint4(ov[4 * k], ov[4 * k + 1], ov[4 * k + 2], ov[4 * k + 3]);
              }
            }
          }
          if (my_row < rows) {
            if (!whole)
              a.w.ml[static_cast<size_t>(slot) * kTileRows + my_row] = make_float2(true_max, l_run);
            else if (a.out.lse)
              a.out.lse[static_cast<size_t>(h) * a.out.n_tokens + token] =
                  l_run == 0.f ? -INFINITY : true_max * 0.6931471805599453f + logf(l_run);
          }
          tc_fence_before_sync();
        }
      } else {
        page_count += static_cast<uint32_t>(g.p1 - g.p0);
      }
      const JoinDesc d = join_desc(cut, g, cta, it.t0, row0, rows);
      if (d.rows > 0) todo = d;
      if (w.g_end >= u1) break;
    }
    if (tid == 0) a.w.desc[cta] = todo;
  } else if (warp < 12) {
    reg_dealloc<kRegsMisc>();
    if (warp == 8) {
      // =============================================================== producer
      uint32_t load = 0, page_count = 0;
      bool ok = true;
      auto issue = [&](const CUtensorMap* map, int block, int half, float scale, int rows) {
        const int slot = load % kRaw;
        if (load >= kRaw) ok = ok && mbar_wait(&s.raw_empty[slot], (load / kRaw - 1) & 1, abort_flag);
        if (!ok) return;
        s.load_scale[load % kInfo] = scale;
        s.load_rows[load % kInfo] = rows;
        mbar_arrive_expect_tx(&s.raw_full[slot], kPageTileBytes / 2);
        tma_load_2d(s.raw[slot], map, &s.raw_full[slot], 0, block * kPage + half * kHalf);
        ++load;
      };
      for (w.seek(s.start, a, u0, lane);; w.next(s.start, a)) {
        if (!w.clip(u0, u1)) {
          if (w.g_end >= u1) break;
          continue;
        }
        const Segment& g = w.g;
        const CacheItem& it = w.it;
        const int* row = a.c.page_table + static_cast<size_t>(it.seq) * a.c.max_pages;
        int block = 0, block_next = 0;  // of pages p and p + 1
        float vs = 0.f, vs_next = 0.f;
        int lane_block = 0;             // 32 table entries and scales at a time, one per lane
        float lane_ks = 0.f, lane_vs = 0.f;
        for (int p = g.p0 - 1; p < g.p1; ++p) {
          const int j = p + 1 - g.p0;   // the page whose K is issued
          const bool more = p + 1 < g.p1;
          float ks = 0.f;
          if (more) {
            if (j % 32 == 0) {
              const int q = p + 1 + lane;
              const bool exists = q < g.p1 && q < pages_of(it.len);  // (an empty sequence has one page of work)
              int page = 0;
              if (exists) {
                page = row[q];
                if (page < 0 || page >= a.c.pages) {
                  cache_fail(a.status, CRISP_ERR_BAD_CACHE);
                  page = 0;
                }
              }
              lane_block = (a.layer * a.c.pages + page) * heads + g.head;  // < 2^24
              lane_ks = exists ? a.c.k_scale[lane_block] : 1.f;
              lane_vs = exists ? a.c.v_scale[lane_block] : 1.f;
            }
            block_next = __shfl_sync(0xffffffffu, lane_block, j % 32);
            ks = __shfl_sync(0xffffffffu, lane_ks, j % 32);
            vs_next = __shfl_sync(0xffffffffu, lane_vs, j % 32);
          }
          if (lane == 0 && ok) {
            if (more) s.page_scale[page_count % kInfo] = ks;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              if (p >= g.p0) issue(&tmap_v, block, half, vs, it.len - p * kPage - half * kHalf);
              if (more) issue(&tmap_k, block_next, half, 1.f, kIsK);
            }
          }
          if (more) ++page_count;
          block = block_next;
          vs = vs_next;
        }
        if (w.g_end >= u1) break;
      }
      if (lane == 0 && !ok) {
        // given up: the copies in flight still write to this CTA's shared memory, so see them in (bounded)
        const unsigned long long t0 = global_timer_ns();
        for (uint32_t i = load >= kRaw ? load - kRaw : 0; i < load; ++i)
          while (!mbar_try_wait(&s.raw_full[i % kRaw], (i / kRaw) & 1) && global_timer_ns() - t0 < kWaitLimitNs) {
          }
      }
      __syncwarp();
    } else if (warp < 11) {
      // =============================================================== MMA issuers, one thread per tile
      constexpr uint32_t idesc_qk = umma_idesc_f16(128, 64);                  // S half: 128 x 64
      constexpr uint32_t idesc_pv = umma_idesc_bf16(128, 128, false, true);   // O: 128 x 128
      const int t = warp - 9;
      auto desc_add = [](uint64_t desc, uint32_t off) {
        return (desc & 0xffffffff00000000ull) | static_cast<uint64_t>(static_cast<uint32_t>(desc) + off);
      };
      const uint64_t q_desc = umma_desc_sw128(smem_u32(s.q[t][0]), 0, 1024);
      const uint64_t k_desc0 = umma_desc_sw128(smem_u32(s.conv[0][0]), 0, 1024);     // K: K-major
      const uint64_t v_desc0 = umma_desc_sw128(smem_u32(s.conv[0][0]), 8192, 1024);  // V: MN-major
      const uint32_t s_tm = tm + t * 128, o_tm = tm + 256 + t * 128;
      // the next half to be used: its ring slot, that slot's phase and its offset in descriptor units (the issuing threads
      // are on the critical path: no divisions, 32-bit adds on the descriptors' low words)
      uint32_t slot = 0, phase = 0, slot_off = 0;
      auto next_load = [&]() {
        ++slot;
        slot_off += 16384u >> 4;
        if (slot == kConv) {
          slot = slot_off = 0;
          phase ^= 1u;
        }
      };
      uint32_t p_count = 0;   // steps whose P has been consumed (phase of p_ready)
      uint32_t q_count = 0;   // segments of this tile (phase of q_full)
      bool ok = true;
      auto wait_load = [&]() {
        ok = ok && mbar_wait(&s.conv_full[slot], phase, abort_flag);
        if (ok) tc_fence_after_sync();
      };
      // S half h = Q K_h^T with the next half in the ring
      auto mma_qk = [&](int h) {
        wait_load();
        if (!ok) return;
        const uint64_t bd0 = desc_add(k_desc0, slot_off);
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) {
          const uint32_t step = (kk & 3) * (32u >> 4);
          umma_ss(s_tm + h * 64, desc_add(q_desc, (kk >> 2) * (16384u >> 4) + step),
                  desc_add(bd0, (kk >> 2) * (8192u >> 4) + step), idesc_qk, kk > 0);
        }
        umma_commit(&s.s_full[t][h]);
        umma_commit(&s.conv_empty[slot]);
        next_load();
      };
      // O += P_h V_h with the next half in the ring
      auto mma_pv = [&](int h, bool first) {
        wait_load();
        if (!ok) return;
        const uint64_t bd0 = desc_add(v_desc0, slot_off);
#pragma unroll
        for (int k4 = 0; k4 < 4; ++k4)
          umma_ts(o_tm, s_tm + h * 64 + k4 * 8, desc_add(bd0, k4 * (2048u >> 4)), idesc_pv, (k4 > 0 || !first) ? 1u : 0u);
        umma_commit(&s.o_done[t][h]);
        umma_commit(&s.conv_empty[slot]);
        next_load();
      };
      for (w.seek(s.start, a, u0, lane);; w.next(s.start, a)) {
        if (!w.clip(u0, u1)) {
          if (w.g_end >= u1) break;
          continue;
        }
        const int rows = w.rows;
        const int n = w.g.p1 - w.g.p0;
        if (lane == 0) {
          if (t * 128 >= rows) {
            // a tile without rows: see the loads through
            for (int i = 0; i < 4 * n && ok; ++i) {
              wait_load();
              if (ok) mbar_arrive(&s.conv_empty[slot]);
              next_load();
            }
          } else {
            ok = ok && mbar_wait(&s.q_full[t], q_count & 1, abort_flag);
            ++q_count;
            // half-step i is P_h V_h and the next page's Q K_h^T, h = i mod 2 (see prefill.cu); the first two are Q K^T
            // alone.  (One copy of the code: the roles share the instruction caches.)
#pragma unroll 1
            for (int i = -2; i < 2 * n && ok; ++i) {
              const int h = i & 1;
              if (i >= 0) {
                ok = mbar_wait(&s.p_ready[t][h], p_count & 1, abort_flag);
                if (!ok) break;
                mma_pv(h, i == 0);
                p_count += h;
              }
              if (i + 2 < 2 * n && ok) mma_qk(h);
            }
          }
        }
        __syncwarp();
        if (w.g_end >= u1) break;
      }
    }
  } else {
    // =============================================================== converters: two pairs of warps, each with its own
    // slots of both rings (cache_ring.h says why)
    reg_dealloc<kRegsConv>();
    const int ct = tid & 63, chunk = ct & 7, row_of = ct >> 3;  // eight threads per token, 16 codes each
    const uint32_t pair = (tid >> 6) & 1;
    uint32_t n_loads = 0;  // four per page
    for (w.seek(s.start, a, u0, lane);; w.next(s.start, a)) {
      if (w.clip(u0, u1)) n_loads += 4u * static_cast<uint32_t>(w.g.p1 - w.g.p0);
      if (w.g_end >= u1) break;
    }
    // A thread's 16 codes become two 16-byte chunks of a 64-dim half; which of the two comes first depends on the half
    // and on the token's parity, so that the threads of a phase touch different banks in the loads (8 bytes) and in the
    // stores (16 bytes).  (A thread's tokens are row_of + 8 j: the swizzle is the same for all of them.)
    const int c0 = (chunk & 3) * 2, swap = (chunk >> 2) ^ (row_of & 1);
    const int src_a = row_of * 128 + ((chunk ^ row_of) << 4) + swap * 8, src_b = src_a ^ 8;
    const int dst_off = (chunk >> 2) * 8192 + row_of * 128;
    const int dst_a = dst_off + (((c0 + swap) ^ row_of) << 4), dst_b = dst_off + (((c0 + 1 - swap) ^ row_of) << 4);
    bool ok = true;
    uint32_t slot = 0, phase = 0;  // of the load, in both rings
    auto next_slot = [&]() {
      if (++slot == kRaw) {
        slot = 0;
        phase ^= 1u;
      }
    };
    for (uint32_t load = 0; load < n_loads; ++load, next_slot()) {
      if ((kPairOfSlot >> slot & 1u) != pair) continue;
      ok = mbar_wait_warp(&s.raw_full[slot], phase, abort_flag);
      if (ok && load >= kConv) ok = mbar_wait_warp(&s.conv_empty[slot], phase ^ 1u, abort_flag);
      if (!ok) break;
      const float scale = *reinterpret_cast<volatile float*>(&s.load_scale[load % kInfo]);
      const int exist = *reinterpret_cast<volatile int*>(&s.load_rows[load % kInfo]);
      const uint8_t* src = s.raw[slot];
      uint8_t* dst = s.conv[slot][0];
      // (short loops on purpose: unrolled eight and four times they made the kernel 27 % slower, because the roles' code no
      // longer fits the instruction caches)
      if (exist == kIsK) {
#pragma unroll 2
        for (int j = 0; j < 8; ++j) {
          const uint2 a8 = *reinterpret_cast<const uint2*>(src + src_a + j * 1024);
          const uint2 b8 = *reinterpret_cast<const uint2*>(src + src_b + j * 1024);
          uint32_t h[8];
          decode4<kFormat>(a8.x, h[0], h[1]);
          decode4<kFormat>(a8.y, h[2], h[3]);
          decode4<kFormat>(b8.x, h[4], h[5]);
          decode4<kFormat>(b8.y, h[6], h[7]);
          *reinterpret_cast<uint4*>(dst + dst_a + j * 1024) = make_uint4(h[0], h[1], h[2], h[3]);
          *reinterpret_cast<uint4*>(dst + dst_b + j * 1024) = make_uint4(h[4], h[5], h[6], h[7]);
        }
      } else {
#pragma unroll 1
        for (int j = 0; j < 8; ++j) {
          uint2 a8 = *reinterpret_cast<const uint2*>(src + src_a + j * 1024);
          uint2 b8 = *reinterpret_cast<const uint2*>(src + src_b + j * 1024);
          if (row_of + 8 * j >= exist) a8 = b8 = make_uint2(0, 0);  // behind the sequence's end
          uint32_t h[8];
          decode_values4<kFormat>(a8.x, scale, h[0], h[1]);
          decode_values4<kFormat>(a8.y, scale, h[2], h[3]);
          decode_values4<kFormat>(b8.x, scale, h[4], h[5]);
          decode_values4<kFormat>(b8.y, scale, h[6], h[7]);
          *reinterpret_cast<uint4*>(dst + dst_a + j * 1024) = make_uint4(h[0], h[1], h[2], h[3]);
          *reinterpret_cast<uint4*>(dst + dst_b + j * 1024) = make_uint4(h[4], h[5], h[6], h[7]);
        }
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(&s.raw_empty[slot]);
        mbar_arrive(&s.conv_full[slot]);
      }
    }
  }
  tc_fence_before_sync();
  __syncthreads();
  if (tid == 0 && s.abort_flag) cache_fail(a.status, CRISP_ERR_DEVICE_TIMEOUT);
  if (warp == 8) tmem_dealloc(tm, 512);
}

template <int kFormat>
int launch_tiles(const CUtensorMap& tk, const CUtensorMap& tv, const TileArgs& a, int n_sm, cudaStream_t stream) {
  const size_t smem = sizeof(TileSmem) + 1024;
  static std::atomic<unsigned long long> done{0};
  const int rc = allow_smem(reinterpret_cast<const void*>(&cache_prefill_kernel<kFormat>), smem, &done);
  if (rc != CRISP_OK) return rc;
  const int grid = n_sm < kMaxTileCtas ? n_sm : kMaxTileCtas;
  CRISP_KERNEL("cache_prefill", stream, launch_pdl(cache_prefill_kernel<kFormat>, dim3(grid), dim3(kPrefillThreads), smem,
                                                   stream, tk, tv, a));
  CRISP_CUDA_TRY(cudaGetLastError(), "cache_attention: launch");
  return launch_cache_join(a.w, a.out, kTileRows, grid, stream);
}

}  // namespace

size_t cache_prefill_ws(void* ws, size_t off) {
  carve_partials(ws, &off, kMaxTileCtas, kTileRows);
  return off;
}

int launch_cache_prefill(const CacheView& v, int layer, const CacheBatch& b, int n_q_heads, float scale, const void* q,
                         void* o, float* lse, void* ws, size_t ws_off, const CUtensorMap& tk, const CUtensorMap& tv, int n_sm,
                         cudaStream_t stream) {
  TileArgs a;
  a.c = v;
  a.b = b;
  a.layer = layer;
  a.group = n_q_heads / v.heads;
  a.tile_tokens = kTileRows / a.group;
  int exponent;
  a.scale_rest = std::frexp(scale * kLog2e, &exponent);
  a.scale_pow2 = std::ldexp(1.f, exponent - 1);
  a.q = static_cast<const __nv_bfloat16*>(q);
  a.out = Output{static_cast<__nv_bfloat16*>(o), lse, n_q_heads, a.group, b.n_tokens, 0.f};
  a.status = static_cast<int*>(ws);
  a.w = carve_partials(ws, &ws_off, kMaxTileCtas, kTileRows);
  return v.format == CRISP_CACHE_E4M3 ? launch_tiles<CRISP_CACHE_E4M3>(tk, tv, a, n_sm, stream)
                                      : launch_tiles<CRISP_CACHE_INT8>(tk, tv, a, n_sm, stream);
}

}  // namespace crisp
