// The product of 8-bit operands: out[m][n] = sum over blocks b of 2^(ea[m,b] + ew[n,b]) * sum_{k in b} A[m,k] W[n,k].
//
// Scales are powers of two, so the tensor core applies them itself (kind::mxf8f6f4) and the accumulators stay in TMEM from the
// first column to the last; a general scale per block of 128 would have to be multiplied in outside, once per block.
// The rows of W (output features) are the 128 rows of the tensor core's tile and the tokens its columns, whatever their number:
// one token costs a tile of 16 columns, and the same kernel serves prompts with up to 256 columns.
//
// Scales reach the tensor core through TMEM: four bytes of a row, the scales of four blocks, are one 32-bit cell, and an
// instruction's descriptor says which byte it uses.  So a cell serves 512 columns, and the cells of 128 rows are four TMEM
// columns: four warps load the words straight from memory and store them to TMEM (each to its own quarter of the lanes, since
// the tensor core wants them in all four).
//
// Bound by latency and L2, not by products.  1 token, 4096 -> 6144: 6.5 us (weights 25 MB, in L2); 33 tokens, 4096 -> 4096: 6.2 us;
// with weights from HBM, as in a model, 7.5 and 7.7 us.
#include <atomic>

#include "matmul.cuh"
#include "sm100_ptx.cuh"

namespace crisp {
namespace {

using namespace sm100;

constexpr int kTileFeatures = 128;
constexpr int kMatmulThreads = 224;    // warps 0..3: scales, then the epilogue; 4 and 5: TMA; 6: MMA
constexpr int kMaxStages = 12;
constexpr int kScaleSlots = 4;         // words of scales (512 columns) in TMEM at a time
constexpr int kMaxSplit = 8;           // CTAs of a cluster

struct __align__(16) MatmulSmem {
  uint64_t full[kMaxStages], empty[kMaxStages], scale_full[kScaleSlots], scale_empty[kScaleSlots], done;
  uint32_t tmem;
  int abort_flag;
};

__global__ void __launch_bounds__(kMatmulThreads, 1) matmul_kernel(const __grid_constant__ CUtensorMap tw,
                                                                   const __grid_constant__ CUtensorMap ta, const MatmulArgs a) {
  extern __shared__ __align__(1024) uint8_t raw[];
  __shared__ MatmulSmem s;
  uint8_t* ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~static_cast<uintptr_t>(1023));
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const int rank = a.split > 1 ? static_cast<int>(cluster_rank()) : 0;
  const int tile = blockIdx.x / a.split;
  const int f0 = (tile % a.n_feature_tiles) * kTileFeatures;
  const int t0 = (tile / a.n_feature_tiles) * a.tile_tokens;
  const int blocks = (a.n_cols + kScaleBlock - 1) / kScaleBlock, words = (a.n_cols + kScaleWord - 1) / kScaleWord;
  const int pairs = (blocks + 1) / 2;   // blocks are dealt in pairs
  const int k0 = static_cast<int>(static_cast<long long>(rank) * pairs / a.split) * 2;
  const int k1 = min(static_cast<int>(static_cast<long long>(rank + 1) * pairs / a.split) * 2, blocks);
  const int stage_bytes = (kTileFeatures + a.tile_tokens) * kScaleBlock;
  const int token_cells = (a.tile_tokens + 31) / 32;            // TMEM columns of the tokens' scales
  const int slot_cols = token_cells > 4 ? 12 : 8;
  if (warp == 4 && elect_one()) {
    // the weights set out for L2 while the kernel before this one ends
    for (int kb = k0; kb < k1; ++kb) tma_prefetch_2d(&tw, kb * kScaleBlock, f0);
    prefetch_tmap(&ta);
  }
  if (tid == 0) {
    for (int i = 0; i < a.stages; ++i) {
      mbar_init(&s.full[i], 1);
      mbar_init(&s.empty[i], 1);
    }
    for (int i = 0; i < kScaleSlots; ++i) {
      mbar_init(&s.scale_full[i], 4);
      mbar_init(&s.scale_empty[i], 1);
    }
    mbar_init(&s.done, 1);
    s.abort_flag = 0;
    fence_mbar_init();
  }
  pdl_enter();
  if (warp == 6) {
    tmem_alloc(&s.tmem, a.tmem_cols);
    tmem_relinquish();
    tc_fence_before_sync();
  }
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tm = s.tmem;
  volatile int* abort_flag = &s.abort_flag;

  // (Loads and products are issued by one elected lane of a warp that stays together, and two blocks at a time: see
  // matmul_pair.cu.)
  if (warp == 4 || warp == 5) {
    // (No more loading warps than stages: one that came to a stage before the use before last had ended would take that use's
    // phase for the last one's.)
    int stage = warp - 4;
    uint32_t phase = 0;
    for (int kb = k0 + warp - 4; kb < k1; kb += 2) {
      if (kb - k0 >= a.stages && !mbar_wait_warp(&s.empty[stage], phase ^ 1u, abort_flag)) break;
      if (elect_one()) {
        uint8_t* slot = ring + stage * stage_bytes;
        mbar_arrive_expect_tx(&s.full[stage], stage_bytes);
        tma_load_2d(slot, &tw, &s.full[stage], kb * kScaleBlock, f0);
        tma_load_2d(slot + kTileFeatures * kScaleBlock, &ta, &s.full[stage], kb * kScaleBlock, t0);
      }
      if ((stage += 2) >= a.stages) {
        stage -= a.stages;
        phase ^= 1u;
      }
    }
  } else if (warp == 6) {
    int stage = 0, slot = 0;
    uint32_t phase = 0, slot_phase = 0;
    const uint32_t scale_base = tm + static_cast<uint32_t>(a.tile_tokens + 31) / 32 * 32;
    for (int kb = k0; kb < k1; kb += 2) {
      const bool two = kb + 1 < k1, word = kb == k0 || (kb & 3) == 0;   // k0 is even
      const int stage1 = stage + 1 == a.stages ? 0 : stage + 1;
      const uint32_t phase1 = phase ^ (stage1 == 0 ? 1u : 0u);
      const bool ready = mbar_try_wait(&s.full[stage], phase) & (!two || mbar_try_wait(&s.full[stage1], phase1)) &
                         (!word || mbar_try_wait(&s.scale_full[slot], slot_phase));
      if (!__all_sync(0xffffffffu, ready)) {
        if (!mbar_wait_warp(&s.full[stage], phase, abort_flag) || (two && !mbar_wait_warp(&s.full[stage1], phase1, abort_flag)) ||
            (word && !mbar_wait_warp(&s.scale_full[slot], slot_phase, abort_flag)))
          break;
      }
      tc_fence_after_sync();
      const uint32_t at = smem_u32(ring + stage * stage_bytes), at1 = smem_u32(ring + stage1 * stage_bytes);
      const uint64_t wd = umma_desc_sw128(at, 0, 1024), wd1 = umma_desc_sw128(at1, 0, 1024);
      constexpr int kTokens = kTileFeatures * kScaleBlock >> 4;   // from a stage's weights to its tokens, in a descriptor
      const uint32_t idesc = umma_idesc_mx_e4m3(kTileFeatures, a.tile_tokens, kb & 3);
      const uint32_t idesc1 = umma_idesc_mx_e4m3(kTileFeatures, a.tile_tokens, (kb & 3) + 1);
      const uint32_t sc = scale_base + slot * slot_cols;
      const bool last = (kb & 2) != 0;   // of a word of scales
      if (elect_one()) {
#pragma unroll
        for (int i = 0; i < 4; ++i)   // 32 columns each
          umma_mx_ss(tm, wd + 2 * i, wd + kTokens + 2 * i, idesc, sc, sc + 4, kb > k0 || i > 0);
        umma_commit(&s.empty[stage]);
        if (two) {
#pragma unroll
          for (int i = 0; i < 4; ++i) umma_mx_ss(tm, wd1 + 2 * i, wd1 + kTokens + 2 * i, idesc1, sc, sc + 4, 1);
          umma_commit(&s.empty[stage1]);
        }
        if (last) umma_commit(&s.scale_empty[slot]);
        if (kb + 2 >= k1) umma_commit(&s.done);
      }
      if ((stage += 2) >= a.stages) {
        stage -= a.stages;
        phase ^= 1u;
      }
      if (last && ++slot == kScaleSlots) {
        slot = 0;
        slot_phase ^= 1u;
      }
    }
  } else {
    const uint32_t quarter = tm + (static_cast<uint32_t>(warp * 32) << 16);
    const uint32_t scale_base = quarter + (a.tile_tokens + 31) / 32 * 32;
    const int w0 = k0 >> 2, w1 = (k1 + 3) >> 2;
    uint32_t next[12][4];   // four words at a time: a fetch takes longer than four words' products
    bool ok = true;
    for (int word = w0; word < w1; ++word) {
      const int i = word - w0, slot = i % kScaleSlots;
      if ((i & 3) == 0) {
#pragma unroll
        for (int c = 0; c < 12; ++c) {
          if (c < 4) {
            load_words(a.w_scales, static_cast<long long>(f0) + 32 * c + lane, a.n_out, words, word, next[c]);
          } else if (c - 4 < token_cells) {
            load_words(a.scales, static_cast<long long>(t0) + 32 * (c - 4) + lane, a.n_rows, words, word, next[c]);
          }
        }
      }
      if (i >= kScaleSlots) ok = mbar_wait_warp(&s.scale_empty[slot], (i / kScaleSlots - 1) & 1, abort_flag);
      if (!ok) break;
      if (i >= kScaleSlots) tc_fence_after_sync();
      const uint32_t at = scale_base + slot * slot_cols;
      uint32_t w[12];
#pragma unroll
      for (int c = 0; c < 12; ++c) w[c] = (i & 2) ? ((i & 1) ? next[c][3] : next[c][2]) : ((i & 1) ? next[c][1] : next[c][0]);
      tmem_st_x4(at, w);
      tmem_st_x4(at + 4, w + 4);
      if (slot_cols > 8) tmem_st_x4(at + 8, w + 8);
      tmem_st_wait();
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive(&s.scale_full[slot]);
      __syncwarp();
    }
    ok = ok && mbar_wait_warp(&s.done, 0, abort_flag, a.wait_ns);
    if (ok) {
      tc_fence_after_sync();
      const int feature = f0 + warp * 32 + lane;
      float* part = reinterpret_cast<float*>(ring);   // [token][128]: every load has been consumed
      for (int c = 0; c < a.tile_tokens; c += 32) {
        if (t0 + c >= a.n_rows) break;
        uint32_t v[32];
        tmem_ld_x32(quarter + c, v);
        tmem_ld_wait();
        const int n = min(min(32, a.tile_tokens - c), a.n_rows - t0 - c);
        if (a.split > 1) {
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if (i < n) part[(c + i) * kTileFeatures + warp * 32 + lane] = __uint_as_float(v[i]);
        } else {
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if (i < n && feature < a.n_out)
              a.out[static_cast<size_t>(t0 + c + i) * a.n_out + feature] = __float2bfloat16_rn(__uint_as_float(v[i]));
        }
      }
    }
  }
  if (a.split > 1) {
    cluster_sync();   // every CTA's partial sums are in its shared memory
    // the tokens are dealt to the cluster's warps, a lane has four features; sums are taken in the order of the columns
    constexpr int kWarps = kMatmulThreads / 32;
    const int n = min(a.tile_tokens, a.n_rows - t0), step = kWarps * a.split;
    const int feature = f0 + 4 * lane;
    const uint32_t mine = smem_u32(ring) + lane * 16;
    for (int t = warp * a.split + rank; t < n; t += 2 * step) {   // two at a time
      float4 v[2][kMaxSplit];
#pragma unroll
      for (int p = 0; p < kMaxSplit; ++p)
        if (p < a.split) {
          const uint32_t from = cluster_map(mine, p);
          v[0][p] = cluster_load4(from + t * (kTileFeatures * 4));
          if (t + step < n) v[1][p] = cluster_load4(from + (t + step) * (kTileFeatures * 4));
        }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int at = t + i * step;
        if (at >= n) break;
        float4 sum = v[i][0];
#pragma unroll
        for (int p = 1; p < kMaxSplit; ++p)
          if (p < a.split) sum.x += v[i][p].x, sum.y += v[i][p].y, sum.z += v[i][p].z, sum.w += v[i][p].w;
        __nv_bfloat16* out = a.out + static_cast<size_t>(t0 + at) * a.n_out + feature;
        if ((a.n_out & 3) == 0) {
          if (feature < a.n_out) *reinterpret_cast<uint2*>(out) = make_uint2(pack_bf16(sum.x, sum.y), pack_bf16(sum.z, sum.w));
        } else {
          const float f[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (feature + j < a.n_out) out[j] = __float2bfloat16_rn(f[j]);
        }
      }
    }
    cluster_sync();   // nobody leaves while its sums are read
  }
  tc_fence_before_sync();
  __syncthreads();
  if (tid == 0 && s.abort_flag) {
    // given up: copies in flight still write to this CTA's shared memory, so give them time to land (bounded)
    const unsigned long long from = global_timer_ns();
    while (global_timer_ns() - from < kWaitLimitNs / 4) {
    }
    cache_fail(a.status, CRISP_ERR_DEVICE_TIMEOUT);
  }
  __syncthreads();
  if (warp == 6) {
    tc_fence_after_sync();
    tmem_dealloc(tm, a.tmem_cols);
  }
}

}  // namespace

namespace {

// How a product is cut, by estimates in ns of what was measured on one B200 (12 to 32 blocks of columns, 1 to 2048 rows).
struct Plan {
  int tile_tokens = 0, split = 0;   // split 0: the kernel for pairs of CTAs
  long long rounds = 0, ns = INT64_MAX;
};

// TMEM columns of a tile: accumulators and the slots of scales, a power of two.
constexpr int tmem_columns(int tile_tokens) {
  const int used = (tile_tokens + 31) / 32 * 32 + kScaleSlots * (tile_tokens > 128 ? 12 : 8);
  int columns = 32;
  while (columns < used) columns *= 2;
  return columns;
}
// Tiles that want all of an SM's TMEM get all of its shared memory, so that no second CTA comes to the SM: it would wait for TMEM
// while its cluster waits for it.  Of the others an SM holds two.
constexpr bool is_wide(int tile_tokens) { return tmem_columns(tile_tokens) > 256; }

// Tiles of 128 features, each block of columns in one of `split` CTAs.  A launch and an exchange take 3 and 0.8 us; a block takes
// a CTA 185 ns with 16 tokens, 290 with 64, 520 with 128 and more (its loads' latency over the few stages of its ring); more
// CTAs than SMs get in each other's way; the sums of a token are read across the cluster in 12 ns.
void plan_split(int n_rows, int n_out, int blocks, int n_sm, int tile_tokens, Plan* best) {
  const long long tiles = static_cast<long long>(ceil_div(n_out, kTileFeatures)) * ceil_div(n_rows, tile_tokens);
  const long long block_ns = tile_tokens < 128 ? 150 + 11 * tile_tokens / 5 : 520;
  for (int split = 1; split <= kMaxSplit && split <= (blocks + 1) / 2; split *= 2) {
    // clusters do not span the SMs of two GPCs: up to 16 CTAs of four, or 32 of eight, find no place
    const long long ctas = tiles * split, room = (is_wide(tile_tokens) ? 1 : 2) * n_sm - (split > 2 ? 4 * split : 0);
    if (ctas > room && split > 1) break;
    const long long rounds = (ctas + room - 1) / room;
    const long long crowd = ctas > n_sm && rounds == 1 ? 100 * ctas / n_sm * ctas / n_sm : 100;
    const long long ns = 3000 + (split > 1 ? 800 + 12 * tile_tokens : 0) + rounds * ceil_div(blocks, split) * block_ns * crowd / 100;
    if (ns < best->ns) *best = Plan{tile_tokens, split, rounds, ns};
  }
}

// Tiles of 256 features and up to 224 tokens, each in a pair of CTAs: 5 us, and 95 + 0.9 tokens ns for a block of a round, or
// 10 ns for a token that is written where there are few blocks.
void plan_pairs(int n_rows, int n_out, int blocks, int n_sm, Plan* best) {
  for (int tokens = 64; tokens <= kPairTokens; tokens += 16) {
    const long long tiles = static_cast<long long>(ceil_div(n_out, 2 * kTileFeatures)) * ceil_div(n_rows, tokens);
    const long long rounds = (tiles + n_sm / 2 - 1) / (n_sm / 2), products = blocks * (95 + 9 * tokens / 10);
    const long long ns = 5000 + rounds * (products > 10 * tokens ? products : 10 * tokens);
    if (ns < best->ns) *best = Plan{tokens, 0, rounds, ns};
    if (n_rows <= tokens) break;
  }
}

}  // namespace

int launch_matmul(const void* codes, const uint8_t* scales, const void* w_codes, const uint8_t* w_scales, int n_rows,
                  int n_out, int n_cols, void* out, void* ws, cudaStream_t stream) {
  MatmulArgs a;
  a.scales = scales;
  a.w_scales = w_scales;
  a.out = static_cast<__nv_bfloat16*>(out);
  a.status = static_cast<int*>(ws);
  a.n_rows = n_rows;
  a.n_out = n_out;
  a.n_cols = n_cols;
  int n_sm = 0;
  int rc = current_sm_count(&n_sm);
  if (rc != CRISP_OK) return rc;
  const int blocks = ceil_div(n_cols, kScaleBlock);
  a.wait_ns = tile_wait_ns(blocks);
  Plan plan;
  if (n_rows > 64) plan_pairs(n_rows, n_out, blocks, n_sm, &plan);
  if (n_rows <= 256) {
    plan_split(n_rows, n_out, blocks, n_sm, ceil_div(n_rows, 16) * 16, &plan);
  } else if (plan.rounds == 1 || n_out <= kTileFeatures) {   // few tiles, which more CTAs may share, or half a pair's features
    plan_split(n_rows, n_out, blocks, n_sm, 128, &plan);
    plan_split(n_rows, n_out, blocks, n_sm, 256, &plan);
  }
  if (plan.split == 0) return launch_matmul_pair(a, codes, w_codes, plan.tile_tokens, n_sm, stream);
  a.tile_tokens = plan.tile_tokens;
  a.split = plan.split;
  a.n_feature_tiles = ceil_div(n_out, kTileFeatures);
  a.n_tiles = static_cast<long long>(a.n_feature_tiles) * ceil_div(n_rows, a.tile_tokens);
  if (a.n_tiles > INT32_MAX / kMaxSplit) return CRISP_ERR_UNSUPPORTED;
  // A CTA that has an SM to itself and much to read gets a longer ring (33 rows, 8192 x 8192 weights: 20.9 -> 16.9 us); with less
  // to read room for the next call's CTAs is worth more (1 row, 6144 x 4096 weights: 7.9 us with the long ring, 7.2 without).
  a.tmem_cols = tmem_columns(a.tile_tokens);
  const bool alone = a.n_tiles * a.split <= n_sm - (a.split > 2 ? 4 * a.split : 0);
  const bool deep = is_wide(a.tile_tokens) || (alone && ceil_div(blocks, a.split) >= 24);
  static_assert(2 * (104 * 1024 + 1024 + sizeof(MatmulSmem) + 1024) <= 228 * 1024 && 3 * 104 > 228 && 200 + 104 > 228, "CTAs of an SM");
  const int budget = (deep ? 200 : 104) * 1024, stage_bytes = (kTileFeatures + a.tile_tokens) * kScaleBlock;
  a.stages = budget / stage_bytes < kMaxStages ? budget / stage_bytes : kMaxStages;   // 2 at least
  const size_t smem = budget + 1024;
  CUtensorMap tw, ta;
  rc = make_tmap_operand(&tw, w_codes, n_out, n_cols, kTileFeatures);
  if (rc == CRISP_OK) rc = make_tmap_operand(&ta, codes, n_rows, n_cols, a.tile_tokens);
  static std::atomic<unsigned long long> done{0};
  if (rc == CRISP_OK) rc = allow_smem(reinterpret_cast<const void*>(&matmul_kernel), 200 * 1024 + 1024, &done);
  if (rc != CRISP_OK) return rc;
  CRISP_KERNEL("matmul", stream, launch_pdl_cluster(matmul_kernel, dim3(static_cast<unsigned>(a.n_tiles * a.split)),
                                                    dim3(kMatmulThreads), smem, a.split, stream, tw, ta, a));
  CRISP_CUDA_TRY(cudaGetLastError(), "matmul: launch");
  return CRISP_OK;
}

}  // namespace crisp
