// The product of 8-bit operands for many rows: tiles of 256 features and up to 224 tokens, each computed by a pair of CTAs
// (tcgen05, cta_group::2): either CTA holds the codes of 128 features and of half the tokens, so that a byte brought to an SM
// serves twice as many products as it would for a CTA alone.  matmul.cu says how the scales get to the tensor core.
//
// The CTAs are persistent.  Roles: warps 0..3 and 11..14 write finished tiles, 4..7 bring scales to TMEM, 8 and 9 load codes (TMA),
// 10 issues the products (first CTA of the pair).  TMEM holds two tiles' accumulators, so that one is written while the other is computed.
//
// 32768 tokens, 4096 -> 6144: 535 to 578 us, 2.9 to 3.1 PFLOP/s, bound by the tensor pipe (91 % active); over seconds the board's
// power cap leaves 2.4 to 2.65 (687 to 622 us).  700 tokens, 3584 -> 4608: 12.0 us, one round of 72 pairs.
#include <atomic>

#include "matmul.cuh"
#include "sm100_ptx.cuh"

namespace crisp {
namespace {

using namespace sm100;

constexpr int kRows = 128;              // features of a CTA
constexpr int kThreads = 480;
constexpr int kStages = 6;
constexpr int kChunk = 32;              // tokens that are written at a time
constexpr int kSlots = 4;               // words of scales in TMEM at a time
constexpr int kSlotCols = 12;           // 4 for the features, 8 for the tokens
constexpr int kScaleColumn = 512 - kSlots * kSlotCols;
static_assert(2 * kPairTokens <= kScaleColumn, "TMEM");

struct __align__(128) PairSmem {
  uint64_t full[kStages], empty[kStages], scale_full[kSlots], scale_empty[kSlots], acc_full[2], acc_empty[2];
  __align__(128) uint16_t out[2][kChunk][kRows];   // bf16, [token][feature]
  uint32_t words[2][4][3 * kRows];      // scales of four words' 128 features and 256 tokens
  uint32_t tmem;
  int abort_flag;
};

__global__ void __launch_bounds__(kThreads, 1) matmul_pair_kernel(const __grid_constant__ CUtensorMap tw,
                                                                  const __grid_constant__ CUtensorMap ta,
                                                                  const __grid_constant__ CUtensorMap to, const MatmulArgs a) {
  extern __shared__ __align__(1024) uint8_t raw[];
  __shared__ PairSmem s;
  uint8_t* ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~static_cast<uintptr_t>(1023));
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const int rank = static_cast<int>(cluster_rank());
  const long long pairs = gridDim.x / 2, first = blockIdx.x / 2;
  const int blocks = (a.n_cols + kScaleBlock - 1) / kScaleBlock, words = (a.n_cols + kScaleWord - 1) / kScaleWord;
  const int stage_bytes = (kRows + a.tile_tokens / 2) * kScaleBlock;
  if (warp == 8 && elect_one()) {   // (what does not depend on the kernel before this one comes before the wait for it)
    prefetch_tmap(&tw);
    prefetch_tmap(&ta);
    prefetch_tmap(&to);
  }
  if (tid == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(&s.full[i], 1);
      mbar_init(&s.empty[i], 1);
    }
    for (int i = 0; i < kSlots; ++i) {
      mbar_init(&s.scale_full[i], 8);
      mbar_init(&s.scale_empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&s.acc_full[i], 1);
      mbar_init(&s.acc_empty[i], 16);
    }
    s.abort_flag = 0;
    fence_mbar_init();
  }
  pdl_enter();
  if (warp == 10) {
    tmem_alloc_pair(&s.tmem, 512);
    tmem_relinquish_pair();
    tc_fence_before_sync();
  }
  cluster_sync();   // both CTAs' barriers are ready
  tc_fence_after_sync();
  const uint32_t tm = s.tmem;
  volatile int* abort_flag = &s.abort_flag;
  auto place = [&](long long tile, int& f0, int& t0) {   // this CTA's first feature, the pair's first token
    f0 = static_cast<int>(tile % a.n_feature_tiles) * (2 * kRows) + rank * kRows;
    t0 = static_cast<int>(tile / a.n_feature_tiles) * a.tile_tokens;
  };

  // Loads and products are issued by one elected lane of a warp that stays together, so that descriptors and coordinates are
  // known to be the warp's: from a branch of one thread a product takes 100 to 190 cycles to issue, and 39 to 128 to compute.
  if (warp == 8 || warp == 9) {
    // Two loading warps take turns: the copies of one follow one another, 16 KB in 200 ns, those of two run side by side.
    int stage = warp - 8;
    uint32_t phase = 0;
    long long step = warp - 8;   // blocks of all tiles, counted through
    bool ok = true;
    long long base = 0;          // step at which the tile began
    for (long long tile = first; tile < a.n_tiles && ok; tile += pairs, base += blocks) {
      int f0, t0;
      place(tile, f0, t0);
      t0 += rank * (a.tile_tokens / 2);
      for (; step < base + blocks; step += 2) {
        if (step >= kStages && !(ok = mbar_wait_warp(&s.empty[stage], phase ^ 1u, abort_flag))) break;
        const int column = static_cast<int>(step - base) * kScaleBlock;
        if (elect_one()) {
          uint8_t* slot = ring + stage * stage_bytes;
          const uint32_t bar = cluster_map(smem_u32(&s.full[stage]), 0);
          // the first CTA's barrier counts both CTAs' bytes (the other's may land before it expects them: the phase cannot
          // end without its arrival)
          if (rank == 0) mbar_arrive_expect_tx(&s.full[stage], 2 * stage_bytes);
          tma_load_2d_pair(slot, &tw, bar, column, f0);
          tma_load_2d_pair(slot + kRows * kScaleBlock, &ta, bar, column, t0);
        }
        if ((stage += 2) >= kStages) {
          stage -= kStages;
          phase ^= 1u;
        }
      }
    }
  } else if (warp == 10) {
    if (rank == 0) {
      // Two blocks at a time: a wait, a fence and a commit take about 50 cycles each between products.
      int stage = 0, slot = 0, turn = 0;
      uint32_t phase = 0, slot_phase = 0;
      bool ok = true;
      for (long long tile = first; tile < a.n_tiles && ok; tile += pairs, ++turn) {
        const int buf = turn & 1;
        if (turn >= 2) ok = mbar_wait_warp(&s.acc_empty[buf], ((turn >> 1) - 1) & 1, abort_flag);
        const uint32_t acc = tm + buf * kPairTokens;
        for (int kb = 0; kb < blocks && ok; kb += 2) {
          const bool two = kb + 1 < blocks, word = (kb & 3) == 0;
          const int stage1 = stage + 1 == kStages ? 0 : stage + 1;
          const uint32_t phase1 = phase ^ (stage1 == 0 ? 1u : 0u);
          const bool ready = mbar_try_wait(&s.full[stage], phase) & (!two || mbar_try_wait(&s.full[stage1], phase1)) &
                             (!word || mbar_try_wait(&s.scale_full[slot], slot_phase));
          if (!__all_sync(0xffffffffu, ready)) {
            ok = mbar_wait_warp(&s.full[stage], phase, abort_flag) &&
                 (!two || mbar_wait_warp(&s.full[stage1], phase1, abort_flag)) &&
                 (!word || mbar_wait_warp(&s.scale_full[slot], slot_phase, abort_flag));
            if (!ok) break;
          }
          tc_fence_after_sync();
          const uint32_t at = smem_u32(ring + stage * stage_bytes), at1 = smem_u32(ring + stage1 * stage_bytes);
          const uint64_t wd = umma_desc_sw128(at, 0, 1024), wd1 = umma_desc_sw128(at1, 0, 1024);
          constexpr int kTokens = kRows * kScaleBlock >> 4;   // from a stage's weights to its tokens, in a descriptor
          const uint32_t idesc = umma_idesc_mx_e4m3(2 * kRows, a.tile_tokens, kb & 3);
          const uint32_t idesc1 = umma_idesc_mx_e4m3(2 * kRows, a.tile_tokens, (kb & 3) + 1);
          const uint32_t sc = tm + kScaleColumn + slot * kSlotCols;
          const bool end = kb + 2 >= blocks, last = (kb & 2) != 0 || end;   // of a word of scales
          if (elect_one()) {
#pragma unroll
            for (int i = 0; i < 4; ++i)   // 32 columns each
              umma_mx_ss_pair(acc, wd + 2 * i, wd + kTokens + 2 * i, idesc, sc, sc + 4, kb > 0 || i > 0);
            umma_commit_pair(&s.empty[stage]);
            if (two) {
#pragma unroll
              for (int i = 0; i < 4; ++i) umma_mx_ss_pair(acc, wd1 + 2 * i, wd1 + kTokens + 2 * i, idesc1, sc, sc + 4, 1);
              umma_commit_pair(&s.empty[stage1]);
            }
            if (last) umma_commit_pair(&s.scale_empty[slot]);
            if (end) umma_commit_pair(&s.acc_full[buf]);
          }
          stage = stage1;
          phase = phase1;
          if (two && ++stage == kStages) {
            stage = 0;
            phase ^= 1u;
          }
          if (last && ++slot == kSlots) {
            slot = 0;
            slot_phase ^= 1u;
          }
        }
      }
    }
  } else if (warp >= 4 && warp < 8) {
    const int row = tid - 128;   // of the features, and of both halves of 256 tokens
    const uint32_t quarter = tm + kScaleColumn + (static_cast<uint32_t>((warp & 3) * 32) << 16);
    uint32_t next[3][4];
    auto fetch = [&](long long tile, int word) {
      int f0, t0;
      place(tile, f0, t0);
      load_words(a.w_scales, static_cast<long long>(f0) + row, a.n_out, words, word, next[0]);
      load_words(a.scales, static_cast<long long>(t0) + row, a.n_rows, words, word, next[1]);
      if (kRows + row < a.tile_tokens) load_words(a.scales, static_cast<long long>(t0) + kRows + row, a.n_rows, words, word, next[2]);
    };
    bool ok = true, round0 = true;
    int slot = 0, side = 0;
    uint32_t phase = 0;
    if (first < a.n_tiles) fetch(first, 0);
    // (after a wait that gave up the loops go on without their work, so that all four warps meet at every barrier)
    for (long long tile = first; tile < a.n_tiles; tile += pairs) {
      for (int word = 0; word < words; ++word) {
        if ((word & 3) == 0) {
          // each warp needs all rows' words: through shared memory (a side is free once everybody has come here again)
          side ^= 1;
#pragma unroll
          for (int c = 0; c < 3; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) s.words[side][i][c * kRows + row] = next[c][i];
          named_bar_sync(1, 128);
          if (word + 4 < words) {
            fetch(tile, word + 4);
          } else if (tile + pairs < a.n_tiles) {
            fetch(tile + pairs, 0);
          }
        }
        if (!round0) ok = ok && mbar_wait_warp(&s.scale_empty[slot], phase ^ 1u, abort_flag);
        if (ok) {
          tc_fence_after_sync();
          uint32_t w[12];
#pragma unroll
          for (int c = 0; c < 12; ++c) w[c] = s.words[side][word & 3][32 * c + lane];
          const uint32_t at = quarter + slot * kSlotCols;
          tmem_st_x4(at, w);
          tmem_st_x4(at + 4, w + 4);
          tmem_st_x4(at + 8, w + 8);
          tmem_st_wait();
          tc_fence_before_sync();
          __syncwarp();
          if (lane == 0) cluster_arrive(cluster_map(smem_u32(&s.scale_full[slot]), 0));
          __syncwarp();
        }
        if (++slot == kSlots) {
          slot = 0;
          phase ^= 1u;
          round0 = false;
        }
      }
    }
  } else {
    // Two groups of four warps take turns with chunks of 32 tokens.  A chunk goes through shared memory, where a thread's feature (a
    // lane of TMEM) becomes a place in a token's row of 256 bytes.  (Straight from registers, 64 bytes of a token at a time, 32768 rows of
    // 8192 features left at 1.8 TB/s.)
    bool ok = true;
    int turn = 0;
    const int group = warp > 10, part = warp & 3, member = group ? warp - 11 : warp;   // part: of TMEM's lanes
    const uint32_t quarter = tm + (static_cast<uint32_t>(part * 32) << 16);
    const bool by_tma = (a.n_out & 7) == 0;
    for (long long tile = first; tile < a.n_tiles; tile += pairs, ++turn) {   // (all four warps meet at every barrier: see above)
      int f0, t0;
      place(tile, f0, t0);
      const int buf = turn & 1;
      ok = ok && mbar_wait_warp(&s.acc_full[buf], (turn >> 1) & 1, abort_flag, a.wait_ns);
      tc_fence_after_sync();
      const int n_tokens = min(a.tile_tokens, a.n_rows - t0);
      for (int c = group * kChunk; c < a.tile_tokens; c += 2 * kChunk) {
        uint32_t v[32];
        if (ok) {
          tmem_ld_x32(quarter + buf * kPairTokens + c, v);
          tmem_ld_wait();
          if (c + 2 * kChunk >= a.tile_tokens) {
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) cluster_arrive(cluster_map(smem_u32(&s.acc_empty[buf]), 0));
            __syncwarp();
          }
        }
        if (by_tma && member == 0) {
          if (elect_one()) tma_store_wait_read0();   // the group's last chunk has been read
          __syncwarp();
        }
        named_bar_sync(2 + group, 128);
        if (ok) {
#pragma unroll
          for (int i = 0; i < 32; i += 2) {
            const uint32_t two = pack_bf16(__uint_as_float(v[i]), __uint_as_float(v[i + 1]));
            s.out[group][i][part * 32 + lane] = static_cast<uint16_t>(two);
            s.out[group][i + 1][part * 32 + lane] = static_cast<uint16_t>(two >> 16);
          }
        }
        if (by_tma) fence_proxy_async_smem();
        named_bar_sync(2 + group, 128);
        if (!ok) continue;
        if (by_tma) {
          if (member == 0 && elect_one()) {
            // in halves, since a tile may end within a chunk; what is behind the last row or feature is left out
            const bool here = f0 < a.n_out;
            if (here && c < n_tokens) tma_store_2d(&to, s.out[group][0], f0, t0 + c);
            if (here && c + kChunk / 2 < n_tokens) tma_store_2d(&to, s.out[group][kChunk / 2], f0, t0 + c + kChunk / 2);
            tma_store_commit();
          }
          continue;
        }
        // Rows that TMA cannot write: a warp writes every fourth, a lane two pairs of neighbouring features; where a row begins at an
        // odd place, pairs are taken from its second feature on and the first is written alone.
        const int token = t0 + c + member, left = n_tokens - c - member, n_features = a.n_out - f0;
        const int odd = a.n_out & token & 1;
        __nv_bfloat16* out = a.out + static_cast<size_t>(token) * a.n_out + f0 + 2 * lane + odd;
        const int have = n_features - 2 * lane - odd;
        uint32_t w[kChunk / 4][2];
#pragma unroll
        for (int i = 0; i < kChunk / 4; ++i) {
          const uint32_t* row = reinterpret_cast<const uint32_t*>(s.out[group][member + 4 * i]) + lane;
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            w[i][j] = row[32 * j];
            if (odd) w[i][j] = __funnelshift_r(w[i][j], 32 * j + lane < 63 ? row[32 * j + 1] : 0, 16);
          }
        }
#pragma unroll
        for (int i = 0; i < kChunk / 4; ++i) {
          if (4 * i >= left) break;
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            __nv_bfloat16* at = out + static_cast<size_t>(4 * i) * a.n_out + 64 * j;
            const bool last = odd && j == 1 && lane == 31;   // its second feature is the next tile's first
            if (have - 64 * j >= 2 && !last) {
              *reinterpret_cast<uint32_t*>(at) = w[i][j];
            } else if (have - 64 * j >= 1) {
              *reinterpret_cast<uint16_t*>(at) = static_cast<uint16_t>(w[i][j]);
            }
          }
          if (odd && lane == 0 && n_features > 0)
            *reinterpret_cast<uint16_t*>(out - 1 + static_cast<size_t>(4 * i) * a.n_out) = s.out[group][member + 4 * i][0];
        }
      }
    }
    if (by_tma && member == 0) {
      if (elect_one()) tma_store_wait0();
      __syncwarp();
    }
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
  cluster_sync();   // nobody leaves while the other CTA's products read its shared memory or arrive on its barriers
  if (warp == 10) {
    tc_fence_after_sync();
    tmem_dealloc_pair(tm, 512);
  }
}

}  // namespace

int launch_matmul_pair(MatmulArgs a, const void* codes, const void* w_codes, int tile_tokens, int n_sm, cudaStream_t stream) {
  a.tile_tokens = tile_tokens;
  a.n_feature_tiles = ceil_div(a.n_out, 2 * kRows);
  a.n_tiles = static_cast<long long>(a.n_feature_tiles) * ceil_div(a.n_rows, tile_tokens);
  constexpr size_t kSmem = kStages * (kRows + kPairTokens / 2) * kScaleBlock + 1024;
  static_assert(kSmem + sizeof(PairSmem) + 1024 <= 228 * 1024, "shared memory of an SM");
  CUtensorMap tw, ta, to;
  int rc = make_tmap_operand(&tw, w_codes, a.n_out, a.n_cols, kRows);
  if (rc == CRISP_OK) rc = make_tmap_operand(&ta, codes, a.n_rows, a.n_cols, tile_tokens / 2);
  to = ta;   // (unused where rows are not whole vectors of 16 bytes)
  if (rc == CRISP_OK && a.n_out % 8 == 0) rc = make_tmap_product(&to, a.out, a.n_rows, a.n_out, kChunk / 2);
  static std::atomic<unsigned long long> done{0};
  if (rc == CRISP_OK) rc = allow_smem(reinterpret_cast<const void*>(&matmul_pair_kernel), kSmem, &done);
  if (rc != CRISP_OK) return rc;
  const long long pairs = a.n_tiles < n_sm / 2 ? a.n_tiles : n_sm / 2;
  CRISP_KERNEL("matmul_pair", stream, launch_pdl_cluster(matmul_pair_kernel, dim3(static_cast<unsigned>(2 * pairs)), dim3(kThreads),
                                                         kSmem, 2, stream, tw, ta, to, a));
  CRISP_CUDA_TRY(cudaGetLastError(), "matmul: launch");
  return CRISP_OK;
}

}  // namespace crisp
