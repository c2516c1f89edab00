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
#include <atomic>

#include "matmul.cuh"
#include "sm100_ptx.cuh"

namespace crisp {
namespace {

using namespace sm100;

constexpr int kTileFeatures = 128;
constexpr int kMatmulThreads = 192;    // warps 0..3: scales, then the epilogue; 4: TMA; 5: MMA
constexpr int kMaxStages = 12;
constexpr int kScaleSlots = 4;         // words of scales (512 columns) in TMEM at a time
constexpr int kMaxSplit = 8;           // CTAs of a cluster
constexpr uint32_t kOnes = 0x7f7f7f7fu;  // four scales of one

struct __align__(16) MatmulSmem {
  uint64_t full[kMaxStages], empty[kMaxStages], scale_full[kScaleSlots], scale_empty[kScaleSlots], done;
  uint32_t tmem;
  int abort_flag;
};

__device__ __forceinline__ uint32_t scale_word(const uint8_t* scales, long long row, int rows, int words, int word) {
  return row < rows ? *reinterpret_cast<const uint32_t*>(scales + (row * words + word) * 4) : kOnes;
}

__global__ void __launch_bounds__(kMatmulThreads, 1) matmul_kernel(const __grid_constant__ CUtensorMap tw,
                                                                   const __grid_constant__ CUtensorMap ta, const MatmulArgs a) {
  extern __shared__ __align__(1024) uint8_t raw[];
  __shared__ MatmulSmem s;
  uint8_t* ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~static_cast<uintptr_t>(1023));
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = a.split > 1 ? static_cast<int>(cluster_rank()) : 0;
  const int tile = blockIdx.x / a.split;
  const int f0 = (tile % a.n_feature_tiles) * kTileFeatures;
  const int t0 = (tile / a.n_feature_tiles) * a.tile_tokens;
  const int blocks = (a.n_cols + kScaleBlock - 1) / kScaleBlock, words = (a.n_cols + kScaleWord - 1) / kScaleWord;
  const int k0 = static_cast<int>(static_cast<long long>(rank) * blocks / a.split);
  const int k1 = static_cast<int>(static_cast<long long>(rank + 1) * blocks / a.split);
  const int stage_bytes = (kTileFeatures + a.tile_tokens) * kScaleBlock;
  const int token_cells = (a.tile_tokens + 31) / 32;            // TMEM columns of the tokens' scales
  const int slot_cols = token_cells > 4 ? 12 : 8;
  pdl_enter();
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
  if (warp == 5) {
    tmem_alloc(&s.tmem, a.tmem_cols);
    tmem_relinquish();
    tc_fence_before_sync();
  }
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tm = s.tmem;
  volatile int* abort_flag = &s.abort_flag;

  if (warp == 4) {
    if (lane == 0) {
      prefetch_tmap(&tw);
      prefetch_tmap(&ta);
      int stage = 0;
      uint32_t phase = 0;
      for (int kb = k0; kb < k1; ++kb) {
        if (kb - k0 >= a.stages && !mbar_wait(&s.empty[stage], phase ^ 1u, abort_flag)) break;
        uint8_t* slot = ring + stage * stage_bytes;
        mbar_arrive_expect_tx(&s.full[stage], stage_bytes);
        tma_load_2d(slot, &tw, &s.full[stage], kb * kScaleBlock, f0);
        tma_load_2d(slot + kTileFeatures * kScaleBlock, &ta, &s.full[stage], kb * kScaleBlock, t0);
        if (++stage == a.stages) {
          stage = 0;
          phase ^= 1u;
        }
      }
    }
    __syncwarp();
  } else if (warp == 5) {
    if (lane == 0) {
      int stage = 0, slot = 0;
      uint32_t phase = 0, slot_phase = 0;
      bool ok = true;
      for (int kb = k0; kb < k1 && ok; ++kb) {
        if (kb == k0 || (kb & 3) == 0) ok = mbar_wait(&s.scale_full[slot], slot_phase, abort_flag);
        ok = ok && mbar_wait(&s.full[stage], phase, abort_flag);
        if (!ok) break;
        tc_fence_after_sync();
        const uint32_t at = smem_u32(ring + stage * stage_bytes);
        const uint64_t wd = umma_desc_sw128(at, 0, 1024), ad = umma_desc_sw128(at + kTileFeatures * kScaleBlock, 0, 1024);
        const uint32_t idesc = umma_idesc_mx_e4m3(kTileFeatures, a.tile_tokens, kb & 3);
        const uint32_t sc = tm + static_cast<uint32_t>(a.tile_tokens + 31) / 32 * 32 + slot * slot_cols;
#pragma unroll
        for (int i = 0; i < 4; ++i)   // 32 columns each
          umma_mx_ss(tm, wd + 2 * i, ad + 2 * i, idesc, sc, sc + 4, kb > k0 || i > 0);
        umma_commit(&s.empty[stage]);
        if (++stage == a.stages) {
          stage = 0;
          phase ^= 1u;
        }
        if ((kb & 3) == 3) {
          umma_commit(&s.scale_empty[slot]);
          if (++slot == kScaleSlots) {
            slot = 0;
            slot_phase ^= 1u;
          }
        }
      }
      if (ok) umma_commit(&s.done);
    }
    __syncwarp();
  } else {
    const uint32_t quarter = tm + (static_cast<uint32_t>(warp * 32) << 16);
    const uint32_t scale_base = quarter + (a.tile_tokens + 31) / 32 * 32;
    uint32_t next[12];
    auto fetch = [&](int word) {
#pragma unroll
      for (int c = 0; c < 4; ++c) next[c] = scale_word(a.w_scales, static_cast<long long>(f0) + 32 * c + lane, a.n_out, words, word);
#pragma unroll
      for (int c = 0; c < 8; ++c)
        next[4 + c] = c < token_cells ? scale_word(a.scales, static_cast<long long>(t0) + 32 * c + lane, a.n_rows, words, word) : kOnes;
    };
    const int w0 = k0 >> 2, w1 = (k1 + 3) >> 2;
    bool ok = true;
    fetch(w0);
    for (int word = w0; word < w1; ++word) {
      const int i = word - w0, slot = i % kScaleSlots;
      if (i >= kScaleSlots) ok = mbar_wait_warp(&s.scale_empty[slot], (i / kScaleSlots - 1) & 1, abort_flag);
      if (!ok) break;
      if (i >= kScaleSlots) tc_fence_after_sync();
      const uint32_t at = scale_base + slot * slot_cols;
      tmem_st_x4(at, next);
      tmem_st_x4(at + 4, next + 4);
      if (slot_cols > 8) tmem_st_x4(at + 8, next + 8);
      if (word + 1 < w1) fetch(word + 1);
      tmem_st_wait();
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive(&s.scale_full[slot]);
    }
    ok = ok && mbar_wait_warp(&s.done, 0, abort_flag);
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
    if (tid < kTileFeatures && f0 + tid < a.n_out) {
      // the tokens are dealt to the CTAs; each sums its own in the order of the columns
      const int n = min(a.tile_tokens, a.n_rows - t0);
      const uint32_t mine = smem_u32(ring) + tid * 4;
      for (int t = rank * n / a.split; t < (rank + 1) * n / a.split; ++t) {
        float sum = 0.f;
        for (int p = 0; p < a.split; ++p) sum += cluster_load(cluster_map(mine + t * (kTileFeatures * 4), p));
        a.out[static_cast<size_t>(t0 + t) * a.n_out + f0 + tid] = __float2bfloat16_rn(sum);
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
  if (warp == 5) {
    tc_fence_after_sync();
    tmem_dealloc(tm, a.tmem_cols);
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
  if (n_rows > 256) return launch_matmul_pair(a, codes, w_codes, 224, n_sm, stream);
  a.tile_tokens = n_rows >= 256 ? 256 : ceil_div(n_rows, 16) * 16;
  a.n_feature_tiles = ceil_div(n_out, kTileFeatures);
  const long long tiles = static_cast<long long>(a.n_feature_tiles) * ceil_div(n_rows, a.tile_tokens);
  const int blocks = ceil_div(n_cols, kScaleBlock);
  if (tiles > INT32_MAX) return CRISP_ERR_UNSUPPORTED;
  int split = static_cast<int>(tiles >= n_sm ? 1 : n_sm / tiles);
  if (split > kMaxSplit) split = kMaxSplit;
  if (split > blocks) split = blocks;
  a.split = split;
  // accumulators, then the slots of scales; an SM holds one CTA of the wide tiles and two of the others, so that the CTAs of
  // an SM never want more than its 512 columns
  const int used = ceil_div(a.tile_tokens, 32) * 32 + kScaleSlots * (a.tile_tokens > 128 ? 12 : 8);
  a.tmem_cols = 32;
  while (a.tmem_cols < used) a.tmem_cols *= 2;
  const int budget = (a.tmem_cols > 256 ? 200 : 104) * 1024, stage_bytes = (kTileFeatures + a.tile_tokens) * kScaleBlock;
  a.stages = budget / stage_bytes < kMaxStages ? budget / stage_bytes : kMaxStages;
  const size_t smem = budget + 1024;
  CUtensorMap tw, ta;
  rc = make_tmap_operand(&tw, w_codes, n_out, n_cols, kTileFeatures);
  if (rc == CRISP_OK) rc = make_tmap_operand(&ta, codes, n_rows, n_cols, a.tile_tokens);
  static std::atomic<unsigned long long> done{0};
  if (rc == CRISP_OK) rc = allow_smem(reinterpret_cast<const void*>(&matmul_kernel), 200 * 1024 + 1024, &done);
  if (rc != CRISP_OK) return rc;
  CRISP_KERNEL("matmul", stream, launch_pdl_cluster(matmul_kernel, dim3(static_cast<unsigned>(tiles * split)),
                                                    dim3(kMatmulThreads), smem, split, stream, tw, ta, a));
  CRISP_CUDA_TRY(cudaGetLastError(), "matmul: launch");
  return CRISP_OK;
}

}  // namespace crisp
