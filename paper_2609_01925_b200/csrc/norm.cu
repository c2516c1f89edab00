// Rows in: the residual's addition, the root-mean-square norm and the conversion to 8 bits; all bound by HBM (or, for a few
// rows, by latency).
//
// norm: h = bf16(x + residual) (or x), y = h / sqrt(mean(h^2) + eps) * weight.  A row lives in the registers of one CTA
// between its only read and its only write: 8 bytes of traffic per element (x, residual, h, and one byte of codes makes 7)
// instead of the 16 and more of separate passes.  What is normalised is h as stored, so that the result does not depend on
// whether the addition was part of this call.  The sum of squares is held in fp32
// (of tiny rows, of the row times 2^100: see kTiny).
//
// Measured: 131072 rows of 4096, addition, 8 bits out: 558 us, 6.7 TB/s; 9001 rows of 3584, 16 bits out: 20 us; one row: 1.9 us.
// quantize, 32768 rows of 4096: 62.7 us, 6.4 TB/s; 6144 rows: 13.0 us.
#include "cache.cuh"
#include "operand.cuh"

namespace crisp {
namespace {

__device__ __forceinline__ uint4 load16(const void* base, size_t offset) {
  return *reinterpret_cast<const uint4*>(static_cast<const char*>(base) + offset);
}
// The same for what is read once and should leave L2 to what is written.
__device__ __forceinline__ uint4 load16_once(const void* base, size_t offset) {
  return __ldcs(reinterpret_cast<const uint4*>(static_cast<const char*>(base) + offset));
}
__device__ __forceinline__ uint32_t add_bf16x2(uint32_t a, uint32_t b) {
  const float lo = __uint_as_float(a << 16) + __uint_as_float(b << 16);
  const float hi = __uint_as_float(a & 0xffff0000u) + __uint_as_float(b & 0xffff0000u);
  const __nv_bfloat162 r = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&r);
}

struct NormArgs {
  const void *x, *residual, *weight;
  void *sum, *y, *codes;
  uint8_t* scales;
  int n_rows, n_cols;
  float eps;
};

// Rows per CTA: four where a warp has a row of its own.
__host__ __device__ constexpr int norm_rows(int threads) { return threads == 32 ? 4 : 1; }

// CTAs of an SM, which bound a thread's registers: three of 256 threads where a row is two streams (see launch_norm).
__host__ __device__ constexpr int norm_ctas(int threads, bool residual) {
  return threads >= 512 ? 1024 / threads : (residual ? 768 : 1024) / (threads * norm_rows(threads));
}

// Below this mean of squares and eps, squares lose bits to fp32's range (down to it 2^-150 each, which is nothing).
constexpr float kTinyMean = 0x1p-100f;

// kThreads threads of a row hold kVecs vectors of 8 elements each; 16 neighbouring lanes hold a block of 128 columns.
//
// kTiny: eps does not keep the mean above kTinyMean.  Rows below it are taken times 2^100, exact in bf16 and with squares below
// 2^116, and eps times 2^200; the factor cancels.  Other calls do without the branch, in front of which the compiler moves
// nothing (32768 rows of 4096 to 8 bits: 80 us without, 97 with; with addition 141 and 142).
template <int kThreads, int kVecs, bool kResidual, bool kQuantize, bool kTiny>
__global__ void __launch_bounds__(kThreads * norm_rows(kThreads), norm_ctas(kThreads, kResidual)) norm_kernel(const NormArgs a) {
  constexpr int kWarps = kThreads / 32, kRows = norm_rows(kThreads);
  __shared__ float part[2][kWarps < 4 ? 4 : kWarps];
  pdl_enter();
  const int tid = threadIdx.x % kThreads, lane = tid & 31, warp = tid >> 5;
  const long long step = static_cast<long long>(gridDim.x) * kRows;
  const int blocks = (a.n_cols + kScaleBlock - 1) / kScaleBlock;
  const int scale_row = 4 * ((a.n_cols + kScaleWord - 1) / kScaleWord);
  const size_t row_bytes = static_cast<size_t>(a.n_cols) * 2;
  bool mine[kVecs];
  uint4 w[kVecs], x[kVecs], r[kVecs];
  auto fetch = [&](long long row) {
#pragma unroll
    for (int v = 0; v < kVecs; ++v) {
      if (!mine[v]) continue;
      const size_t at = row * row_bytes + static_cast<size_t>(v * kThreads + tid) * 16;
      // (9001 rows of 3584 to bf16: 22.6 -> 20.0 us; with a second stream, 131072 rows of 4096, it costs 563 -> 578)
      x[v] = kResidual ? load16(a.x, at) : load16_once(a.x, at);
      if (kResidual) r[v] = load16(a.residual, at);
    }
  };
#pragma unroll
  for (int v = 0; v < kVecs; ++v) {
    mine[v] = (v * kThreads + tid) * 8 < a.n_cols;
    x[v] = r[v] = make_uint4(0, 0, 0, 0);
    w[v] = make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u);
  }
  long long row = static_cast<long long>(blockIdx.x) * kRows + threadIdx.x / kThreads;
  if (row < a.n_rows) fetch(row);
#pragma unroll
  for (int v = 0; v < kVecs; ++v)
    if (a.weight && mine[v]) w[v] = load16(a.weight, static_cast<size_t>(v * kThreads + tid) * 16);

  for (int turn = 0; row < a.n_rows; row += step, turn ^= 1) {
    uint4 h[kVecs];
    uint64_t ss2 = 0;   // even and odd columns
#pragma unroll
    for (int v = 0; v < kVecs; ++v) {
      h[v] = x[v];
      if (kResidual) {
        h[v] = make_uint4(add_bf16x2(x[v].x, r[v].x), add_bf16x2(x[v].y, r[v].y), add_bf16x2(x[v].z, r[v].z),
                          add_bf16x2(x[v].w, r[v].w));
        if (mine[v])
          *reinterpret_cast<uint4*>(static_cast<char*>(a.sum) + row * row_bytes +
                                    static_cast<size_t>(v * kThreads + tid) * 16) = h[v];
      }
      float f[8];
      unpack_bf16(h[v], f);
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        const uint64_t p = pack2(f[i], f[i + 1]);
        ss2 = fma2(p, p, ss2);
      }
    }
    float ss, odd;
    unpack2(ss2, ss, odd);
    ss += odd;
    // the next row is on its way while this one's sum is joined
    if (row + step < a.n_rows) fetch(row + step);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    if (kWarps > 1) {
      if (lane == 0) part[turn][warp] = ss;
      __syncthreads();   // one per row: the other half of `part` is free once everybody has passed it
      ss = 0.f;
#pragma unroll
      for (int i = 0; i < kWarps; ++i) ss += part[turn][i];
    }
    float m = ss / static_cast<float>(a.n_cols) + a.eps;
    if (kTiny && m < kTinyMean) {   // (the same for all of the row's threads)
      ss = 0.f;
#pragma unroll
      for (int v = 0; v < kVecs; ++v) {
        uint32_t* u = reinterpret_cast<uint32_t*>(&h[v]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float lo = __uint_as_float(u[i] << 16) * 0x1p100f, hi = __uint_as_float(u[i] & 0xffff0000u) * 0x1p100f;
          ss = fmaf(lo, lo, fmaf(hi, hi, ss));
          u[i] = __float_as_uint(hi) | __float_as_uint(lo) >> 16;
        }
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
      if (kWarps > 1) {
        __syncthreads();   // everybody has read this half of `part`
        if (lane == 0) part[turn][warp] = ss;
        __syncthreads();
        ss = 0.f;
#pragma unroll
        for (int i = 0; i < kWarps; ++i) ss += part[turn][i];
      }
      m = ss / static_cast<float>(a.n_cols) + a.eps * 0x1p100f * 0x1p100f;
    }
    const float s0 = rsqrtf(m);
    // one step of Newton: half a rounding instead of two (not where squares have left fp32, and the row becomes 0)
    const float s = m < INFINITY ? fmaf(0.5f * s0, fmaf(-m * s0, s0, 1.f), s0) : s0;
#pragma unroll
    for (int v = 0; v < kVecs; ++v) {
      float f[8], g[8];
      unpack_bf16(h[v], f);
      unpack_bf16(w[v], g);
#pragma unroll
      for (int i = 0; i < 8; i += 2)
        unpack2(mul2(mul2(pack2(f[i], f[i + 1]), pack2(s, s)), pack2(g[i], g[i + 1])), f[i], f[i + 1]);
      const size_t vec = static_cast<size_t>(v * kThreads + tid);
      if (kQuantize) {
        float inverse;
        const uint32_t byte = scale_byte(block_amax(f), inverse);
        if (mine[v]) {
          *reinterpret_cast<uint2*>(static_cast<char*>(a.codes) + static_cast<size_t>(row) * a.n_cols + vec * 8) =
              pack_codes(f, inverse);
          if ((tid & 15) == 0) a.scales[static_cast<size_t>(row) * scale_row + (vec >> 4)] = static_cast<uint8_t>(byte);
        }
      } else if (mine[v]) {
        uint32_t o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const __nv_bfloat162 p = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
          o[i] = *reinterpret_cast<const uint32_t*>(&p);
        }
        *reinterpret_cast<uint4*>(static_cast<char*>(a.y) + row * row_bytes + vec * 16) = make_uint4(o[0], o[1], o[2], o[3]);
      }
    }
    if (kQuantize && tid < scale_row - blocks) a.scales[static_cast<size_t>(row) * scale_row + blocks + tid] = kScaleOne;
  }
}

constexpr int kQuantThreads = 256, kQuantRows = 4;

// 2^tx_log threads share a row (16 for each block of 128 columns), every thread has one vector of kQuantRows rows.  kWide: more
// groups of columns than blockIdx.y counts, from 2^27 columns on (apart: asking costs ordinary calls up to 1 %).
template <bool kWide>
__global__ void __launch_bounds__(kQuantThreads) quantize_kernel(const void* x, int n_rows, int n_cols, int tx_log, void* codes,
                                                                 uint8_t* scales) {
  pdl_enter();
  const int tx = threadIdx.x & ((1 << tx_log) - 1), ty = threadIdx.x >> tx_log, step = kQuantThreads >> tx_log;
  const int blocks = (n_cols + kScaleBlock - 1) / kScaleBlock;
  const int scale_row = 4 * ((n_cols + kScaleWord - 1) / kScaleWord);
  const long long across = kWide ? static_cast<long long>(blockIdx.z) * gridDim.y + blockIdx.y : blockIdx.y;
  const long long vec = (across << tx_log) + tx;
  const bool inside = vec * 8 < n_cols;
  const long long row0 = static_cast<long long>(blockIdx.x) * (step * kQuantRows) + ty;
  uint4 v[kQuantRows];
#pragma unroll
  for (int i = 0; i < kQuantRows; ++i) {
    const long long row = row0 + i * step;
    v[i] = inside && row < n_rows ? load16(x, (static_cast<size_t>(row) * n_cols + vec * 8) * 2) : make_uint4(0, 0, 0, 0);
  }
#pragma unroll
  for (int i = 0; i < kQuantRows; ++i) {
    const long long row = row0 + i * step;
    float f[8], inverse;
    unpack_bf16(v[i], f);
    const uint32_t byte = scale_byte(block_amax(f), inverse);
    if (row >= n_rows) continue;
    if (inside) {
      *reinterpret_cast<uint2*>(static_cast<char*>(codes) + static_cast<size_t>(row) * n_cols + vec * 8) = pack_codes(f, inverse);
      if ((tx & 15) == 0) scales[static_cast<size_t>(row) * scale_row + (vec >> 4)] = static_cast<uint8_t>(byte);
    }
    if (across == 0 && tx < scale_row - blocks) scales[static_cast<size_t>(row) * scale_row + blocks + tx] = kScaleOne;
  }
}

template <int kThreads, int kVecs, bool kTiny>
int launch_norm(const NormArgs& a, int n_sm, cudaStream_t stream) {
  void (*kernel)(NormArgs) =
      a.residual ? (a.codes ? norm_kernel<kThreads, kVecs, true, true, kTiny> : norm_kernel<kThreads, kVecs, true, false, kTiny>)
                 : (a.codes ? norm_kernel<kThreads, kVecs, false, true, kTiny> : norm_kernel<kThreads, kVecs, false, false, kTiny>);
  // A whole number of rounds of the CTAs that are resident at a time: one (131072 rows of 4096, with addition: 3 per SM 558 us,
  // 4 per SM 715, 8 per SM 590), or several where a CTA's rows are long or short, so that the CTAs of an SM fall out of step (16384
  // rows of 8192: 151 us with one round, 142 with four; 30000 rows of 2048: 72 and 68).
  constexpr int kRounds = kThreads == 512 ? 4 : kThreads == 128 || (kThreads == 1024 && kVecs == 2) ? 2 : 1;
  static std::atomic<int> known[2][2][64];
  int per_sm = 0;
  constexpr int kRows = norm_rows(kThreads);
  const int rc = resident_ctas(reinterpret_cast<const void*>(kernel), kThreads * kRows,
                               known[a.residual != nullptr][a.codes != nullptr], &per_sm);
  if (rc != CRISP_OK) return rc;
  const int most = n_sm * per_sm * kRounds, rows = (a.n_rows + kRows - 1) / kRows;
  CRISP_KERNEL("rms_norm", stream, launch_pdl(kernel, dim3(rows < most ? rows : most), dim3(kThreads * kRows), 0, stream, a));
  CRISP_CUDA_TRY(cudaGetLastError(), "rms_norm: launch");
  return CRISP_OK;
}

template <bool kTiny>
int launch_norm_cols(const NormArgs& a, int n_sm, cudaStream_t stream) {
  if (a.n_cols <= 256) return launch_norm<32, 1, kTiny>(a, n_sm, stream);
  if (a.n_cols <= 512) return launch_norm<32, 2, kTiny>(a, n_sm, stream);
  if (a.n_cols <= 1024) return launch_norm<128, 1, kTiny>(a, n_sm, stream);
  if (a.n_cols <= 2048) return launch_norm<128, 2, kTiny>(a, n_sm, stream);
  if (a.n_cols <= 4096) return launch_norm<256, 2, kTiny>(a, n_sm, stream);
  if (a.n_cols <= 8192) return launch_norm<512, 2, kTiny>(a, n_sm, stream);
  if (a.n_cols <= 16384) return launch_norm<1024, 2, kTiny>(a, n_sm, stream);
  return launch_norm<1024, 4, kTiny>(a, n_sm, stream);
}

}  // namespace

int launch_rms_norm(const void* x, const void* residual, const void* weight, int n_rows, int n_cols, float eps, void* sum,
                    void* y, void* codes, uint8_t* scales, cudaStream_t stream) {
  const NormArgs a{x, residual, weight, sum, y, codes, scales, n_rows, n_cols, eps};
  int n_sm = 0;
  const int rc = current_sm_count(&n_sm);
  if (rc != CRISP_OK) return rc;
  return eps < kTinyMean ? launch_norm_cols<true>(a, n_sm, stream) : launch_norm_cols<false>(a, n_sm, stream);
}

int launch_quantize(const void* x, int n_rows, int n_cols, void* codes, uint8_t* scales, cudaStream_t stream) {
  int tx_log = 4;
  while (tx_log < 8 && (8 << tx_log) < n_cols) ++tx_log;
  const long long vecs = (static_cast<long long>(n_cols) + 7) / 8, rows = static_cast<long long>(kQuantThreads >> tx_log) * kQuantRows;
  const long long across = (vecs + (1 << tx_log) - 1) >> tx_log, deep = (across + 65534) / 65535;   // 3 at most
  const dim3 grid(static_cast<unsigned>((n_rows + rows - 1) / rows), static_cast<unsigned>((across + deep - 1) / deep),
                  static_cast<unsigned>(deep));
  CRISP_KERNEL("quantize", stream, launch_pdl(deep > 1 ? quantize_kernel<true> : quantize_kernel<false>, grid, dim3(kQuantThreads), 0,
                                              stream, x, n_rows, n_cols, tx_log, codes, scales));
  CRISP_CUDA_TRY(cudaGetLastError(), "quantize: launch");
  return CRISP_OK;
}

}  // namespace crisp
