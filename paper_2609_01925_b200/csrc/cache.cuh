// Shared declarations of the 8-bit paged K/V cache (cache_pages.cu, cache_attention.cu).
#pragma once
#include <atomic>

#include "common.cuh"

namespace crisp {

constexpr int kPage = kBlock;              // tokens of a page = the block of the sparse path
constexpr int kPageTileBytes = kPage * kHeadDim;  // codes of one page and KV head, K or V: 16 KB
constexpr int kDecodeRows = 24;  // most rows per KV head for the kernel for few rows
constexpr int kMaxCacheBatch = CRISP_CACHE_MAX_BATCH;

// A crisp_cache passed to kernels by value.
struct CacheView {
  uint8_t *k_codes, *v_codes;   // [layers][pages][heads][128][128]
  float *k_scale, *v_scale;     // [layers][pages][heads]
  int32_t *page_table;          // [max_seqs][max_pages]
  int32_t *seq_lens;            // [max_seqs]
  int32_t *page_refs;           // [pages]
  int format, layers, heads, pages, max_seqs, max_pages;
};

// The sequences of one call: item i is sequence seq_ids[i] (i when seq_ids is null) and owns the packed tokens
// cu[i] .. cu[i+1] - 1 (per .. per of them each when cu is null), the last positions that its length covers.
struct CacheBatch {
  const int32_t* seq_ids;
  const int32_t* cu;
  int batch, n_tokens, per, max_new;
  int lo, hi;  // items with fewer than lo or more than hi tokens are another kernel's
};

// Multiprocessors of the current device (asked once per device).
int current_sm_count(int* n_sm);

// cudaFuncSetAttribute of a kernel's dynamic shared memory, once per device (`done`: a bit per device, the kernel's own).
int allow_smem(const void* kernel, size_t bytes, std::atomic<unsigned long long>* done);

// CTAs of a kernel without dynamic shared memory that an SM holds at a time, asked once per device (`known`: 64 numbers, the
// kernel's own).
int resident_ctas(const void* kernel, int threads, std::atomic<int>* known, int* per_sm);

int check_cache(const crisp_cache* c, CacheView* v);
int check_batch(const int32_t* seq_ids, const int32_t* cu, int32_t batch, int32_t n_tokens,
                int32_t max_new, CacheBatch* b);

// Tensor map of the code tiles, [rows][128] bytes, with a {128, box_rows} box and 128-byte swizzle.
int make_tmap_codes(CUtensorMap* out, const void* base, size_t rows, int box_rows);

int launch_cache_reserve(const CacheView& v, const int32_t* seq_ids, const int32_t* n_new, int batch, void* ws,
                         cudaStream_t stream);
int launch_cache_append(const CacheView& v, int layer, const CacheBatch& b, const void* k, const void* vv, void* ws,
                        cudaStream_t stream);
int launch_cache_fork(const CacheView& v, const int32_t* src, const int32_t* dst, const int32_t* n_tokens, int count,
                      int share, void* ws, cudaStream_t stream);
int launch_cache_free(const CacheView& v, const int32_t* seq_ids, int count, void* ws, cudaStream_t stream);
int launch_cache_compact(const CacheView& v, int32_t* n_used, void* ws, cudaStream_t stream);
// Attention: the kernel for few rows per KV head (cache_attention.cu) and the one for many (cache_prefill.cu).  The
// workspace is the header, then each kernel's part; *_ws returns the offset behind it.
int launch_cache_decode(const CacheView& v, int layer, const CacheBatch& b, int n_q_heads, float scale, const void* q,
                        void* o, float* lse, void* ws, size_t ws_off, const CUtensorMap& tk, const CUtensorMap& tv, int n_sm,
                        cudaStream_t stream);
int launch_cache_prefill(const CacheView& v, int layer, const CacheBatch& b, int n_q_heads, float scale, const void* q,
                         void* o, float* lse, void* ws, size_t ws_off, const CUtensorMap& tk, const CUtensorMap& tv, int n_sm,
                         cudaStream_t stream);
size_t cache_decode_ws(void* ws, size_t off);
size_t cache_prefill_ws(void* ws, size_t off);
size_t cache_pages_ws_bytes(const CacheView& v);

#ifdef __CUDACC__
__host__ __device__ __forceinline__ int pages_of(int tokens) { return (tokens + kPage - 1) / kPage; }

// The first error of a workspace stays in its status word until it is polled.
__device__ __forceinline__ void cache_fail(int* status, int code) { atomicCAS(status, 0, code); }

struct CacheItem {
  int seq, len, t0, n;  // t0: first packed token; n: new tokens; seq < 0: nothing to do
};

// Item i of a batch, with everything that it names checked: a padding entry (negative sequence) and an entry that
// breaks a rule both come back with seq = -1, the latter with the status word set.
__device__ __forceinline__ CacheItem load_item(const CacheView& c, const CacheBatch& b, int i, int* status) {
  CacheItem it;
  it.seq = b.seq_ids ? b.seq_ids[i] : i;
  it.t0 = b.cu ? b.cu[i] : i * b.per;
  it.n = b.cu ? b.cu[i + 1] - it.t0 : b.per;
  it.len = 0;
  if (it.seq < 0) return it;
  bool bad = it.seq >= c.max_seqs || it.t0 < 0 || it.n < 0 || it.n > b.max_new || it.t0 > b.n_tokens - it.n;
  if (!bad) {
    it.len = c.seq_lens[it.seq];
    bad = it.len < 0 || it.len > c.max_pages * kPage;
  }
  if (bad) cache_fail(status, CRISP_ERR_BAD_CACHE);
  if (bad || it.n < b.lo || it.n > b.hi) {
    it.seq = -1;
    it.len = 0;
  }
  return it;
}

// 2^e for -126 <= e <= 127.
__device__ __forceinline__ float pow2i(int e) { return __int_as_float((e + 127) << 23); }
#endif

}  // namespace crisp
