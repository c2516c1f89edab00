// The pages of the 8-bit K/V cache: allocation (reserve), the quantising write of new tokens (append), branching
// (fork), release (free) and compaction.
//
// A page is free when its reference count is zero; there is no other allocator state, so "the lowest free pages, in
// the order of the batch" defines every allocation, and a plan is one scan of the reference counts by one CTA (512
// counts per warp and step, in ballots).  A plan checks its whole batch before it changes anything.  Page contents
// are moved by a second kernel over all SMs, which reads the plan's list of moves: a stream of 16 KB tiles (one page, one
// KV head, K or V), bound by HBM.  Measured: branching 16 sequences four times each, 8 layers of 8 heads, 150 MB: 28 us with
// the release of the old branches; a compaction that moves 426 MB (read + written): 77 us, 8 of them the plan; releasing 32
// sequences and reserving 32: 8 us.
#include <cuda_fp8.h>

#include "cache.cuh"

namespace crisp {
namespace {

struct Move {
  int src, dst, rows;  // pages and how many of their tokens are copied
};

// Which sequences' latest reserve was refused.  An append takes its place from the sequence's length, so behind a reserve that
// changed nothing it would overwrite the newest tokens; it asks here first.  The codes are kept in the workspace, for the
// cache whose page_table `owner` is; another cache that plans in the same workspace drops them.
struct alignas(16) Refusals {
  const int32_t* owner;
  int any;  // 0: no code is set and the array may hold anything
  int pad;
};

struct PagesWs {
  int* status;         // the workspace's first word
  int* n_moves;        // word 16 of the header
  int* n_left;         // word 17: pages in use after a compaction
  Refusals* refusals;  // words 20 .. 23
  int* refused;        // [max_seqs] status codes, 0 = not refused
  int* marks;          // [max_seqs]
  int* found;    // [n_pages] pages picked by a scan
  int* remap;    // [n_pages]
  Move* moves;   // [n_pages]
};

PagesWs carve(const CacheView& v, void* ws, size_t* total) {
  uint8_t* base = static_cast<uint8_t*>(ws);
  PagesWs w;
  w.status = reinterpret_cast<int*>(base);
  w.n_moves = w.status + 16;
  w.n_left = w.status + 17;
  w.refusals = reinterpret_cast<Refusals*>(w.status + 20);
  size_t off = kWsHeader;
  auto take = [&](size_t bytes) {
    void* p = base + off;
    off += align_up(bytes, 256);
    return p;
  };
  w.refused = static_cast<int*>(take(sizeof(int) * static_cast<size_t>(v.max_seqs)));
  w.marks = static_cast<int*>(take(sizeof(int) * static_cast<size_t>(v.max_seqs)));
  w.found = static_cast<int*>(take(sizeof(int) * static_cast<size_t>(v.pages)));
  w.remap = static_cast<int*>(take(sizeof(int) * static_cast<size_t>(v.pages)));
  w.moves = static_cast<Move*>(take(sizeof(Move) * static_cast<size_t>(v.pages)));
  *total = off;
  return w;
}

constexpr int kPlanThreads = 1024;
constexpr int kScanRows = 16;  // groups of 32 reference counts that a warp holds at a time

// Pages p of [lo, hi) with (refs[p] == 0) == want_free, ascending: the first `most` of them go to out.  Stops early
// once `need` are found; returns how many were seen (all of them when need is not reached).  Whole block.
__device__ int scan_pages(const int* refs, int lo, int hi, bool want_free, int need, int most, int* out,
                          long long* scratch) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  constexpr int kPerWarp = 32 * kScanRows, kStep = kPerWarp * (kPlanThreads / 32);
  int seen = 0;
  for (int base = lo; base < hi && seen < need; base += kStep) {
    const int p0 = base + warp * kPerWarp + lane;
    uint32_t hit[kScanRows];
    int mine = 0;
    int val[kScanRows];
#pragma unroll
    for (int j = 0; j < kScanRows; ++j) val[j] = p0 + 32 * j < hi ? refs[p0 + 32 * j] : (want_free ? 1 : 0);
#pragma unroll
    for (int j = 0; j < kScanRows; ++j) {
      hit[j] = __ballot_sync(0xffffffffu, (val[j] == 0) == want_free);
      mine += __popc(hit[j]);
    }
    // all lanes hold the warp's count; the block's scan runs over it in lane 0
    long long total;
    const long long before = block_exclusive_scan<kPlanThreads>(lane == 0 ? mine : 0, scratch, &total);
    int at = seen + static_cast<int>(__shfl_sync(0xffffffffu, before, 0));
    if (out != nullptr && at < most) {
#pragma unroll
      for (int j = 0; j < kScanRows; ++j) {
        if ((hit[j] >> lane) & 1u) {
          const int k = at + __popc(hit[j] & ((1u << lane) - 1u));
          if (k < most) out[k] = p0 + 32 * j;
        }
        at += __popc(hit[j]);
      }
    }
    seen += static_cast<int>(total);
  }
  __syncthreads();  // out is read by other threads
  return seen;
}

// Largest i in [0, n) with start[i] <= x, for ascending start with start[0] <= x.
__device__ __forceinline__ int find_item(const int* start, int n, int x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (start[mid] <= x) lo = mid; else hi = mid;
  }
  return lo;
}

// One thread, before a plan of cache c uses the workspace's arrays.
__device__ __forceinline__ void drop_others_refusals(const CacheView& c, const PagesWs& w) {
  if (w.refusals->owner != c.page_table) w.refusals->any = 0;
}
// The code that the latest reserve of sequence s was refused with, 0 if it was not.
__device__ __forceinline__ int refusal_of(const CacheView& c, const Refusals& r, const int* refused, int s) {
  return r.any != 0 && r.owner == c.page_table ? refused[s] : 0;
}

// ---------------------------------------------------------------- reserve
__global__ void __launch_bounds__(kPlanThreads)
cache_reserve_kernel(const CacheView c, const int32_t* __restrict__ seq_ids, const int32_t* __restrict__ n_new, int batch,
                     PagesWs w) {
  pdl_enter();
  __shared__ long long scratch[33];
  __shared__ int off[kMaxCacheBatch + 1];  // first of an item's new pages in the list of found ones
  const int tid = threadIdx.x;
  if (tid == 0) drop_others_refusals(c, w);
  for (int i = tid; i < batch; i += kPlanThreads) {
    const int s = seq_ids ? seq_ids[i] : i;
    if (s >= 0 && s < c.max_seqs) w.marks[s] = i;
  }
  __syncthreads();
  const bool any_refused = w.refusals->any != 0;
  int error = 0;
  long long carry = 0;
  for (int base = 0; base < batch; base += kPlanThreads) {
    const int i = base + tid;
    int need = 0;
    if (i < batch) {
      const int s = seq_ids ? seq_ids[i] : i;
      if (s >= 0) {
        const int n = n_new ? n_new[i] : 1;
        if (s >= c.max_seqs || n < 0 || w.marks[s] != i) {
          error = CRISP_ERR_BAD_CACHE;
        } else {
          const int len = c.seq_lens[s], room = c.max_pages * kPage;
          if (len < 0 || len > room) {
            error = CRISP_ERR_BAD_CACHE;
          } else if (n > room - len) {
            error = CRISP_ERR_NO_PAGES;
          } else {
            need = pages_of(len + n) - pages_of(len);
            if (n > 0 && len % kPage != 0) {  // the page that is already begun must belong to this sequence alone
              const int p = c.page_table[static_cast<size_t>(s) * c.max_pages + len / kPage];
              if (p < 0 || p >= c.pages || c.page_refs[p] != 1) error = CRISP_ERR_BAD_CACHE;
            }
          }
        }
      }
    }
    long long total;
    const long long before = block_exclusive_scan<kPlanThreads>(need, scratch, &total);
    if (i < batch) off[i] = static_cast<int>(min(carry + before, static_cast<long long>(c.pages) + 1));
    carry += total;
  }
  const bool short_of_pages = carry > c.pages;
  const int need_all = short_of_pages ? 0 : static_cast<int>(carry);
  if (tid == 0) off[batch] = need_all;
  if (error == 0 && short_of_pages) error = CRISP_ERR_NO_PAGES;
  // an error of any item refuses the whole batch; a broken table is reported before missing pages
  if (__syncthreads_or(error == CRISP_ERR_BAD_CACHE)) error = CRISP_ERR_BAD_CACHE;
  else if (__syncthreads_or(error != 0)) error = CRISP_ERR_NO_PAGES;
  if (error == 0 && need_all > 0 &&
      scan_pages(c.page_refs, 0, c.pages, true, need_all, need_all, w.found, scratch) < need_all)
    error = CRISP_ERR_NO_PAGES;
  if (error != 0) {
    if (!any_refused)
      for (int s = tid; s < c.max_seqs; s += kPlanThreads) w.refused[s] = 0;
    __syncthreads();
    for (int i = tid; i < batch; i += kPlanThreads) {
      const int s = seq_ids ? seq_ids[i] : i;
      if (s >= 0 && s < c.max_seqs && (n_new == nullptr || n_new[i] != 0)) w.refused[s] = error;
    }
    if (tid == 0) {
      w.refusals->owner = c.page_table;
      w.refusals->any = 1;
      cache_fail(w.status, error);
    }
    return;
  }
  if (any_refused)
    for (int i = tid; i < batch; i += kPlanThreads) {
      const int s = seq_ids ? seq_ids[i] : i;
      if (s >= 0) w.refused[s] = 0;
    }
  for (int k = tid; k < need_all; k += kPlanThreads) {
    const int i = find_item(off, batch, k);
    const int s = seq_ids ? seq_ids[i] : i;
    const int page = w.found[k];
    c.page_table[static_cast<size_t>(s) * c.max_pages + pages_of(c.seq_lens[s]) + (k - off[i])] = page;
    c.page_refs[page] = 1;
  }
  __syncthreads();
  for (int i = tid; i < batch; i += kPlanThreads) {
    const int s = seq_ids ? seq_ids[i] : i;
    if (s >= 0) c.seq_lens[s] += n_new ? n_new[i] : 1;
  }
}

// ---------------------------------------------------------------- append
// Codes.  A block (page, head) of K or of V has the scale 2^e with e the smallest integer that brings its largest
// finite magnitude within the format (448 for e4m3, 127 for int8), never below what the block's earlier tokens have
// set.  Powers of two make every product below exact in fp32, so a value is rounded once, to the nearest code (ties
// to even); when a later token raises e, the earlier codes move by 2^(e_old - e), exactly but for bits that leave at
// the bottom, which are rounded the same way.
struct Quant {
  int lead_m, power;  // largest code = (1 + lead_m / 128) 2^power
};
template <int kFormat>
__device__ __forceinline__ constexpr Quant quant_of() {
  return kFormat == CRISP_CACHE_E4M3 ? Quant{96, 8} : Quant{126, 6};
}

// exponent for the largest magnitude given as bf16 bits (finite)
template <int kFormat>
__device__ __forceinline__ int block_exponent(uint32_t amax) {
  constexpr Quant q = quant_of<kFormat>();
  const int e = static_cast<int>(amax >> 7) - 127 - q.power + (static_cast<int>(amax & 127u) > q.lead_m ? 1 : 0);
  return e < -126 ? -126 : e;
}

// Four finite bf16 values (two words of two) times f, a power of two that brings them within the format -> four bytes.
// int8: x f + 1.5 2^23 is one exact product and one rounding to an integer (ties to even), whose low byte is the code;
// a conversion instruction per value would be bound by its pipe's quarter rate.
template <int kFormat>
__device__ __forceinline__ uint32_t encode_finite4(uint32_t w0, uint32_t w1, float f) {
  const float a = __uint_as_float(w0 << 16), b = __uint_as_float(w0 & 0xffff0000u);
  const float c = __uint_as_float(w1 << 16), d = __uint_as_float(w1 & 0xffff0000u);
  if (kFormat == CRISP_CACHE_E4M3) {
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a * f, b * f), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c * f, d * f), __NV_SATFINITE, __NV_E4M3);
    return __byte_perm(lo, hi, 0x5410);
  }
  auto whole = [&](float x) { return __float_as_uint(fmaf(x, f, 12582912.0f)); };
  return __byte_perm(__byte_perm(whole(a), whole(b), 0x0040), __byte_perm(whole(c), whole(d), 0x0040), 0x5410);
}

// four values in units of the scale -> four bytes, infinities and NaN among them
template <int kFormat>
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
  if (kFormat == CRISP_CACHE_E4M3) {
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
    return lo | (hi << 16);
  }
  auto one = [](float x) {  // NaN -> 0, infinities -> +-127
    int i = __float2int_rn(x);
    i = i > 127 ? 127 : (i < -127 ? -127 : i);
    return static_cast<uint32_t>(i) & 0xffu;
  };
  return one(a) | (one(b) << 8) | (one(c) << 16) | (one(d) << 24);
}

// four codes times f (a power of two) -> four codes
template <int kFormat>
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float f) {
  float v[4];
  if (kFormat == CRISP_CACHE_E4M3) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(w >> (16 * i)), __NV_E4M3);
      const float2 x = __half22float2(__half2(h));
      v[2 * i] = x.x * f;
      v[2 * i + 1] = x.y * f;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = static_cast<float>(static_cast<int8_t>(w >> (8 * i))) * f;
  }
  return encode4<kFormat>(v[0], v[1], v[2], v[3]);
}

// One CTA writes the new tokens of one page, one KV head, K or V.  Bound by HBM: 256 B of bf16 in and 128 B of codes
// out per token (40027 tokens of three prompts, 8 heads, int8: 42 us, 5.9 TB/s; 32 single tokens: 4 us); the tokens of the page stay in registers between the search for the largest magnitude and the
// conversion.  Eight threads per token (16 values each: two 16-byte loads, one 16-byte store).
constexpr int kAppendThreads = 256;
template <int kFormat>
__global__ void __launch_bounds__(kAppendThreads)
cache_append_kernel(const CacheView c, int layer, const CacheBatch b, const __nv_bfloat16* __restrict__ k,
                    const __nv_bfloat16* __restrict__ v, int slots_per_item, const PagesWs w) {
  pdl_enter();
  int* status = w.status;
  const Refusals refusals = *w.refusals;  // (beside the loads of the search below)
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int head = blockIdx.y, kind = blockIdx.z;
  // ---- which item and which of its pages: item i owns the slots floor(cu[i] / 128) + 2 i .., which are at least as
  // many as the pages that n tokens can touch (with equal shares: a fixed number of slots per item)
  int i, page_at;
  if (b.cu == nullptr) {
    i = blockIdx.x / slots_per_item;
    page_at = blockIdx.x % slots_per_item;
  } else {
    int lo = 0, hi = b.batch;  // search 32 ways at a time: each step costs one load's latency
    const int slot = blockIdx.x;
    while (hi - lo > 1) {
      const int step = (hi - lo + 31) / 32;
      const int at = lo + lane * step;
      const bool le = at < hi && (b.cu[at] >> 7) + 2 * at <= slot;
      // a malformed cu may give any pattern here: the highest set bit still lies in [lo, hi)
      const uint32_t m = __ballot_sync(0xffffffffu, le) | 1u;
      const int top = 31 - __clz(m);
      lo = lo + top * step;
      hi = min(hi, lo + step);
    }
    i = lo;
    page_at = slot - ((b.cu[i] >> 7) + 2 * i);
    if (page_at < 0) return;
  }
  const CacheItem it = load_item(c, b, i, status);
  if (it.seq < 0 || it.n == 0) return;
  if (const int code = refusal_of(c, refusals, w.refused, it.seq)) {
    if (tid == 0) cache_fail(status, code);
    return;
  }
  if (it.n > it.len) {
    if (tid == 0) cache_fail(status, CRISP_ERR_BAD_CACHE);
    return;
  }
  const int pos0 = it.len - it.n;                  // position of the item's first new token
  const long long at_page = static_cast<long long>(pos0 / kPage) + page_at;
  if (at_page * kPage >= it.len) return;
  if (page_at == 0 && head == 0 && kind == 0 && b.seq_ids != nullptr)  // the same sequence twice: say so
    for (int j = tid; j < i; j += kAppendThreads)
      if (b.seq_ids[j] == it.seq) cache_fail(status, CRISP_ERR_BAD_CACHE);
  const int page = c.page_table[static_cast<size_t>(it.seq) * c.max_pages + at_page];
  // a page that several sequences share is never written
  if (page < 0 || page >= c.pages || c.page_refs[page] != 1) {
    if (tid == 0) cache_fail(status, CRISP_ERR_BAD_CACHE);
    return;
  }
  const int held = page_at == 0 ? pos0 % kPage : 0;  // earlier tokens of this page
  const int first = static_cast<int>(at_page) * kPage + held;
  const int rows = min(kPage - held, it.len - first);
  const size_t block = (static_cast<size_t>(layer) * c.pages + page) * c.heads + head;
  float* scale = (kind == 0 ? c.k_scale : c.v_scale) + block;
  uint8_t* codes = (kind == 0 ? c.k_codes : c.v_codes) + block * kPageTileBytes;
  const __nv_bfloat16* src = (kind == 0 ? k : v) +
                             (static_cast<size_t>(it.t0 + (first - pos0)) * c.heads + head) * kHeadDim;
  const size_t row_stride = static_cast<size_t>(c.heads) * kHeadDim;
  const int old = held > 0 ? (__float_as_int(*scale) >> 23 & 255) - 127 : -127;

  const int part = tid & 7, row0 = tid >> 3;
  uint4 x[4][2];
  uint32_t amax = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int r = row0 + 32 * j;
    if (r < rows) {
      const uint4* p = reinterpret_cast<const uint4*>(src + static_cast<size_t>(r) * row_stride) + part * 2;
      x[j][0] = __ldg(p);
      x[j][1] = __ldg(p + 1);
    } else {
      x[j][0] = x[j][1] = make_uint4(0, 0, 0, 0);
    }
  }
  uint32_t top2 = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const uint32_t wd[4] = {x[j][u].x, x[j][u].y, x[j][u].z, x[j][u].w};
#pragma unroll
      for (int g = 0; g < 4; ++g) top2 = __vmaxu2(top2, wd[g] & 0x7fff7fffu);
    }
  amax = max(top2 & 0xffffu, top2 >> 16);
  const bool finite = amax < 0x7f80u;
  if (!finite) {  // infinities and NaN do not set the scale
    amax = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const uint32_t wd[4] = {x[j][u].x, x[j][u].y, x[j][u].z, x[j][u].w};
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const uint32_t lo = wd[g] & 0x7fffu, hi = (wd[g] >> 16) & 0x7fffu;
          if (lo < 0x7f80u) amax = max(amax, lo);
          if (hi < 0x7f80u) amax = max(amax, hi);
        }
      }
  }
  amax = __reduce_max_sync(0xffffffffu, amax);
  __shared__ uint32_t warp_max[kAppendThreads / 32];
  if (lane == 0) warp_max[warp] = amax;
  __syncthreads();  // also: *scale has been read by everyone before it is written
  amax = 0;
#pragma unroll
  for (int j = 0; j < kAppendThreads / 32; ++j) amax = max(amax, warp_max[j]);
  int e = block_exponent<kFormat>(amax);
  if (held > 0 && old > e) e = old;
  const float f = pow2i(-e);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int r = row0 + 32 * j;
    if (r >= rows) continue;
    uint32_t out[4];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const uint32_t wd[4] = {x[j][u].x, x[j][u].y, x[j][u].z, x[j][u].w};
      if (finite) {
        out[2 * u] = encode_finite4<kFormat>(wd[0], wd[1], f);
        out[2 * u + 1] = encode_finite4<kFormat>(wd[2], wd[3], f);
      } else {
        float y[8];
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          y[2 * g] = __uint_as_float(wd[g] << 16) * f;
          y[2 * g + 1] = __uint_as_float(wd[g] & 0xffff0000u) * f;
        }
        out[2 * u] = encode4<kFormat>(y[0], y[1], y[2], y[3]);
        out[2 * u + 1] = encode4<kFormat>(y[4], y[5], y[6], y[7]);
      }
    }
    reinterpret_cast<uint4*>(codes + static_cast<size_t>(held + r) * kHeadDim)[part] =
        make_uint4(out[0], out[1], out[2], out[3]);
  }
  if (held > 0 && e > old) {  // the scale has grown: the page's earlier codes move with it
    const float shrink = pow2i(max(old - e, -126));
    for (int r = row0; r < held; r += kAppendThreads / 8) {
      uint4* p = reinterpret_cast<uint4*>(codes + static_cast<size_t>(r) * kHeadDim) + part;
      uint4 old_codes = *p;
      old_codes.x = rescale4<kFormat>(old_codes.x, shrink);
      old_codes.y = rescale4<kFormat>(old_codes.y, shrink);
      old_codes.z = rescale4<kFormat>(old_codes.z, shrink);
      old_codes.w = rescale4<kFormat>(old_codes.w, shrink);
      *p = old_codes;
    }
  }
  if (tid == 0) *scale = pow2i(e);
}

// ---------------------------------------------------------------- fork
__global__ void __launch_bounds__(kPlanThreads)
cache_fork_kernel(const CacheView c, const int32_t* __restrict__ src, const int32_t* __restrict__ dst,
                  const int32_t* __restrict__ n_tokens, int count, int share, PagesWs w) {
  pdl_enter();
  __shared__ long long scratch[33];
  __shared__ int own_off[kMaxCacheBatch + 1];  // first of an item's own (copied) pages in the list of found ones
  __shared__ int all_off[kMaxCacheBatch + 1];  // first of an item's pages among those of all items
  const int tid = threadIdx.x;
  if (tid == 0) drop_others_refusals(c, w);
  for (int i = tid; i < count; i += kPlanThreads)
    if (src[i] >= 0 && dst[i] >= 0 && dst[i] < c.max_seqs) w.marks[dst[i]] = i;
  __syncthreads();
  // tokens that item i copies or shares; 0 for padding.  Every check is made on the state before the call.
  auto tokens_of = [&](int i, int* error) -> int {
    const int a = src[i], d = dst[i];
    if (a < 0 || d < 0) return 0;
    if (a >= c.max_seqs || d >= c.max_seqs || w.marks[d] != i || c.seq_lens[d] != 0) {
      *error = CRISP_ERR_BAD_CACHE;
      return 0;
    }
    const int len = c.seq_lens[a], n = n_tokens ? n_tokens[i] : len;
    if (n < 0 || n > len || len > c.max_pages * kPage) {
      *error = CRISP_ERR_BAD_CACHE;
      return 0;
    }
    return n;
  };
  int error = 0;
  long long carry_own = 0, carry_all = 0;
  const long long limit = 0x7fffffffLL;
  for (int base = 0; base < count; base += kPlanThreads) {
    const int i = base + tid;
    int n = 0;
    if (i < count) n = tokens_of(i, &error);
    const int pages = pages_of(n), mine = share ? pages - n / kPage : pages;
    long long total;
    long long before = block_exclusive_scan<kPlanThreads>(mine, scratch, &total);
    if (i < count) own_off[i] = static_cast<int>(min(carry_own + before, limit));
    carry_own += total;
    before = block_exclusive_scan<kPlanThreads>(pages, scratch, &total);
    if (i < count) all_off[i] = static_cast<int>(min(carry_all + before, limit));
    carry_all += total;
  }
  if (carry_all > limit) error = CRISP_ERR_BAD_CACHE;
  const int all = carry_all > limit ? 0 : static_cast<int>(carry_all);
  if (tid == 0) all_off[count] = all;
  __syncthreads();
  // the source rows must name real pages, or a reference would be counted for none
  for (int k = tid; k < all; k += kPlanThreads) {
    const int i = find_item(all_off, count, k);
    const int p = c.page_table[static_cast<size_t>(src[i]) * c.max_pages + (k - all_off[i])];
    if (p < 0 || p >= c.pages) error = CRISP_ERR_BAD_CACHE;
  }
  if (error == 0 && carry_own > c.pages) error = CRISP_ERR_NO_PAGES;
  if (__syncthreads_or(error == CRISP_ERR_BAD_CACHE)) error = CRISP_ERR_BAD_CACHE;
  else if (__syncthreads_or(error != 0)) error = CRISP_ERR_NO_PAGES;
  const int need = static_cast<int>(carry_own);
  if (error == 0 && need > 0 && scan_pages(c.page_refs, 0, c.pages, true, need, need, w.found, scratch) < need)
    error = CRISP_ERR_NO_PAGES;
  if (tid == 0) *w.n_moves = error == 0 ? need : 0;
  if (error != 0) {
    if (tid == 0) cache_fail(w.status, error);
    return;
  }
  for (int k = tid; k < all; k += kPlanThreads) {
    const int i = find_item(all_off, count, k);
    const int a = src[i], d = dst[i], j = k - all_off[i];
    const int n = n_tokens ? n_tokens[i] : c.seq_lens[a];
    const int from = c.page_table[static_cast<size_t>(a) * c.max_pages + j];
    int to = from;
    if (share && j < n / kPage) {
      atomicAdd(&c.page_refs[from], 1);
    } else {
      const int m = own_off[i] + (share ? 0 : j);
      to = w.found[m];
      c.page_refs[to] = 1;
      w.moves[m] = Move{from, to, min(kPage, n - j * kPage)};
    }
    c.page_table[static_cast<size_t>(d) * c.max_pages + j] = to;
  }
  __syncthreads();
  // (an item without pages leaves its destination empty; the source of any other is no item's destination)
  for (int i = tid; i < count; i += kPlanThreads)
    if (all_off[i + 1] > all_off[i]) c.seq_lens[dst[i]] = n_tokens ? n_tokens[i] : c.seq_lens[src[i]];
}

// ---------------------------------------------------------------- moving page contents (fork, compact)
// Units of one 16 KB tile: (move, layer, head, K or V).  Sources and destinations never overlap: a destination was
// free before the plan.  After a compaction the rows of the page table are rewritten as well.
constexpr int kMoveThreads = 256;
constexpr int kMoveGrid = 32;  // CTAs per SM, in four rounds: a compaction of 426 MB takes 76 us, with one round (8) 84 us
__global__ void __launch_bounds__(kMoveThreads)
cache_move_kernel(const CacheView c, const PagesWs w, int compacting) {
  pdl_enter();
  const int tid = threadIdx.x;
  const long long per_move = 2LL * c.layers * c.heads;
  const long long units = *w.n_moves * per_move;
  for (long long u = blockIdx.x; u < units; u += gridDim.x) {
    const Move m = w.moves[u / per_move];
    const int rest = static_cast<int>(u % per_move), kind = rest & 1;
    const int head = (rest >> 1) % c.heads, layer = (rest >> 1) / c.heads;
    const size_t from = (static_cast<size_t>(layer) * c.pages + m.src) * c.heads + head;
    const size_t to = (static_cast<size_t>(layer) * c.pages + m.dst) * c.heads + head;
    uint8_t* codes = kind == 0 ? c.k_codes : c.v_codes;
    float* scale = kind == 0 ? c.k_scale : c.v_scale;
    const uint4* a = reinterpret_cast<const uint4*>(codes + from * kPageTileBytes);
    uint4* d = reinterpret_cast<uint4*>(codes + to * kPageTileBytes);
    const int n = m.rows * (kHeadDim / 16);
    uint4 x[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (tid + j * kMoveThreads < n) x[j] = __ldcs(a + tid + j * kMoveThreads);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (tid + j * kMoveThreads < n) __stcs(d + tid + j * kMoveThreads, x[j]);
    if (tid == 0) scale[to] = scale[from];
  }
  if (!compacting) return;
  const int left = *w.n_left;
  for (int s = blockIdx.x; s < c.max_seqs; s += gridDim.x) {
    const int len = c.seq_lens[s];
    if (len < 0 || len > c.max_pages * kPage) {
      if (tid == 0) cache_fail(w.status, CRISP_ERR_BAD_CACHE);
      continue;
    }
    int* row = c.page_table + static_cast<size_t>(s) * c.max_pages;
    for (int j = tid; j < pages_of(len); j += kMoveThreads) {
      const int p = row[j];
      if (p < left) continue;
      const int to = p < c.pages ? w.remap[p] : -1;
      if (to >= 0) row[j] = to; else cache_fail(w.status, CRISP_ERR_BAD_CACHE);
    }
  }
}

// ---------------------------------------------------------------- free
// One CTA per listed sequence.  The length is taken with an exchange, so a sequence that is listed twice, or is
// empty, is freed once.
__global__ void __launch_bounds__(256)
cache_free_kernel(const CacheView c, const int32_t* __restrict__ seq_ids, int* status) {
  pdl_enter();
  __shared__ int s_len;
  const int s = seq_ids[blockIdx.x];
  if (s < 0) return;
  if (s >= c.max_seqs) {
    if (threadIdx.x == 0) cache_fail(status, CRISP_ERR_BAD_CACHE);
    return;
  }
  if (threadIdx.x == 0) s_len = atomicExch(&c.seq_lens[s], 0);
  __syncthreads();
  const int len = s_len;
  if (len < 0 || len > c.max_pages * kPage) {
    if (threadIdx.x == 0) {
      c.seq_lens[s] = len;  // what breaks its rule stays
      cache_fail(status, CRISP_ERR_BAD_CACHE);
    }
    return;
  }
  int* row = c.page_table + static_cast<size_t>(s) * c.max_pages;
  for (int j = threadIdx.x; j < pages_of(len); j += blockDim.x) {
    const int p = row[j];
    row[j] = -1;
    if (p < 0 || p >= c.pages) {
      cache_fail(status, CRISP_ERR_BAD_CACHE);
    } else if (atomicSub(&c.page_refs[p], 1) <= 0) {  // was free already
      atomicAdd(&c.page_refs[p], 1);
      cache_fail(status, CRISP_ERR_BAD_CACHE);
    }
  }
}

// ---------------------------------------------------------------- compact
// With U pages in use, the used pages at or above U move, in ascending order, to the free ones below U.
__global__ void __launch_bounds__(kPlanThreads)
cache_compact_kernel(const CacheView c, int32_t* n_used, PagesWs w) {
  pdl_enter();
  __shared__ long long scratch[33];
  const int tid = threadIdx.x, most = c.pages;
  if (tid == 0) drop_others_refusals(c, w);
  const int left = scan_pages(c.page_refs, 0, c.pages, false, 0x7fffffff, 0, nullptr, scratch);
  // the free pages below `left` are as many as the used ones from it on
  const int n = scan_pages(c.page_refs, 0, left, true, 0x7fffffff, most, w.found, scratch);
  scan_pages(c.page_refs, left, c.pages, false, 0x7fffffff, most, w.remap, scratch);
  for (int k = tid; k < n; k += kPlanThreads) {
    const int from = w.remap[k], to = w.found[k];
    w.moves[k] = Move{from, to, kPage};
  }
  __syncthreads();
  for (int p = left + tid; p < c.pages; p += kPlanThreads) w.remap[p] = -1;
  __syncthreads();
  for (int k = tid; k < n; k += kPlanThreads) {
    const Move m = w.moves[k];
    w.remap[m.src] = m.dst;
    c.page_refs[m.dst] = c.page_refs[m.src];
    c.page_refs[m.src] = 0;
  }
  if (tid == 0) {
    *w.n_moves = n;
    *w.n_left = left;
    *n_used = left;
  }
}

}  // namespace

size_t cache_pages_ws_bytes(const CacheView& v) {
  size_t total;
  carve(v, nullptr, &total);
  return total;
}

int launch_cache_reserve(const CacheView& v, const int32_t* seq_ids, const int32_t* n_new, int batch, void* ws,
                         cudaStream_t stream) {
  size_t total;
  const PagesWs w = carve(v, ws, &total);
  CRISP_KERNEL("cache_reserve", stream,
               launch_pdl(cache_reserve_kernel, dim3(1), dim3(kPlanThreads), 0, stream, v, seq_ids, n_new, batch, w));
  CRISP_CUDA_TRY(cudaGetLastError(), "cache_reserve: launch");
  return CRISP_OK;
}

int launch_cache_append(const CacheView& v, int layer, const CacheBatch& b, const void* k, const void* vv, void* ws,
                        cudaStream_t stream) {
  const int slots_per_item = b.cu ? 0 : (b.per + 2 * kPage - 2) / kPage;
  const long long slots = b.cu ? b.n_tokens / kPage + 2LL * b.batch : static_cast<long long>(slots_per_item) * b.batch;
  const dim3 grid(static_cast<unsigned>(slots), v.heads, 2), block(kAppendThreads);
  const auto* kp = static_cast<const __nv_bfloat16*>(k);
  const auto* vp = static_cast<const __nv_bfloat16*>(vv);
  size_t total;
  const PagesWs w = carve(v, ws, &total);
  if (v.format == CRISP_CACHE_E4M3) {
    CRISP_KERNEL("cache_append", stream, launch_pdl(cache_append_kernel<CRISP_CACHE_E4M3>, grid, block, 0, stream, v, layer, b,
                                                    kp, vp, slots_per_item, w));
  } else {
    CRISP_KERNEL("cache_append", stream, launch_pdl(cache_append_kernel<CRISP_CACHE_INT8>, grid, block, 0, stream, v, layer, b,
                                                    kp, vp, slots_per_item, w));
  }
  CRISP_CUDA_TRY(cudaGetLastError(), "cache_append: launch");
  return CRISP_OK;
}

int launch_cache_fork(const CacheView& v, const int32_t* src, const int32_t* dst, const int32_t* n_tokens, int count,
                      int share, void* ws, cudaStream_t stream) {
  size_t total;
  const PagesWs w = carve(v, ws, &total);
  int n_sm = 0;
  const int rc = current_sm_count(&n_sm);
  if (rc != CRISP_OK) return rc;
  const int grid = kMoveGrid * n_sm;
  CRISP_KERNEL("cache_fork", stream, launch_pdl(cache_fork_kernel, dim3(1), dim3(kPlanThreads), 0, stream, v, src, dst,
                                                n_tokens, count, share, w));
  CRISP_KERNEL("cache_move", stream, launch_pdl(cache_move_kernel, dim3(grid), dim3(kMoveThreads), 0, stream, v, w, 0));
  CRISP_CUDA_TRY(cudaGetLastError(), "cache_fork: launch");
  return CRISP_OK;
}

int launch_cache_free(const CacheView& v, const int32_t* seq_ids, int count, void* ws, cudaStream_t stream) {
  CRISP_KERNEL("cache_free", stream, launch_pdl(cache_free_kernel, dim3(count), dim3(256), 0, stream, v, seq_ids,
                                                static_cast<int*>(ws)));
  CRISP_CUDA_TRY(cudaGetLastError(), "cache_free: launch");
  return CRISP_OK;
}

int launch_cache_compact(const CacheView& v, int32_t* n_used, void* ws, cudaStream_t stream) {
  size_t total;
  const PagesWs w = carve(v, ws, &total);
  int n_sm = 0;
  const int rc = current_sm_count(&n_sm);
  if (rc != CRISP_OK) return rc;
  const int grid = kMoveGrid * n_sm;
  CRISP_KERNEL("cache_compact", stream, launch_pdl(cache_compact_kernel, dim3(1), dim3(kPlanThreads), 0, stream, v, n_used, w));
  CRISP_KERNEL("cache_move", stream, launch_pdl(cache_move_kernel, dim3(grid), dim3(kMoveThreads), 0, stream, v, w, 1));
  CRISP_CUDA_TRY(cudaGetLastError(), "cache_compact: launch");
  return CRISP_OK;
}

}  // namespace crisp
