// Paged key / value caches: shared by the kernels that append to them, read them back and attend over them.
#pragma once
#include "sp_common.cuh"

namespace sp {

constexpr int kCacheGroup = SP_CACHE_GROUP;

struct CacheView {
  uint8_t *k, *v, *ks, *vs;                // first page; scales (4 bits): pairs of bf16, scale and offset
  int64_t step, scale_step;                // bytes from a page to the next
  const int32_t* table;
  const int32_t* lens;
  int64_t table_ld;
  int32_t n_pages, page_len, max_pages, n_kv, dh, n_seq;
};

#ifdef __CUDACC__
__device__ __forceinline__ int32_t bounded(int32_t x, int32_t n) { return x < 0 ? 0 : x > n ? n : x; }
// The sequence that row belongs to (the last one that starts at or before it), -1 for none.  All lanes of a warp call with one row.
__device__ __forceinline__ int32_t sequence_of(const int32_t* cu, int32_t n_seq, int32_t rows, int32_t row) {
  const int lane = threadIdx.x & 31;
  int32_t lo = 0, len = n_seq + 1;         // entries lo .. lo + len - 1 are left
  while (true) {
    const int32_t step = (len + 31) / 32, at = lane * step;
    const bool below = at < len && bounded(cu[lo + at], rows) <= row;
    const int32_t k = __popc(__ballot_sync(0xffffffffu, below)) - 1;
    if (k < 0) return -1;                  // (the first probe of all: every sequence starts behind the row)
    lo += k * step;
    len = min(step, len - k * step);
    if (step == 1) return lo < n_seq ? lo : -1;
  }
}
// The same of every lane for itself, and any row: the last one that starts at or before it (the first one if none does).
__device__ __forceinline__ int32_t sequence_near(const int32_t* cu, int32_t n_seq, int32_t rows, int64_t row) {
  int32_t s = 0;
  for (int32_t len = n_seq; len > 1;) {
    const int32_t half = len / 2;
    const bool there = bounded(cu[s + half], rows) <= row;
    s += there ? half : 0;
    len = there ? len - half : half;
  }
  return s;
}
// Page of a sequence's token, -1 where there is none: no such entry of the table, or one that names no page.
__device__ __forceinline__ int32_t page_of(const CacheView& c, int32_t s, int32_t entry) {
  if (entry < 0 || entry >= c.max_pages) return -1;
  const int32_t page = c.table[(int64_t)s * c.table_ld + entry];
  return page >= 0 && page < c.n_pages ? page : -1;
}
#endif

// What every call refuses of a cache (pages: whether it has to have any).
sp_status check_cache(const sp_kv_cache* c, bool pages);
CacheView cache_view(const sp_kv_cache* c);
// Reads n = cu[s + 1] - cu[s] last tokens of every sequence (sp_cache_read).
cudaError_t cache_read(const sp_kv_cache* c, const int32_t* cu, int64_t rows, void* K, void* V, int64_t ldk, int64_t ldv, int32_t dtype,
                       int32_t* status, cudaStream_t stream);
// The same for whole sequences, whole[s] tokens, into contiguous rows of bf16 (those of a sequence with another number than n are NaN); with tops as fp16 in
// the units that these give a text's key head, or bf16 (HalfTops, sp_attention.cuh).  cache_tops finds them among the scales of the same rows, and Q_half
// [Nq, n_heads * d_head] takes the queries alike, q_unit [Nq, n_heads] their units.
struct HalfTops;
cudaError_t cache_open(const sp_kv_cache* c, const int32_t* cu, const int32_t* whole, int64_t rows, void* K, void* V, const HalfTops* tops,
                       int32_t* status, cudaStream_t stream);
cudaError_t cache_tops(const sp_kv_cache* c, const int32_t* cu, const int32_t* whole, int64_t rows, HalfTops* tops, cudaStream_t stream);
cudaError_t queries_to_half(const sp_kv_cache* c, const sp_mat* Q, const int32_t* cu_q, void* Q_half, float* q_unit, const HalfTops* tops,
                            cudaStream_t stream);

}  // namespace sp
