// The paged cache and what its kernels share (contracts in include/sdq.h).
#pragma once

#include "common.cuh"

struct sdq_cache_s {
  sdq_cache_desc desc;
  int device, sm_count;
  uint16_t *k, *v;
  int64_t rows;          // token rows of each array: n_pages * kv_heads * page_tokens
  CUtensorMap kmap, vmap;     // rows x head_dim in boxes of min(page_tokens, 64) rows x 64 elements, 128-byte swizzle
  CUtensorMap ktile, vtile;   // 64 elements x rows x halves of a row in boxes of 16 rows, all of their elements
};

namespace sdq {

// Rows of one box of the cache's tensor maps.
inline int cache_box_rows(const sdq_cache_desc& d) { return d.page_tokens < 64 ? d.page_tokens : 64; }
// SDQ_OK, or why `b` cannot be run on `c` (host values only).
int check_batch(const sdq_cache_s* c, const sdq_batch* b, int32_t q_heads);
// SDQ_OK when the current device is the cache's.
int check_cache_device(const sdq_cache_s* c);

// New tokens [first, first + count) of sequence s, and its own tokens, within
// the bounds that the host gave (whatever the device arrays hold).
struct SeqSpan {
  int first, count, own;
};
__device__ __forceinline__ SeqSpan seq_span(const sdq_batch& b, int s) {
  SeqSpan r;
  r.first = min(max(b.token_start[s], 0), b.n_tokens);
  const int end = min(max(b.token_start[s + 1], 0), b.n_tokens);
  r.count = min(max(end - r.first, 0), b.max_new);
  r.own = min(max(b.own_len[s], 0), b.max_own);
  return r;
}
// The sequence of token t: the last s with token_start[s] <= t (empty ones
// before it have the same start).
__device__ __forceinline__ int seq_of_token(const int32_t* start, int n_seqs, int t) {
  int lo = 0, hi = n_seqs - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (start[mid] <= t) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

}  // namespace sdq
