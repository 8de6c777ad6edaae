// What the attention kernels share (contracts in include/sdq.h).
#pragma once

#include "cache.cuh"

namespace sdq {

// A part of the keys of a call: each sequence's own tokens, or the shared prefix.
constexpr int kOwn = 0, kPrefix = 1;
// Keys of one tile of a page table are whole tiles from its first token on.
// Scores are kept in log2 units: s = scale log2(e) q.k, weights 2^(s - m).
// A partial result of a row (token, query head; index token * q_heads + head)
// over some of its keys: the fp32 sum of 2^(s - m) v, and (m, sum of 2^(s -
// m)); m = -inf where it saw none.

// Workspace (byte offsets).  rows = n_tokens * q_heads.
struct AttendWs {
  size_t rec;               // call record
  size_t base;              // first global tile of each sequence (int64 x n_seqs)
  size_t o[2], ml[2];       // partials by row: [split][row][head_dim], [split][row]
  size_t slot_o, slot_ml;   // partials of row blocks continued from the thread block before
  size_t total;
};

struct AttendParams {
  sdq_batch b;
  const uint16_t* q;
  int64_t ldq;              // elements between tokens
  uint16_t* out;
  float* lse;               // natural log-sum-exp per row, may be null
  float scale;              // softmax scale times log2(e)
  int q_heads, kv_heads, group, page_shift, box_shift, n_pages;
  int narrow[2], wide[2];   // which kernel takes a part (neither: it has no keys)
  int direct;               // one part only: whole rows may go straight to `out`
  int chained;              // the wide kernel's rows of kOwn run over the prefix first (no kPrefix part)
  int splits[2];            // partials by row of each part that the join reads
  uint64_t* rec;
  uint64_t call;
  int64_t* base;
  float *o[2], *slot_o;
  float2 *ml[2], *slot_ml;
  int ctas;                 // thread blocks of the narrow kernel
};

__device__ __forceinline__ float exp2_approx(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;\n" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float log2_approx(float x) {
  float r;
  asm("lg2.approx.f32 %0, %1;\n" : "=f"(r) : "f"(x));
  return r;
}

// The wide kernel on `part`, and how many ways it splits the keys of a row
// block (p.splits[part]).
int wide_splits(const sdq_cache_s* c, const sdq_batch* b, int q_heads, int part, bool chained);
cudaError_t launch_wide(const sdq_cache_s* c, const AttendParams& p, int part, cudaStream_t st);

}  // namespace sdq
