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

constexpr int kNarrowRows = 32;   // query rows per key head that the narrow kernel takes

// Workspace (byte offsets).  rows = n_tokens * q_heads.
struct AttendWs {
  size_t rec;                // call record
  size_t tickets[2];         // of (sequence, key head) and of the prefix's key heads
  size_t o[2], ml[2];        // partials by row: [split][row][head_dim], [split][row]
  size_t warp_o;             // narrow kernel: a piece per warp
  size_t block_o, block_ml;  // and two parts per thread block
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
  int parts;                // parts that are computed apart (1, 2)
  int direct;               // the wide kernel writes `out` itself
  int chained;              // the wide kernel's rows of kOwn run over the prefix first (no kPrefix part)
  int splits[2];            // partials by row that a part leaves
  uint64_t* rec;
  uint64_t call;
  uint64_t* tickets[2];
  float *o[2], *warp_o, *block_o;
  float2 *ml[2], *block_ml;
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

// Adds n partial results (`ml(i)`, `src(i)`: this lane's V columns of partial
// i) to a row whose sums so far are acc, top, sum: a whole warp per row, in
// the order of i, so that results do not depend on timing.
template <int V, class Ml, class Src>
__device__ __forceinline__ void join_partials(int n, Ml ml_of, Src src, float (&acc)[V], float& top, float& sum) {
  const int lane = threadIdx.x & 31;
  for (int i0 = 0; i0 < n; i0 += 32) {
    float2 ml = make_float2(-INFINITY, 0.f);
    if (i0 + lane < n) ml = ml_of(i0 + lane);
    float mx = ml.x;
    for (int d = 16; d; d >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
    mx = fmaxf(mx, top);
    const float old = top == -INFINITY ? 0.f : exp2_approx(top - mx);
    const float f = ml.x == -INFINITY ? 0.f : exp2_approx(ml.x - mx);
    float add = ml.x == -INFINITY ? 0.f : ml.y * f;
    for (int d = 16; d; d >>= 1) add += __shfl_xor_sync(0xffffffffu, add, d);
    if (top != -INFINITY) {
      sum *= old;
#pragma unroll
      for (int k = 0; k < V; ++k) acc[k] *= old;
    }
    sum += add;
    top = mx;
    const int m = min(32, n - i0);
#pragma unroll 4
    for (int j = 0; j < m; ++j) {
      const float fj = __shfl_sync(0xffffffffu, f, j);
      const float* at = src(i0 + j);
      float v[V];
      if (V == 4) {
        const float4 x = __ldcg(reinterpret_cast<const float4*>(at));
        v[0] = x.x;
        v[1] = x.y;
        v[V - 2] = x.z;
        v[V - 1] = x.w;
      } else {
        const float2 x = __ldcg(reinterpret_cast<const float2*>(at));
        v[0] = x.x;
        v[1] = x.y;
      }
      if (fj != 0.f) {   // (a partial that saw nothing holds anything)
#pragma unroll
        for (int k = 0; k < V; ++k) acc[k] += fj * v[k];
      }
    }
  }
}
// The partials by row that `part` left.
template <int D, int V>
__device__ __forceinline__ void join_rows(const AttendParams& p, int part, int64_t row, int n, float (&acc)[V], float& top, float& sum) {
  const int64_t rows = (int64_t)p.b.n_tokens * p.q_heads;
  const int lane = threadIdx.x & 31;
  join_partials<V>(n, [&](int i) { return __ldcg(p.ml[part] + i * rows + row); },
                   [&](int i) { return p.o[part] + (i * rows + row) * D + V * lane; }, acc, top, sum);
}
// Row r of a unit whose parts thread blocks first .. first + n - 1 of the
// narrow kernel left: where it began, then continued.
template <int D, int V>
__device__ __forceinline__ void join_slots(const AttendParams& p, int r_block, int first, int n, int r, float (&acc)[V], float& top,
                                           float& sum) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int k = 0; k < V; ++k) acc[k] = 0.f;
  top = -INFINITY;
  sum = 0.f;
  auto at = [&](int i) { return (2 * (int64_t)(first + i) + (i == 0 ? 1 : 0)) * r_block + r; };
  join_partials<V>(n, [&](int i) { return __ldcg(p.block_ml + at(i)); }, [&](int i) { return p.block_o + at(i) * D + V * lane; }, acc, top, sum);
}
// A finished row: this lane's V columns.
template <int D, int V>
__device__ __forceinline__ void write_row(const AttendParams& p, int64_t row, const float (&acc)[V], float top, float sum) {
  const int lane = threadIdx.x & 31;
  const float k = sum > 0.f ? 1.f / sum : sum;   // (0 where nothing is seen; NaN stays)
  uint32_t* dst = reinterpret_cast<uint32_t*>(p.out + row * D + V * lane);
  if (V == 4) *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16x2(acc[0] * k, acc[1] * k), pack_bf16x2(acc[V - 2] * k, acc[V - 1] * k));
  else *dst = pack_bf16x2(acc[0] * k, acc[1] * k);
  if (p.lse && lane == 0) p.lse[row] = top == -INFINITY ? top : (top + log2_approx(sum)) * 0.69314718056f;
}

// The narrow kernel on `part`; late: behind this call's kernel on the prefix.
int narrow_groups(const sdq_batch* b, int group, int part);   // of 8 query rows
int narrow_warps();                                           // per thread block
cudaError_t launch_narrow(const sdq_cache_s* c, const AttendParams& p, int part, bool late, cudaStream_t st);
// The wide kernel on `part`, and how many ways it splits the keys of a row
// block (p.splits[part]).
int wide_splits(const sdq_cache_s* c, const sdq_batch* b, int q_heads, int part, bool chained);
cudaError_t launch_wide(const sdq_cache_s* c, const AttendParams& p, int part, cudaStream_t st);

}  // namespace sdq
