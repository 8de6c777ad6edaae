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
  size_t o[2], ml[2];        // two parts' results by row, for their join
  size_t split_o[2], split_ml[2];   // wide kernel: [thread block of a row block's][row]
  size_t warp_o[2];          // narrow kernel: a piece per warp
  size_t block_o[2], block_ml[2];   // and two parts per thread block
  size_t total;
};

struct AttendParams {
  sdq_batch b;
  const uint16_t *q, *v;    // v: the cache's values
  int64_t ldq;              // elements between tokens
  uint16_t* out;
  float* lse;               // natural log-sum-exp per row, may be null
  float scale;              // softmax scale times log2(e)
  int q_heads, kv_heads, group, page_shift, box_shift, n_pages;
  uint32_t group_inverse;   // 2^16 / group + 1
  int window, sinks;        // a token sees its last `window` positions and the first `sinks` (window 0: all)
  int apart;                // with a window: the prefix is a part of its own, for all sequences together
  int keep;                 // rows of the output that no sequence has stay as they were (called with a window, whatever that covers)
  int narrow[2], wide[2];   // which kernel takes a part (neither: it has no keys)
  int parts;                // parts that are computed apart (1, 2; above 1 their rows go to the join)
  int chained;              // the wide kernel's rows of kOwn run over the prefix first (no kPrefix part)
  int splits[2];            // thread blocks that share a row block's keys in the wide kernel
  uint64_t* rec;
  uint64_t call;
  uint64_t* tickets[2];
  int early, ahead;         // narrow kernel: thread blocks that start beside the wide one, places that a warp of them takes ahead
  float *o[2], *split_o[2], *warp_o[2], *block_o[2];
  float2 *ml[2], *split_ml[2], *block_ml[2];
  int ctas;                 // thread blocks of the narrow kernel
};

// With a window: the tiles of `keys` keys, the first at position `base`, that a
// run of tokens sees, whose first is at position `first` and whose last sees up
// to the last key.  They are tiles 0 .. a - 1 and those from a + skip on.
struct Line {
  int a, skip, tiles;
  __device__ int tile(int i) const volatile { return i < a ? i : i + skip; }
};
template <int K>
__device__ __forceinline__ Line line_of(const AttendParams& p, int keys, int base, int first) {
  Line l;
  const int all = (keys + K - 1) / K, low = first - p.window + 1 - base;
  l.a = (min(max(p.sinks - base, 0), keys) + K - 1) / K;
  l.skip = max(l.a, low >= keys ? all : max(low, 0) / K) - l.a;
  l.tiles = all - l.skip;
  return l;
}
// The position of a sequence's token at place `at` among its own (a token that
// has none stands behind the prefix).
__device__ __forceinline__ int position_of(const AttendParams& p, int at) { return p.b.prefix_len + max(at, -1); }

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

// Natural log-sum-exp of a row from its maximum and sum.  (Scores that are all
// NaN leave no maximum, but a sum that is NaN; -inf is a row that sees nothing.)
__device__ __forceinline__ float natural_lse(float top, float sum) {
  return top == -INFINITY && sum == sum ? top : (top + log2_approx(sum)) * 0.69314718056f;
}

// Of two bf16: which are infinite or NaN, as their 16 bits each.
__device__ __forceinline__ uint32_t not_finite(uint32_t w) {
  return ((w & 0x7F80u) == 0x7F80u ? 0xFFFFu : 0u) | ((w & 0x7F800000u) == 0x7F800000u ? 0xFFFF0000u : 0u);
}
// Is one of 8 bf16 infinite or NaN?  (An exponent of ones and 1 more carries into the sign's place.)
__device__ __forceinline__ bool some_not_finite(uint4 v) {
  auto up = [](uint32_t w) { return (w & 0x7F807F80u) + 0x00800080u; };
  return ((up(v.x) | up(v.y) | up(v.z) | up(v.w)) & 0x80008000u) != 0;
}
__device__ __forceinline__ uint4 ld_shared16(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];\n" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ void st_shared16(uint32_t a, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
  asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};\n" ::"r"(a), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}

// This lane's V columns of a row of D fp32 that another thread block wrote.
template <int D, int V>
__device__ __forceinline__ void load_row(const float* row, float (&v)[V]) {
  const float* at = row + V * (threadIdx.x & 31);
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
}
// A finished row: this lane's V columns.
template <int D, int V>
__device__ __forceinline__ void write_row(const AttendParams& p, int64_t row, const float (&acc)[V], float top, float sum) {
  const int lane = threadIdx.x & 31;
  const float k = sum > 0.f ? 1.f / sum : sum;   // (0 where nothing is seen; NaN stays)
  uint32_t* dst = reinterpret_cast<uint32_t*>(p.out + row * D + V * lane);
  if (V == 4) *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16x2(acc[0] * k, acc[1] * k), pack_bf16x2(acc[V - 2] * k, acc[V - 1] * k));
  else *dst = pack_bf16x2(acc[0] * k, acc[1] * k);
  if (p.lse && lane == 0) p.lse[row] = natural_lse(top, sum);
}

// The narrow kernel on `part`; late: behind this call's kernel on the prefix,
// beside which it may run.
int narrow_groups(const AttendParams& p, int part);           // of 8 query rows (1 to 4; 0 without keys)
int narrow_warps();                                           // per thread block
cudaError_t launch_narrow(const sdq_cache_s* c, const AttendParams& p, int part, bool late, cudaStream_t st);
// The wide kernel on `part`, and how many thread blocks share the keys of a
// row block (p.splits[part]); narrow: the narrow kernel runs beside it.
constexpr int kMaxWideSplits = 16;
constexpr double kNarrowStart = 4.0;   // us that the narrow kernel takes beyond its reading
int wide_splits(const sdq_cache_s* c, const AttendParams& p, int q_heads, int part, bool narrow);
double wide_time(const sdq_cache_s* c, const AttendParams& p, int q_heads, int part, int splits);   // us, estimated
int64_t wide_grid(const sdq_cache_s* c, const AttendParams& p, int part);   // thread blocks
cudaError_t launch_wide(const sdq_cache_s* c, const AttendParams& p, int part, cudaStream_t st);

}  // namespace sdq
