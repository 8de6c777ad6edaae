// One token per row of logits with temperature, top-k, top-p and min-p, from
// given random numbers (include/sdq.h).
//
// A cluster of up to 8 thread blocks keeps a row in its shared memory, so that
// HBM is read once however often the row is looked at:
//   1  load, largest logit.  For a top-k of k: the k / (blocks) largest of each
//      block's threads' own largest are as many logits, so that the least of
//      them over the blocks bounds the row's k-th from below.  Usually little
//      more than k lie above the bound: they are gathered as in 3, without 2
//   2  a histogram (count and mass) of the logits within 12 T of the largest,
//      and where top-p has no top-k ahead of it the mass of all; where a cut
//      lies further down, a histogram of the rest
//   3  top-k's bucket (top-p's where there is no top-k) from the joined
//      histogram.  Where no more than kCap logits lie in it and above, they are
//      gathered in one thread block, a thread each, which counts every one's
//      rank and the mass before it, cuts, and finds the token among what is
//      left (sorting 512 of them took 12000 cycles).  Otherwise
//   4  top-k, then top-p: the bucket is narrowed (by histograms of its parts,
//      at last by the logits' bits) until kCap or fewer are left, they are
//      gathered, and every one's rank and mass before it counted, which gives
//      the cut as a (logit, index) pair
//   5  mass of what is left in index order, and the token at u times it
// A pass looks at the largest of 4 neighbours first: few logits are near enough
// to the row's largest to need a weight.
// No sort, and no step depends on the order of its atomics: masses are whole
// numbers, weights in units of 2^-44 of the largest (a row of 2^19 weights
// fits 64 bits; a weight below half a unit, 2^-45, counts as 0), so every sum
// is exact.
// Masses are added as two 32-bit words, the carry from what the first add
// returns: 11 cycles a warp instruction against 27 to 250 for a 64-bit add in
// shared memory, which is a compare-and-swap loop.
// What bounds it: the instructions of the passes over many rows (a row is read
// once from HBM); for few rows the chain of passes and cluster barriers.  96 rows
// of 128255 fp32 with settings of all kinds: 66 to 80 us by the logits (two waves
// of clusters of 3); 32 of 50272 bf16: 17 to 48 likewise; one of 32000: 6.5.
#include <algorithm>

#include "common.cuh"

namespace sdq {

namespace {

constexpr int kThreads = 1024, kWarps = kThreads / 32;
constexpr int kBins = 128, kCap = 512;           // bins of a level; logits that are gathered, at most one per thread
constexpr int kMaxCluster = 8;
constexpr int kMaxVocab = 393216;            // (2^19 weights of 2^44 units fit 64 bits)
constexpr float kUnit = 17592186044416.f;        // 2^44
constexpr float kLeast = -31.2f;                 // exp(kLeast) 2^44 < 1/2

struct SampleParams {
  const void* logits;
  int64_t ld;
  const float *temperature, *top_p, *min_p, *u;
  const int32_t* top_k;
  int32_t* tokens;
  int vocab, chunk, cluster;
};

constexpr int kLevels = 2;

// A cut: kept are the logits above (key), and those equal to it up to index idx.
struct Cut {
  uint32_t key;
  int idx;
};

struct Histogram {            // of a block's logits
  uint32_t cnt[kBins], lo[kBins], hi[kBins];
};
struct Cumulative {           // of the row's: counts and masses up to and with a bin
  uint32_t cnt[kBins];
  unsigned long long mass[kBins];
};

struct alignas(16) Shared {   // (the logits behind it are read 4 at a time)
  Histogram own;
  Cumulative row[2];                     // level 0, the level below it that was last looked at
  uint32_t level_cnt[kLevels];           // of the levels looked at
  unsigned long long level_mass[kLevels];
  uint32_t list_key[kCap];               // gathered here
  int list_idx[kCap];
  uint32_t list_n;
  union {
    Cumulative sub;                      // of a narrowed bucket
    struct {
      // gathered in the cluster; order: the key above the index from the end,
      // so that a larger word comes first
      unsigned long long order[kCap], w[kCap];
      uint32_t rank[kCap];
    } all;
  };
  // partial sums of a step that several threads share
  uint32_t part_n[kThreads];
  unsigned long long part_m[kThreads];
  // posted for the cluster: written before a cluster barrier, read after it,
  // not written again before the next one
  float post_max;
  int post_first, post_cut;
  uint32_t post_cnt, post_ties, post_lo, post_hi;
  unsigned long long post_mass, post_kept;
  // results of block-wide steps
  float red_f[kWarps];
  uint32_t red_c[kWarps];
  unsigned long long red_u[kWarps], wsum[kWarps];
  uint32_t found_cnt, found_above_cnt, nkeep;
  unsigned long long found_above_mass, keep_mass;
  int found;
  Cut cut;
};

__device__ __forceinline__ uint32_t remote_u32(const void* p, int rank) {
  uint32_t r;
  asm volatile("ld.shared::cluster.u32 %0, [%1];\n" : "=r"(r) : "r"(cluster_addr(p, (uint32_t)rank)) : "memory");
  return r;
}
__device__ __forceinline__ unsigned long long remote_u64(const void* p, int rank) {
  unsigned long long r;
  asm volatile("ld.shared::cluster.u64 %0, [%1];\n" : "=l"(r) : "r"(cluster_addr(p, (uint32_t)rank)) : "memory");
  return r;
}
// A posted word of every thread block of the cluster, lane q's that of block q
// (a whole warp; lanes beyond the cluster: `none`).
__device__ __forceinline__ uint32_t posted(const uint32_t* p, int cluster, uint32_t none) {
  const int lane = threadIdx.x & 31;
  return lane < cluster ? remote_u32(p, lane) : none;
}
__device__ __forceinline__ unsigned long long posted(const unsigned long long* p, int cluster) {
  const int lane = threadIdx.x & 31;
  return lane < cluster ? remote_u64(p, lane) : 0ull;
}
__device__ __forceinline__ unsigned long long warp_sum(unsigned long long v) {
  for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
  return v;
}
// Monotone in the logit (no NaN): larger logits have larger keys; -0 as +0.
__device__ __forceinline__ uint32_t key_of(float z) {
  const uint32_t b = __float_as_uint(z + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t key) {
  return __uint_as_float(key & 0x80000000u ? key & 0x7FFFFFFFu : ~key);
}
// (z - max) / T by the rounded reciprocal of T, 0 for the largest also where it is infinite.
__device__ __forceinline__ float scaled(float z, float top, float inv_t) { return z == top ? 0.f : (z - top) * inv_t; }
__device__ __forceinline__ float weight_f(float x) { return expf(x); }
__device__ __forceinline__ unsigned long long weight(float x) {
  // (from 9 on below 2^32: a cheaper conversion to the same number)
  return x > -9.f ? __float2ull_rn(weight_f(x) * kUnit) : x > kLeast ? (unsigned long long)__float2uint_rn(weight_f(x) * kUnit) : 0ull;
}
// Where a logit of weight above 0 stands: its level (distances of 0 to 12 T,
// beyond), and its place there, 0 .. kBins 2^14 - 1 from the level's nearest on:
// the place's upper 7 bits are its bin, the next 7 its bin in a bin, and again.
constexpr int kPlaceBits = 14;
__device__ __forceinline__ float level_from(int l) { return l == 0 ? 0.f : 12.f; }
__device__ __forceinline__ float level_width(int l) { return l == 0 ? 12.f : 20.f; }
__device__ __forceinline__ int level_of(float x) { return x > -12.f ? 0 : 1; }
__device__ __forceinline__ uint32_t place_of(float x, int l) {
  return min((uint32_t)(kBins << kPlaceBits) - 1, (uint32_t)((-x - level_from(l)) * ((kBins << kPlaceBits) / level_width(l))));
}
__device__ __forceinline__ int bin_of(float x, int l) { return (int)(place_of(x, l) >> kPlaceBits); }
__device__ __forceinline__ void add_to(Histogram& h, int b, unsigned long long w) {
  atomicAdd(&h.cnt[b], 1u);
  const uint32_t lo = (uint32_t)w, old = atomicAdd(&h.lo[b], lo);
  const uint32_t hi = (uint32_t)(w >> 32) + (old + lo < old);
  if (hi) atomicAdd(&h.hi[b], hi);
}

__device__ __forceinline__ unsigned long long block_sum(Shared& s, unsigned long long v) {
  v = warp_sum(v);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) s.red_u[threadIdx.x >> 5] = v;
  __syncthreads();
  static_assert(kWarps == 32, "a lane each");
  return warp_sum(s.red_u[threadIdx.x & 31]);
}

__device__ __forceinline__ void clear_histogram(Histogram& h) {
  if (threadIdx.x < kBins) h.cnt[threadIdx.x] = h.lo[threadIdx.x] = h.hi[threadIdx.x] = 0;
}

// Cumulative counts and masses of the row's bins, from all blocks of the cluster.
__device__ __forceinline__ void join_histogram(Shared& s, Cumulative& to, int cluster) {
  static_assert(kThreads >= kMaxCluster * kBins, "a thread for each bin of each block");
  {
    const int q = threadIdx.x / kBins, b = threadIdx.x % kBins;
    uint32_t cnt = 0;
    unsigned long long mass = 0;
    if (q < cluster) {
      cnt = remote_u32(&s.own.cnt[b], q);
      const uint32_t lo = remote_u32(&s.own.lo[b], q), hi = remote_u32(&s.own.hi[b], q);
      mass = ((unsigned long long)hi << 32) + lo;
    }
    s.part_n[threadIdx.x] = cnt;
    s.part_m[threadIdx.x] = mass;
  }
  __syncthreads();
  uint32_t c = 0;
  unsigned long long m = 0;
  const bool mine = threadIdx.x < kBins;
  if (mine) {
#pragma unroll
    for (int q = 0; q < kMaxCluster; ++q) {
      c += s.part_n[q * kBins + threadIdx.x];
      m += s.part_m[q * kBins + threadIdx.x];
    }
  }
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int d = 1; d < 32; d <<= 1) {
    const uint32_t a = __shfl_up_sync(0xffffffffu, c, d);
    const unsigned long long b = __shfl_up_sync(0xffffffffu, m, d);
    if (lane >= d) {
      c += a;
      m += b;
    }
  }
  __syncthreads();
  if (lane == 31) {
    s.red_c[warp] = c;
    s.red_u[warp] = m;
  }
  __syncthreads();
  if (mine) {
    for (int w = 0; w < warp; ++w) {
      c += s.red_c[w];
      m += s.red_u[w];
    }
    to.cnt[threadIdx.x] = c;
    to.mass[threadIdx.x] = m;
  }
  __syncthreads();
}

// What a cut is looked for by: the first top_k, or those before which less
// than `mass` lies.
struct Goal {
  bool by_count;
  uint32_t count;
  unsigned long long mass;
};

// The first bin whose cumulative count or mass reaches the goal (found =
// kBins: none), what lies above it, and its own count.
__device__ __forceinline__ void pick(Shared& s, const Cumulative& h, const Goal& g, uint32_t above_cnt, unsigned long long above_mass) {
  auto reached = [&](int b) { return g.by_count ? above_cnt + h.cnt[b] >= g.count : above_mass + h.mass[b] >= g.mass; };
  const int b = threadIdx.x;
  if (b == 0) s.found = kBins;
  __syncthreads();
  if (b < kBins && reached(b) && (b == 0 || !reached(b - 1))) s.found = b;
  __syncthreads();
  if (b == 0) {
    const int f = s.found;
    const uint32_t c0 = f > 0 ? h.cnt[f - 1] : 0;
    s.found_above_cnt = above_cnt + c0;
    s.found_above_mass = above_mass + (f > 0 ? h.mass[f - 1] : 0);
    s.found_cnt = f < kBins ? h.cnt[f] - c0 : 0;
  }
  __syncthreads();
}

// 4 neighbouring logits, the address of the first a multiple of their size.
__device__ __forceinline__ float4 read4(const float* p) { return __ldg(reinterpret_cast<const float4*>(p)); }
__device__ __forceinline__ float4 read4(const uint16_t* p) {
  const uint2 r = __ldg(reinterpret_cast<const uint2*>(p));
  return make_float4(__uint_as_float(r.x << 16), __uint_as_float(r.x & 0xFFFF0000u), __uint_as_float(r.y << 16),
                     __uint_as_float(r.y & 0xFFFF0000u));
}
__device__ __forceinline__ float read1(const float* p) { return __ldg(p); }
__device__ __forceinline__ float read1(const uint16_t* p) { return __uint_as_float((uint32_t)__ldg(p) << 16); }
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;\n" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// This block's part of the row in shared memory, as its addresses in memory
// fall into groups of 4: logit i at z[i] = quads[(i + pad) / 4], -inf in the
// places before the first and behind the last.  NaN is kept: no comparison
// with it holds, and its weight is 0.
struct Row {
  const float4* quads;
  const float* z;
  int groups, pad;
  int lo, n;         // the first logit's index in the row, their number
  float top, t, inv_t;
  int cluster, rank;
};

// f(i, z, x, w) for each of this block's logits z of weight w above 0 whose
// distance from the largest is within a, b times T (both with room for
// rounding: f looks at x = (z - max) / T itself).
template <class F>
__device__ __forceinline__ void each_between(const Row& r, float a, float b, F f) {
  const float near = r.t * a * 0.9999f, far = r.t * b * 1.0001f;   // (NaN bounds pass everything)
#pragma unroll 2
  for (int q = threadIdx.x; q < r.groups; q += kThreads) {
    const float4 z4 = r.quads[q];
    if (r.top - fmaxf(max3(z4.x, z4.y, z4.z), z4.w) > far) continue;
    const float z[4] = {z4.x, z4.y, z4.z, z4.w};
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const float d = r.top - z[c];   // (NaN for the largest where it is infinite)
      if (d < near || d > far) continue;
      const float x = scaled(z[c], r.top, r.inv_t);   // (-inf or NaN, weight 0, for a logit of -inf)
      const unsigned long long w = weight(x);
      if (w) f(4 * q + c - r.pad, z[c], x, w);
    }
  }
}

// Level l's histogram into `to`, its totals into s.level_*.
__device__ __forceinline__ void look_at(Shared& s, const Row& r, int l, Cumulative& to) {
  cluster_sync();   // nobody reads the last histogram any more
  clear_histogram(s.own);
  __syncthreads();
  each_between(r, level_from(l), level_from(l) + level_width(l), [&](int, float, float x, unsigned long long w) {
    if (level_of(x) == l) add_to(s.own, bin_of(x, l), w);
  });
  cluster_sync();
  join_histogram(s, to, r.cluster);
  if (threadIdx.x == 0) {
    s.level_cnt[l] = to.cnt[kBins - 1];
    s.level_mass[l] = to.mass[kBins - 1];
  }
  __syncthreads();
}

// Where a goal's cut falls.
struct Place {
  int level;                     // -1: nothing is cut off (then all levels were looked at)
  int bin;
  uint32_t above_cnt, n;         // logits above the bucket, in it
  unsigned long long above_mass;
  float from, to;                // its range of distances, in T
};

// The bucket in which goal g's cut falls.  Every block of the cluster finds
// the same.  held: the level in s.row[1] (0: none).
__device__ __forceinline__ Place locate(Shared& s, const Row& r, const Goal& g, int* held) {
  Place at;
  int level = 0;
  uint32_t cnt = 0;
  unsigned long long mass = 0;
  __syncthreads();
  pick(s, s.row[0], g, 0, 0);
  while (s.found == kBins) {
    cnt += s.level_cnt[level];
    mass += s.level_mass[level];
    if (++level == kLevels) {
      at.level = -1;
      return at;
    }
    if (*held != level) look_at(s, r, level, s.row[1]);
    *held = level;
    __syncthreads();
    pick(s, s.row[1], g, cnt, mass);
  }
  at.level = level;
  at.bin = s.found;
  at.above_cnt = s.found_above_cnt;
  at.above_mass = s.found_above_mass;
  at.n = s.found_cnt;
  at.from = level_from(level) + s.found * (level_width(level) / kBins);
  at.to = at.from + level_width(level) / kBins;
  return at;
}

__device__ __forceinline__ unsigned long long order_of(uint32_t key, uint32_t idx) { return ((unsigned long long)key << 32) | (uint32_t)~idx; }
__device__ __forceinline__ uint32_t key_in(unsigned long long order) { return (uint32_t)(order >> 32); }
__device__ __forceinline__ int idx_in(unsigned long long order) { return (int)~(uint32_t)order; }
// Rank of the gathered logit that is this thread's (order; thread c has logit
// c), and the mass before it: all threads of the block, as many to a logit as
// there are.
__device__ __forceinline__ void rank_in(Shared& s, uint32_t have, uint32_t* rank, unsigned long long* before) {
  const uint32_t width = (have + 31) & ~31u, parts = kThreads / width;   // (have >= 1)
  const uint32_t c = threadIdx.x % width, part = threadIdx.x / width;
  uint32_t n = 0;
  unsigned long long m = 0;
  if (part < parts && c < have) {
    const unsigned long long order = s.all.order[c];
    const uint32_t j1 = (part + 1) * have / parts;
#pragma unroll 8
    for (uint32_t j = part * have / parts; j < j1; ++j) {
      const bool better = s.all.order[j] > order;
      const unsigned long long w = s.all.w[j];
      n += better;
      m += better ? w : 0ull;
    }
  }
  s.part_n[threadIdx.x] = n;
  s.part_m[threadIdx.x] = m;
  __syncthreads();
  *rank = 0;
  *before = 0;
  if (threadIdx.x < have)
    for (uint32_t q = 0; q < parts; ++q) {
      *rank += s.part_n[q * width + threadIdx.x];
      *before += s.part_m[q * width + threadIdx.x];
    }
  __syncthreads();
}

// This block's share of a gathered list: those of the logits between two
// distances that `take` (z, x) takes.
template <class Take>
__device__ __forceinline__ void gather(Shared& s, const Row& r, float from, float to, Take take) {
  if (threadIdx.x == 0) s.list_n = 0;
  __syncthreads();
  each_between(r, from, to, [&](int i, float z, float x, unsigned long long) {
    if (!take(z, x)) return;
    const uint32_t at = atomicAdd(&s.list_n, 1u);
    if (at < kCap) {   // (always: they were counted)
      s.list_key[at] = key_of(z);
      s.list_idx[at] = r.lo + i;
    }
  });
}
// The cluster's lists into s.all (after a cluster barrier); their number.
__device__ __forceinline__ uint32_t collect(Shared& s, const Row& r) {
  const uint32_t mine = posted(&s.list_n, r.cluster, 0u);
  uint32_t upto = mine;
  for (int d = 1; d < kMaxCluster; d <<= 1) {
    const uint32_t o = __shfl_up_sync(0xffffffffu, upto, d);
    if ((int)(threadIdx.x & 31) >= d) upto += o;
  }
  const uint32_t have = min((uint32_t)kCap, __shfl_sync(0xffffffffu, upto, kMaxCluster - 1));
  const int warp = threadIdx.x >> 5, q = warp % r.cluster, per = kWarps / r.cluster;   // warps to a block's list
  const uint32_t m = __shfl_sync(0xffffffffu, mine, q), at = __shfl_sync(0xffffffffu, upto, q) - m;
  if (warp < per * r.cluster)
    for (uint32_t j = 32 * (warp / r.cluster) + (threadIdx.x & 31); j < m && at + j < have; j += 32 * per) {
      const uint32_t k = remote_u32(&s.list_key[j], q);
      s.all.order[at + j] = order_of(k, remote_u32(&s.list_idx[j], q));
      s.all.w[at + j] = weight(scaled(logit_of(k), r.top, r.inv_t));
    }
  __syncthreads();
  return have;
}

// The cut of goal g, which falls at `at`: s.cut, and the mass that is kept in
// s.keep_mass.  Every block of the cluster finds the same.  use: 0 for a
// kernel's first call, 1 for its second.
__device__ __forceinline__ void resolve(Shared& s, const Row& r, const Goal& g, const Place& at0, int use) {
  const int level = at0.level;
  uint32_t above_cnt = at0.above_cnt, n = at0.n;
  unsigned long long above_mass = at0.above_mass;
  const float from = at0.from, to = at0.to;
  uint32_t prefix = (uint32_t)at0.bin;
  int shift = kPlaceBits;   // the bucket: places of this prefix above `shift` bits
  auto inside = [&](float x) { return level_of(x) == level && place_of(x, level) >> shift == prefix; };
#pragma unroll 1
  while (n > kCap && shift > 0) {
    cluster_sync();   // nobody reads the last histogram any more
    clear_histogram(s.own);
    __syncthreads();
    each_between(r, from, to, [&](int, float, float x, unsigned long long w) {
      if (inside(x)) add_to(s.own, place_of(x, level) >> (shift - 7) & (kBins - 1), w);
    });
    cluster_sync();
    join_histogram(s, s.sub, r.cluster);
    pick(s, s.sub, g, above_cnt, above_mass);
    n = s.found_cnt;
    above_cnt = s.found_above_cnt;
    above_mass = s.found_above_mass;
    prefix = prefix << 7 | (uint32_t)s.found;
    shift -= 7;
    __syncthreads();
  }
  uint32_t klo = 0, khi = 0xFFFFFFFFu;
  const bool by_key = n > kCap;
  if (by_key) {
    // the bucket's range of keys, then bins of that range until few are left or one value
    uint32_t lo = 0xFFFFFFFFu, hi = 0;
    each_between(r, from, to, [&](int, float z, float x, unsigned long long) {
      if (!inside(x)) return;
      lo = min(lo, key_of(z));
      hi = max(hi, key_of(z));
    });
    lo = __reduce_min_sync(0xffffffffu, lo);
    hi = __reduce_max_sync(0xffffffffu, hi);
    if (threadIdx.x == 0) {
      s.post_lo = 0xFFFFFFFFu;
      s.post_hi = 0;
    }
    __syncthreads();
    if ((threadIdx.x & 31) == 0) {
      atomicMin(&s.post_lo, lo);
      atomicMax(&s.post_hi, hi);
    }
    cluster_sync();
    klo = __reduce_min_sync(0xffffffffu, posted(&s.post_lo, r.cluster, 0xFFFFFFFFu));
    khi = __reduce_max_sync(0xffffffffu, posted(&s.post_hi, r.cluster, 0u));
    while (n > kCap && klo < khi) {
      static_assert(kBins == 128, "7 bits of the range");
      const int bits = max(0, 32 - __clz(khi - klo) - 7);
      cluster_sync();   // nobody reads the last histogram any more
      clear_histogram(s.own);
      __syncthreads();
      each_between(r, from, to, [&](int, float z, float, unsigned long long w) {
        const uint32_t k = key_of(z);
        if (k >= klo && k <= khi) add_to(s.own, (khi - k) >> bits, w);
      });
      cluster_sync();
      join_histogram(s, s.sub, r.cluster);
      pick(s, s.sub, g, above_cnt, above_mass);
      if (s.found >= kBins) break;   // (not reached: the goal lies in this range)
      n = s.found_cnt;
      above_cnt = s.found_above_cnt;
      above_mass = s.found_above_mass;
      khi -= (uint32_t)s.found << bits;
      klo = max(klo, khi - ((1u << bits) - 1));   // (keys of finite logits are at least 2^23)
    }
    cluster_sync();   // the same, ahead of the next call's; and of the posted range
  }
  if (n > kCap) {
    // equal logits: as many of them as the goal takes, by index
    const unsigned long long w = weight(scaled(logit_of(khi), r.top, r.inv_t));
    const uint32_t take = g.by_count ? g.count - above_cnt : (uint32_t)((g.mass - above_mass + w - 1) / w);
    uint32_t ties = 0;
    for (int i = threadIdx.x; i < r.n; i += kThreads) ties += key_of(r.z[i]) == khi;
    ties = (uint32_t)block_sum(s, ties);
    if (threadIdx.x == 0) s.post_ties = ties;
    cluster_sync();
    uint32_t before = 0;
    int owner = 0;
    for (; owner < r.cluster - 1; ++owner) {
      const uint32_t t = remote_u32(&s.post_ties, owner);
      if (before + t >= take) break;
      before += t;
    }
    if (owner == r.rank && threadIdx.x < 32) {
      uint32_t seen = before;
      int at = r.lo;
      for (int i0 = 0; i0 < r.n; i0 += 32) {
        const int i = i0 + (int)threadIdx.x;
        uint32_t hit = __ballot_sync(0xffffffffu, i < r.n && key_of(r.z[i]) == khi);
        if (seen + __popc(hit) >= take) {
          for (uint32_t k = seen + 1; k < take; ++k) hit &= hit - 1;   // drop those before the last one taken
          at = r.lo + i0 + __ffs(hit) - 1;
          break;
        }
        seen += __popc(hit);
      }
      if (threadIdx.x == 0) s.post_cut = at;
    }
    cluster_sync();
    const int at = (int)remote_u32(&s.post_cut, owner);
    if (threadIdx.x == 0) {
      s.cut = {khi, at};
      s.keep_mass = above_mass + w * take;
    }
    cluster_sync();   // what was posted may be written again
    return;
  }
  // the bucket's members from the cluster
  if (use) cluster_sync();   // nobody reads the first call's list any more
  if (threadIdx.x == 0) {
    s.nkeep = 0;
    s.keep_mass = above_mass;
  }
  gather(s, r, from, to, [&](float z, float x) {
    const uint32_t k = key_of(z);
    return by_key ? k >= klo && k <= khi : inside(x);
  });
  cluster_sync();
  const uint32_t have = collect(s, r);
  const uint32_t c = threadIdx.x;   // (have <= kCap, a thread each)
  uint32_t rank;
  unsigned long long before;
  rank_in(s, max(have, 1u), &rank, &before);
  if (c < have) {
    s.all.rank[c] = rank;
    if (g.by_count ? above_cnt + rank < g.count : above_mass + before < g.mass) {
      atomicMax(&s.nkeep, rank + 1);
      atomicAdd(&s.keep_mass, s.all.w[c]);
    }
  }
  __syncthreads();
  if (c < have && s.all.rank[c] + 1 == s.nkeep) s.cut = {key_in(s.all.order[c]), idx_in(s.all.order[c])};
  __syncthreads();
}

// The n-th largest of the threads' keys (n <= kThreads), 8 bits at a time.
__device__ __forceinline__ uint32_t nth_largest(Shared& s, uint32_t key, uint32_t n) {
  uint32_t prefix = 0;
#pragma unroll 1
  for (int shift = 24; shift >= 0; shift -= 8) {
    __syncthreads();
    if (threadIdx.x < 256) s.part_n[threadIdx.x] = 0;
    __syncthreads();
    if (shift == 24 || key >> (shift + 8) == prefix) atomicAdd(&s.part_n[key >> shift & 255u], 1u);
    __syncthreads();
    if (threadIdx.x < 32) {
      // lane l: bins 255 - 8 l and the 7 below
      const int lane = threadIdx.x, first = 255 - 8 * lane;
      uint32_t own = 0;
      for (int b = 0; b < 8; ++b) own += s.part_n[first - b];
      uint32_t upto = own;
      for (int d = 1; d < 32; d <<= 1) {
        const uint32_t o = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= d) upto += o;
      }
      if (upto >= n && upto - own < n) {   // (one lane)
        uint32_t left = n - (upto - own);
        int b = first;
        while (s.part_n[b] < left) left -= s.part_n[b--];
        s.found = b;
        s.found_cnt = left;
      }
    }
    __syncthreads();
    prefix = prefix << 8 | (uint32_t)s.found;
    n = s.found_cnt;
  }
  return prefix;
}

// f times a mass, f in [0, 1), rounded down, and whether that left a rest.
// (In whole numbers: 64-bit floating point is slow here, 3000 cycles for a
// thread block's two products.)
__device__ __forceinline__ unsigned long long share_of(float f, unsigned long long mass, bool* rest) {
  const uint32_t bits = __float_as_uint(f), e = bits >> 23;
  const uint32_t m = (bits & 0x7FFFFFu) | (e ? 0x800000u : 0u);
  const int k = 150 - (int)max(e, 1u);   // f = m 2^-k, k >= 24
  const unsigned long long hi = __umul64hi(mass, m), lo = mass * m;
  if (k < 64) {
    *rest = (lo & ((1ull << k) - 1)) != 0;
    return (hi << (64 - k)) | (lo >> k);
  }
  *rest = lo != 0 || hi != 0;
  return k < 128 ? hi >> (k - 64) : 0ull;   // (hi < 2^24: a share of 0 or 1 has a rest wherever it is below it)
}
// What a share u of a mass comes to; the token lies where the running sum exceeds it.
__device__ __forceinline__ unsigned long long target_of(float u, unsigned long long total) {
  bool rest;
  if (!(u > 0.f)) return 0;
  return u < 1.f ? min(share_of(u, total, &rest), total - 1) : total - 1;
}
// Mass before which a logit lies that top-p (below 1) keeps: below top_p of
// `mass`, that is, below that rounded up (the first one always).
__device__ __forceinline__ unsigned long long mass_goal(float top_p, unsigned long long mass) {
  bool rest = false;
  const unsigned long long v = top_p > 0.f ? share_of(top_p, mass, &rest) : 0ull;
  return max(1ull, v + rest);
}

// The token of a row whose first `have` logits are in s.all (one thread block;
// everything that is cut off among them or below).  top_k 0: none; mass: of
// all, for top_p alone.
__device__ __forceinline__ int choose(Shared& s, const Row& r, uint32_t have, int top_k, bool cut_p, float top_p, float least, float u,
                      unsigned long long mass) {
  const uint32_t c = threadIdx.x;
  const unsigned long long order = c < have ? s.all.order[c] : 0;
  unsigned long long w = c < have ? s.all.w[c] : 0, before = 0;
  uint32_t rank = 0;
  rank_in(s, max(have, 1u), &rank, &before);
  if (top_k > 0) {
    if (rank >= (uint32_t)top_k) w = 0;
    mass = block_sum(s, w);
  }
  if (cut_p && c < have && before >= mass_goal(top_p, mass)) w = 0;
  if (weight_f(scaled(logit_of(key_in(order)), r.top, r.inv_t)) < least) w = 0;
  const unsigned long long total = block_sum(s, w), target = target_of(u, total);
  if (c < have) s.all.w[c] = w;
  if (c == 0) s.found = -1;
  __syncthreads();
  if (w) {
    unsigned long long lower = 0;
#pragma unroll 8
    for (uint32_t j = 0; j < have; ++j) {
      const bool first = (uint32_t)s.all.order[j] > (uint32_t)order;   // a smaller index
      const unsigned long long v = s.all.w[j];
      lower += first ? v : 0ull;
    }
    if (lower <= target && target < lower + w) s.found = idx_in(order);   // (one thread)
  }
  __syncthreads();
  return s.found;
}

template <class T>
__global__ void __launch_bounds__(kThreads, 1) sample_kernel(const SampleParams p) {
  extern __shared__ __align__(16) uint8_t smem_raw[];
  Shared& s = *reinterpret_cast<Shared*>(smem_raw);
  float4* quads = reinterpret_cast<float4*>(smem_raw + sizeof(Shared));
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, row = blockIdx.y;
  pdl_wait();
  pdl_launch_dependents();
  Row r;
  r.rank = (int)cluster_rank();
  r.cluster = p.cluster;
  r.lo = r.rank * p.chunk;
  r.n = max(0, min(p.chunk, p.vocab - r.lo));
  r.t = p.temperature ? __ldg(p.temperature + row) : 1.f;
  r.inv_t = __frcp_rn(r.t);
  const int top_k = p.top_k ? __ldg(p.top_k + row) : 0;
  const float top_p = p.top_p ? __ldg(p.top_p + row) : 1.f, min_p = p.min_p ? __ldg(p.min_p + row) : 0.f;
  const float u = __ldg(p.u + row), least = min_p > 0.f ? min_p : 0.f;
  // 1: the row, its largest logit
  const T* src = static_cast<const T*>(p.logits) + (int64_t)row * p.ld + r.lo;
  r.pad = (int)((reinterpret_cast<uintptr_t>(src) / sizeof(T)) & 3);
  r.groups = r.n > 0 ? (r.pad + r.n + 3) / 4 : 0;
  r.quads = quads;
  r.z = reinterpret_cast<const float*>(quads) + r.pad;
  float top = -INFINITY;
  constexpr int kBatch = 4;   // loads under way at once
  for (int q0 = tid; q0 < r.groups; q0 += kBatch * kThreads) {
    float4 v[kBatch];
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const int q = q0 + j * kThreads, i = 4 * q - r.pad;
      if (i >= 0 && i + 4 <= r.n) {
        v[j] = read4(src + i);
      } else {
        v[j] = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
        if (i >= 0 && i < r.n) v[j].x = read1(src + i);
        if (i + 1 >= 0 && i + 1 < r.n) v[j].y = read1(src + i + 1);
        if (i + 2 >= 0 && i + 2 < r.n) v[j].z = read1(src + i + 2);
        if (i + 3 >= 0 && i + 3 < r.n) v[j].w = read1(src + i + 3);
      }
    }
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      if (q0 + j * kThreads < r.groups) quads[q0 + j * kThreads] = v[j];
      top = fmaxf(top, fmaxf(max3(v[j].x, v[j].y, v[j].z), v[j].w));
    }
  }
  const bool cut_k = top_k > 0 && top_k < p.vocab, cut_p = top_p < 1.f;
  const bool bound = cut_k && top_k <= kCap / 2;
  if (bound) {
    const uint32_t key = nth_largest(s, key_of(top), ((uint32_t)top_k + p.cluster - 1) / p.cluster);   // of a block's threads' largest
    if (tid == 0) s.post_lo = key;
  }
  for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
  if (lane == 0) s.red_f[warp] = top;
  clear_histogram(s.own);
  __syncthreads();
  for (int w = 0; w < kWarps; ++w) top = fmaxf(top, s.red_f[w]);
  if (tid == 0) s.post_max = top;
  cluster_sync();
  top = __uint_as_float(posted(reinterpret_cast<const uint32_t*>(&s.post_max), r.cluster, 0xFF800000u));
  for (int d = 4; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
  top = __shfl_sync(0xffffffffu, top, 0);
  r.top = top;
  if (top == -INFINITY || !(r.t > 0.f) || min_p > 1.f) {
    // nothing to choose from, or the first of the largest logits alone
    if (tid == 0) s.post_first = 0x7FFFFFFF;
    __syncthreads();
    if (top > -INFINITY) {
      int first = 0x7FFFFFFF;
      for (int q = tid; q < r.groups; q += kThreads) {
        const float4 v = quads[q];
        const int at = v.x == top ? 0 : v.y == top ? 1 : v.z == top ? 2 : v.w == top ? 3 : 4;
        if (at < 4) first = min(first, r.lo + 4 * q + at - r.pad);
      }
      first = __reduce_min_sync(0xffffffffu, first);
      if (lane == 0) atomicMin(&s.post_first, first);
    }
    cluster_sync();
    if (r.rank == 0 && warp == 0) {
      const uint32_t first = __reduce_min_sync(0xffffffffu, posted(reinterpret_cast<const uint32_t*>(&s.post_first), r.cluster, 0x7FFFFFFFu));
      if (tid == 0) p.tokens[row] = first == 0x7FFFFFFFu ? -1 : (int)first;
    }
    cluster_sync();   // no block ends while its memory is being read
    return;
  }
  if (bound) {
    // (-inf: too few logits for a bound; all are listed then, if they are few enough)
    const float least_z = logit_of(__reduce_min_sync(0xffffffffu, posted(&s.post_lo, r.cluster, 0xFFFFFFFFu)));
    if (tid == 0) s.list_n = 0;
    __syncthreads();
    for (int q = tid; q < r.groups; q += kThreads) {
      const float4 z4 = quads[q];
      const float z[4] = {z4.x, z4.y, z4.z, z4.w};
      if (!(fmaxf(max3(z4.x, z4.y, z4.z), z4.w) >= least_z)) continue;
#pragma unroll
      for (int c = 0; c < 4; ++c)
        if (z[c] >= least_z && z[c] > -INFINITY) {
          const uint32_t at = atomicAdd(&s.list_n, 1u);
          if (at < kCap) {
            s.list_key[at] = key_of(z[c]);
            s.list_idx[at] = r.lo + 4 * q + c - r.pad;
          }
        }
    }
    cluster_sync();
    if (warp_sum(posted(&s.list_n, r.cluster, 0u)) <= kCap) {
      uint32_t have = 0;
      if (r.rank == 0) have = collect(s, r);
      cluster_sync();   // no block ends while its memory is being read
      if (r.rank != 0) return;
      const int token = choose(s, r, have, top_k, cut_p, top_p, least, u, 0);
      if (tid == 0) p.tokens[row] = token;
      return;
    }
    cluster_sync();   // nobody reads what was posted any more
  }
  // 2: the histogram; where top-p has no top-k ahead of it, the mass of all
  s.cut = {0, 0x7FFFFFFF};   // everything
  if (cut_k || cut_p) {
    unsigned long long mass = 0;
    if (cut_k) {
      each_between(r, 0.f, level_width(0), [&](int, float, float x, unsigned long long w) {
        if (level_of(x) == 0) add_to(s.own, bin_of(x, 0), w);
      });
    } else {
      // (as each_between; groups beyond the level have weights below 2^32 units and take no part in the histogram)
      const float far = r.t * level_width(0) * 1.0001f;
#pragma unroll 2
      for (int q = tid; q < r.groups; q += kThreads) {
        const float4 z4 = quads[q];
        const float z[4] = {z4.x, z4.y, z4.z, z4.w};
        if (r.top - fmaxf(max3(z4.x, z4.y, z4.z), z4.w) > far) {
          uint32_t w[4];
#pragma unroll
          for (int c = 0; c < 4; ++c) w[c] = __float2uint_rn(weight_f((z[c] - r.top) * r.inv_t) * kUnit);   // (0 for NaN)
          mass += (unsigned long long)w[0] + w[1] + ((unsigned long long)w[2] + w[3]);
        } else {
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const float x = scaled(z[c], r.top, r.inv_t);
            const unsigned long long w = weight(x);
            mass += w;
            if (w && level_of(x) == 0) add_to(s.own, bin_of(x, 0), w);
          }
        }
      }
      mass = block_sum(s, mass);
      if (tid == 0) s.post_mass = mass;
    }
    cluster_sync();
    join_histogram(s, s.row[0], r.cluster);
    if (tid == 0) {
      s.level_cnt[0] = s.row[0].cnt[kBins - 1];
      s.level_mass[0] = s.row[0].mass[kBins - 1];
    }
    // 3 and 4: the cuts' buckets, top-k's first.  (A loop, so that the code of a cut is there once.)
    int held = 0;
    bool by_k = cut_k;   // top_k cuts something off
    if (!cut_k) mass = warp_sum(posted(&s.post_mass, r.cluster));
#pragma unroll 1
    for (int step = cut_k ? 0 : 1; step < 2; ++step) {
      if (step == 1 && !cut_p) break;
      const Goal g = step == 0 ? Goal{true, (uint32_t)top_k, 0} : Goal{false, 0, mass_goal(top_p, mass)};
      const Place at = locate(s, r, g, &held);
      if (at.level < 0) {   // (fewer than top_k)
        by_k = false;
        mass = 0;
        for (int l = 0; l < kLevels; ++l) mass += s.level_mass[l];
        continue;
      }
      if ((step == 0 || !by_k) && at.above_cnt + at.n <= kCap) {
        gather(s, r, 0.f, at.to, [&](float, float x) {
          const int l = level_of(x);
          return l < at.level || (l == at.level && bin_of(x, l) <= at.bin);
        });
        cluster_sync();
        uint32_t have = 0;
        if (r.rank == 0) have = collect(s, r);
        cluster_sync();   // no block ends while its memory is being read
        if (r.rank != 0) return;
        const int token = choose(s, r, have, by_k ? top_k : 0, cut_p, top_p, least, u, mass);
        if (tid == 0) p.tokens[row] = token;
        return;
      }
      resolve(s, r, g, at, step);
      mass = s.keep_mass;
    }
  }
  __syncthreads();
  const Cut cut = s.cut;
  const float zcut = logit_of(cut.key), furthest = r.t * fminf(least > 0.f ? -logf(least) : 32.f, 32.f) * 1.0001f;
  auto kept = [&](int i, float zi) -> unsigned long long {
    if (top - zi > furthest || zi < zcut) return 0;   // (either may be NaN: then x decides)
    const uint32_t k = key_of(zi);
    if (k < cut.key || (k == cut.key && r.lo + i > cut.idx)) return 0;
    const float x = scaled(zi, top, r.inv_t);
    return weight_f(x) >= least ? weight(x) : 0ull;
  };
  // 5: mass of what is kept, by index: a warp's segment (a lane 4 neighbours), the blocks before this one
  const int seg = (r.groups + kThreads - 1) / kThreads * 32, q0 = warp * seg, q1 = min(r.groups, q0 + seg);
  unsigned long long sum = 0;
#pragma unroll 2
  for (int q = q0 + lane; q < q1; q += 32) {
    const float4 v = quads[q];
    const float most = fmaxf(max3(v.x, v.y, v.z), v.w);
    if (top - most > furthest || most < zcut) continue;
    const int i = 4 * q - r.pad;
    sum += kept(i, v.x) + kept(i + 1, v.y) + kept(i + 2, v.z) + kept(i + 3, v.w);
  }
  for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  if (lane == 0) s.wsum[warp] = sum;
  __syncthreads();
  if (tid == 0) {
    unsigned long long all = 0;
    for (int w = 0; w < kWarps; ++w) all += s.wsum[w];
    s.post_kept = all;
  }
  cluster_sync();
  const unsigned long long kept_of = posted(&s.post_kept, r.cluster), total = warp_sum(kept_of);
  unsigned long long before = warp_sum(lane < r.rank ? kept_of : 0ull);
  // the first kept index whose running sum exceeds u times the mass
  const unsigned long long target = target_of(u, total);
  for (int w = 0; w < warp; ++w) before += s.wsum[w];
  if (before <= target && target < before + s.wsum[warp]) {   // (one warp of the cluster)
    for (int q = q0; q < q1; q += 32) {
      unsigned long long w[4] = {0, 0, 0, 0};
      const int i = 4 * (q + lane) - r.pad;
      if (q + lane < q1) {
        const float4 v = quads[q + lane];
        w[0] = kept(i, v.x);
        w[1] = kept(i + 1, v.y);
        w[2] = kept(i + 2, v.z);
        w[3] = kept(i + 3, v.w);
      }
      unsigned long long c = w[0] + w[1] + w[2] + w[3], own = c;
      for (int d = 1; d < 32; d <<= 1) {
        const unsigned long long o = __shfl_up_sync(0xffffffffu, c, d);
        if (lane >= d) c += o;
      }
      const uint32_t past = __ballot_sync(0xffffffffu, before + c > target);
      if (past) {
        if (lane == __ffs(past) - 1) {
          unsigned long long upto = before + c - own;
          int at = 0;
          while (at < 3 && (upto += w[at]) <= target) ++at;
          p.tokens[row] = r.lo + i + at;
        }
        break;
      }
      before += __shfl_sync(0xffffffffu, c, 31);
    }
  }
  cluster_sync();   // no block ends while its memory is being read
}

static_assert(sizeof(Shared) % 16 == 0, "the logits behind it are read 4 at a time");
constexpr int kMaxChunk = (227 * 1024 - (int)sizeof(Shared)) / 4 / 32 * 32 - 32;   // logits of a thread block

template <class T>
cudaError_t launch_sample(const SampleParams& p, int rows, int device, cudaStream_t st) {
  static std::atomic<int> smem_set[64];
  const cudaError_t e = smem_limit_once(sample_kernel<T>, (int)sizeof(Shared) + 4 * kMaxChunk + 32, device, smem_set);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)p.cluster, (unsigned)rows);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = sizeof(Shared) + 4 * (size_t)p.chunk + 32;   // (up to 3 places before and behind)
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)p.cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, sample_kernel<T>, p);
}

}  // namespace

}  // namespace sdq

using namespace sdq;

extern "C" int sdq_sample(const void* logits, int32_t type, int32_t rows, int32_t vocab, int64_t ld, const float* u,
                          const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p,
                          int32_t* tokens, void* stream) {
  if (!logits || !u || !tokens || (type != SDQ_F32 && type != SDQ_BF16)) return SDQ_ERR_INVALID_ARG;
  if (rows < 1 || rows > 65535 || vocab < 1 || vocab > kMaxVocab || ld < vocab) return SDQ_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(logits) % (type == SDQ_F32 ? 4 : 2)) return SDQ_ERR_INVALID_ARG;
  int dev = -1, major = 0, minor = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&minor, cudaDevAttrComputeCapabilityMinor, dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return SDQ_ERR_CUDA;
  if (major != 10 || minor != 3) return SDQ_ERR_UNSUPPORTED;
  SampleParams p;
  p.logits = logits; p.ld = ld;
  p.temperature = temperature; p.top_k = top_k; p.top_p = top_p; p.min_p = min_p; p.u = u;
  p.tokens = tokens;
  p.vocab = vocab;
  // Thread blocks per row: the least time over waves of one to an SM, of which
  // each takes about 8 us in barriers and joins and 0.4 us per 1000 logits.
  double best = 0;
  for (int c = 1; c <= kMaxCluster; ++c) {
    const int chunk = ((vocab + c - 1) / c + 31) / 32 * 32;
    const double t = (double)(((int64_t)rows * c + sms - 1) / sms) * (8.0 + 0.4e-3 * chunk);
    if (chunk > kMaxChunk || (best > 0 && t > 0.97 * best)) continue;
    best = t;
    p.cluster = c;
    p.chunk = chunk;
  }
  static_assert((kMaxVocab + kMaxCluster - 1) / kMaxCluster <= kMaxChunk, "a row fits in the cluster's shared memory");
  const cudaError_t e = type == SDQ_F32 ? launch_sample<float>(p, rows, dev, (cudaStream_t)stream)
                                        : launch_sample<uint16_t>(p, rows, dev, (cudaStream_t)stream);
  return e == cudaSuccess ? SDQ_OK : SDQ_ERR_CUDA;
}
