// One token per row of logits with temperature, top-k, top-p and min-p, from
// given random numbers (include/sdq.h).
//
// A cluster of up to 8 thread blocks keeps a row in its shared memory, so that
// HBM is read once however often the row is looked at:
//   1  load, largest logit
//   2  weights, their sum, and a histogram (count and mass) of the logits
//      within 16 T of the largest, in steps of T / 32
//   3  top-k, then top-p: the bucket in which the cut falls, from the joined
//      histogram; its members are gathered and every one's rank and mass
//      before it counted, which gives the cut as a (logit, index) pair.  A
//      bucket of more than kCap members is narrowed by its logits' bits first
//   4  mass of what is left in index order, and the token at u times it
// No sort, and no step depends on the order of its atomics: masses are whole
// numbers, weights in units of 2^-44 of the largest (a row of 2^19 weights
// fits 64 bits; a weight below half a unit, 2^-45, counts as 0), so every sum
// is exact.
// What bounds it: HBM for many rows; for few the chain of passes and cluster
// barriers.
#include <algorithm>

#include "common.cuh"

namespace sdq {

namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kBins = kThreads, kCap = 512;     // a bin per thread
constexpr int kMaxCluster = 8;
constexpr int kMaxVocab = kMaxCluster * 49152;
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

// A cut: kept are the logits above (key), and those equal to it up to index idx.
struct Cut {
  uint32_t key;
  int idx;
};

struct Histogram {
  uint32_t cnt[kBins];
  unsigned long long mass[kBins];
};

struct Shared {
  Histogram own;                         // of this block's logits
  Histogram row;                         // of the row: counts and masses up to and with a bin
  uint32_t list_key[2][kCap];            // gathered here, for the first and the second cut
  int list_idx[2][kCap];
  uint32_t list_n[2];
  union {
    Histogram sub;                       // of a narrowed bucket, as `row`
    struct {
      uint32_t key[kCap], rank[kCap];    // gathered in the cluster
      int idx[kCap];
      unsigned long long w[kCap];
    } all;
  };
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
// Monotone in the logit (no NaN): larger logits have larger keys; -0 as +0.
__device__ __forceinline__ uint32_t key_of(float z) {
  const uint32_t b = __float_as_uint(z + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t key) {
  return __uint_as_float(key & 0x80000000u ? key & 0x7FFFFFFFu : ~key);
}
// (z - max) / T, 0 for the largest also where it is infinite.
__device__ __forceinline__ float scaled(float z, float top, float t) { return z == top ? 0.f : __fdiv_rn(z - top, t); }
__device__ __forceinline__ float weight_f(float x) { return expf(x); }
__device__ __forceinline__ unsigned long long weight(float x) {
  return x > kLeast ? __float2ull_rn(weight_f(x) * kUnit) : 0ull;
}

__device__ __forceinline__ unsigned long long block_sum(Shared& s, unsigned long long v) {
  for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) s.red_u[threadIdx.x >> 5] = v;
  __syncthreads();
  v = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) v += s.red_u[w];
  return v;
}

__device__ __forceinline__ void clear_histogram(Histogram& h) {
  h.cnt[threadIdx.x] = 0;
  h.mass[threadIdx.x] = 0;
}

// Cumulative counts and masses of the row's bins, from all blocks of the cluster.
__device__ void join_histogram(Shared& s, Histogram& to, int cluster) {
  uint32_t c = 0;
  unsigned long long m = 0;
  for (int r = 0; r < cluster; ++r) {
    c += remote_u32(&s.own.cnt[threadIdx.x], r);
    m += remote_u64(&s.own.mass[threadIdx.x], r);
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
  for (int w = 0; w < warp; ++w) {
    c += s.red_c[w];
    m += s.red_u[w];
  }
  to.cnt[threadIdx.x] = c;
  to.mass[threadIdx.x] = m;
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
__device__ void pick(Shared& s, const Histogram& h, const Goal& g, uint32_t above_cnt, unsigned long long above_mass) {
  auto reached = [&](int b) { return g.by_count ? above_cnt + h.cnt[b] >= g.count : above_mass + h.mass[b] >= g.mass; };
  const int b = threadIdx.x;
  if (b == 0) s.found = kBins;
  __syncthreads();
  if (reached(b) && (b == 0 || !reached(b - 1))) s.found = b;
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

struct Row {
  const float* z;    // this block's logits (shared memory)
  int lo, n;         // its first index, its count
  float top, t;
  int cluster, rank;
  __device__ float x(int i) const { return scaled(z[i], top, t); }   // (-inf or NaN, weight 0, for a logit of -inf)
};
__device__ __forceinline__ int bin_of(float x) { return min(kBins, (int)(x * -32.f)); }

// The cut of goal g among the row's `count` logits of weight above 0: s.cut,
// and the mass that is kept in s.keep_mass.  Every block of the cluster finds
// the same.  use: 0 for a kernel's first call, 1 for its second.
__device__ void resolve(Shared& s, const Row& r, const Goal& g, uint32_t count, int use) {
  pick(s, s.row, g, 0, 0);
  const int bucket = s.found;
  uint32_t above_cnt = s.found_above_cnt;
  unsigned long long above_mass = s.found_above_mass;
  uint32_t n = bucket < kBins ? s.found_cnt : count - above_cnt;   // (kBins: all below the histogram)
  uint32_t klo = 0, khi = 0xFFFFFFFFu;
  const bool by_key = n > kCap;
  if (by_key) {
    // the bucket's range of keys, then bins of that range until few are left or one value
    uint32_t lo = 0xFFFFFFFFu, hi = 0;
    for (int i = threadIdx.x; i < r.n; i += kThreads) {
      const float x = r.x(i);
      if (weight(x) == 0 || bin_of(x) != bucket) continue;
      lo = min(lo, key_of(r.z[i]));
      hi = max(hi, key_of(r.z[i]));
    }
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
    klo = 0xFFFFFFFFu;
    khi = 0;
    for (int q = 0; q < r.cluster; ++q) {
      klo = min(klo, remote_u32(&s.post_lo, q));
      khi = max(khi, remote_u32(&s.post_hi, q));
    }
    while (n > kCap && klo < khi) {
      static_assert(kBins == 512, "9 bits of the range");
      const int shift = max(0, 32 - __clz(khi - klo) - 9);
      cluster_sync();   // nobody reads the last histogram any more
      clear_histogram(s.own);
      __syncthreads();
      for (int i = threadIdx.x; i < r.n; i += kThreads) {
        const uint32_t k = key_of(r.z[i]);
        if (k < klo || k > khi) continue;
        const unsigned long long w = weight(r.x(i));
        if (w == 0) continue;
        atomicAdd(&s.own.cnt[(khi - k) >> shift], 1u);
        atomicAdd(&s.own.mass[(khi - k) >> shift], w);
      }
      cluster_sync();
      join_histogram(s, s.sub, r.cluster);
      pick(s, s.sub, g, above_cnt, above_mass);
      if (s.found >= kBins) break;   // (not reached: the goal lies in this range)
      n = s.found_cnt;
      above_cnt = s.found_above_cnt;
      above_mass = s.found_above_mass;
      khi -= (uint32_t)s.found << shift;
      klo = max(klo, khi - ((1u << shift) - 1));   // (keys of finite logits are at least 2^23)
    }
    cluster_sync();   // the same, ahead of the next call's; and of the posted range
  }
  if (n > kCap) {
    // equal logits: as many of them as the goal takes, by index
    const unsigned long long w = weight(scaled(logit_of(khi), r.top, r.t));
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
  // gather the bucket's members from the cluster
  if (threadIdx.x == 0) {
    s.list_n[use] = 0;
    s.nkeep = 0;
    s.keep_mass = above_mass;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < r.n; i += kThreads) {
    const float x = r.x(i);
    const uint32_t k = key_of(r.z[i]);
    if (weight(x) == 0 || (by_key ? k < klo || k > khi : bin_of(x) != bucket)) continue;
    const uint32_t at = atomicAdd(&s.list_n[use], 1u);
    if (at < kCap) {   // (always: n counts them)
      s.list_key[use][at] = k;
      s.list_idx[use][at] = r.lo + i;
    }
  }
  cluster_sync();
  uint32_t have = 0;
  for (int q = 0; q < r.cluster; ++q) {
    const uint32_t m = min(remote_u32(&s.list_n[use], q), (uint32_t)kCap - have);
    for (uint32_t j = threadIdx.x; j < m; j += kThreads) {
      const uint32_t k = remote_u32(&s.list_key[use][j], q);
      s.all.key[have + j] = k;
      s.all.idx[have + j] = (int)remote_u32(&s.list_idx[use][j], q);
      s.all.w[have + j] = weight(scaled(logit_of(k), r.top, r.t));
    }
    have += m;
  }
  __syncthreads();
  for (uint32_t c = threadIdx.x; c < have; c += kThreads) {
    const uint32_t key = s.all.key[c];
    const int idx = s.all.idx[c];
    uint32_t rank = 0;
    unsigned long long before = 0;
    for (uint32_t j = 0; j < have; ++j) {
      const bool better = s.all.key[j] > key || (s.all.key[j] == key && s.all.idx[j] < idx);
      rank += better;
      before += better ? s.all.w[j] : 0ull;
    }
    s.all.rank[c] = rank;
    if (g.by_count ? above_cnt + rank < g.count : above_mass + before < g.mass) {
      atomicMax(&s.nkeep, rank + 1);
      atomicAdd(&s.keep_mass, s.all.w[c]);
    }
  }
  __syncthreads();
  for (uint32_t c = threadIdx.x; c < have; c += kThreads)
    if (s.all.rank[c] + 1 == s.nkeep) s.cut = {s.all.key[c], s.all.idx[c]};
  __syncthreads();
}

__device__ __forceinline__ float read_logit(const float* p) { return __ldg(p); }
__device__ __forceinline__ float read_logit(const uint16_t* p) { return __uint_as_float((uint32_t)__ldg(p) << 16); }

template <class T>
__global__ void __launch_bounds__(kThreads) sample_kernel(const SampleParams p) {
  extern __shared__ __align__(16) uint8_t smem_raw[];
  Shared& s = *reinterpret_cast<Shared*>(smem_raw);
  float* z = reinterpret_cast<float*>(smem_raw + sizeof(Shared));
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, row = blockIdx.y;
  pdl_wait();
  pdl_launch_dependents();
  Row r;
  r.z = z;
  r.rank = (int)cluster_rank();
  r.cluster = p.cluster;
  r.lo = r.rank * p.chunk;
  r.n = max(0, min(p.chunk, p.vocab - r.lo));
  r.t = p.temperature ? __ldg(p.temperature + row) : 1.f;
  const int top_k = p.top_k ? __ldg(p.top_k + row) : 0;
  const float top_p = p.top_p ? __ldg(p.top_p + row) : 1.f, min_p = p.min_p ? __ldg(p.min_p + row) : 0.f;
  const float u = __ldg(p.u + row);
  // 1: the row, its largest logit
  const T* src = static_cast<const T*>(p.logits) + (int64_t)row * p.ld + r.lo;
  float top = -INFINITY;
#pragma unroll 8
  for (int i = tid; i < r.n; i += kThreads) {
    float v = read_logit(src + i);
    if (v != v) v = -INFINITY;
    z[i] = v;
    top = fmaxf(top, v);
  }
  for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
  if (lane == 0) s.red_f[warp] = top;
  clear_histogram(s.own);
  __syncthreads();
  for (int w = 0; w < kWarps; ++w) top = fmaxf(top, s.red_f[w]);
  if (tid == 0) s.post_max = top;
  cluster_sync();
  for (int q = 0; q < r.cluster; ++q) top = fmaxf(top, __uint_as_float(remote_u32(&s.post_max, q)));
  r.top = top;
  if (top == -INFINITY || !(r.t > 0.f) || min_p > 1.f) {
    // nothing to choose from, or the first of the largest logits alone
    if (tid == 0) s.post_first = 0x7FFFFFFF;
    __syncthreads();
    if (top > -INFINITY) {
      int first = 0x7FFFFFFF;
      for (int i = tid; i < r.n; i += kThreads)
        if (z[i] == top) first = min(first, r.lo + i);
      first = __reduce_min_sync(0xffffffffu, first);
      if (lane == 0) atomicMin(&s.post_first, first);
    }
    cluster_sync();
    if (r.rank == 0 && tid == 0) {
      int first = 0x7FFFFFFF;
      for (int q = 0; q < r.cluster; ++q) first = min(first, (int)remote_u32(&s.post_first, q));
      p.tokens[row] = first == 0x7FFFFFFF ? -1 : first;
    }
    cluster_sync();   // no block ends while its memory is being read
    return;
  }
  // 2: weights, their sum, the histogram
  const bool cut_k = top_k > 0 && top_k < p.vocab, cut_p = top_p < 1.f;
  unsigned long long mass = 0;
  uint32_t count = 0;
  s.cut = {0, 0x7FFFFFFF};   // everything
  if (cut_k || cut_p) {
    for (int i = tid; i < r.n; i += kThreads) {
      const float x = r.x(i);
      const unsigned long long w = weight(x);
      if (w == 0) continue;
      mass += w;
      ++count;
      const int b = bin_of(x);
      if (b < kBins) {
        atomicAdd(&s.own.cnt[b], 1u);
        atomicAdd(&s.own.mass[b], w);
      }
    }
    mass = block_sum(s, mass);
    count = (uint32_t)block_sum(s, count);
    if (tid == 0) {
      s.post_mass = mass;
      s.post_cnt = count;
    }
    cluster_sync();
    mass = 0;
    count = 0;
    for (int q = 0; q < r.cluster; ++q) {
      mass += remote_u64(&s.post_mass, q);
      count += remote_u32(&s.post_cnt, q);
    }
    join_histogram(s, s.row, r.cluster);
    // 3: the cuts
    if (cut_k && (uint32_t)top_k < count) {
      resolve(s, r, Goal{true, (uint32_t)top_k, 0}, count, 0);
      mass = s.keep_mass;
    }
    if (cut_p) {
      // kept: mass before it < top_p mass, that is, below that rounded up (the first one always)
      const double goal = ceil(fmax((double)top_p, 0.0) * (double)mass);
      resolve(s, r, Goal{false, 0, max(1ull, min(mass, (unsigned long long)goal))}, count, 1);
    }
  }
  __syncthreads();
  const Cut cut = s.cut;
  const float least = min_p > 0.f ? min_p : 0.f;
  auto kept = [&](int i) -> unsigned long long {
    const uint32_t k = key_of(z[i]);
    if (k < cut.key || (k == cut.key && r.lo + i > cut.idx)) return 0;
    const float x = r.x(i);
    return weight_f(x) >= least ? weight(x) : 0ull;
  };
  // 4: mass of what is kept, by index: a warp's segment, the blocks before this one
  const int seg = (r.n + kThreads - 1) / kThreads * 32, i0 = warp * seg, i1 = min(r.n, i0 + seg);
  unsigned long long sum = 0;
  for (int i = i0 + lane; i < i1; i += 32) sum += kept(i);
  for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  if (lane == 0) s.wsum[warp] = sum;
  __syncthreads();
  if (tid == 0) {
    unsigned long long all = 0;
    for (int w = 0; w < kWarps; ++w) all += s.wsum[w];
    s.post_kept = all;
  }
  cluster_sync();
  unsigned long long total = 0, before = 0;
  for (int q = 0; q < r.cluster; ++q) {
    const unsigned long long m = remote_u64(&s.post_kept, q);
    total += m;
    if (q < r.rank) before += m;
  }
  // the first kept index whose running sum exceeds u times the mass
  const double goal = floor(fmin(fmax((double)u, 0.0), 1.0) * (double)total);
  const unsigned long long target = min((unsigned long long)goal, total - 1);
  for (int w = 0; w < warp; ++w) before += s.wsum[w];
  if (before <= target && target < before + s.wsum[warp]) {   // (one warp of the cluster)
    for (int i = i0; i < i1; i += 32) {
      unsigned long long c = i + lane < i1 ? kept(i + lane) : 0;
      for (int d = 1; d < 32; d <<= 1) {
        const unsigned long long o = __shfl_up_sync(0xffffffffu, c, d);
        if (lane >= d) c += o;
      }
      const uint32_t past = __ballot_sync(0xffffffffu, before + c > target);
      if (past) {
        if (lane == 0) p.tokens[row] = r.lo + i + __ffs(past) - 1;
        break;
      }
      before += __shfl_sync(0xffffffffu, c, 31);
    }
  }
  cluster_sync();   // no block ends while its memory is being read
}

constexpr int kMaxChunk = (227 * 1024 - (int)sizeof(Shared)) / 4 / 32 * 32;

template <class T>
cudaError_t launch_sample(const SampleParams& p, int rows, int device, cudaStream_t st) {
  const int bytes = (int)sizeof(Shared) + 4 * p.chunk;
  static std::atomic<int> smem_set[64];
  const cudaError_t e = smem_limit_once(sample_kernel<T>, (int)sizeof(Shared) + 4 * kMaxChunk, device, smem_set);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)p.cluster, (unsigned)rows);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = (size_t)bytes;
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
  int dev = -1, major = 0, minor = 0;
  if (cudaGetDevice(&dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&minor, cudaDevAttrComputeCapabilityMinor, dev) != cudaSuccess)
    return SDQ_ERR_CUDA;
  if (major != 10 || minor != 3) return SDQ_ERR_UNSUPPORTED;
  SampleParams p;
  p.logits = logits; p.ld = ld;
  p.temperature = temperature; p.top_k = top_k; p.top_p = top_p; p.min_p = min_p; p.u = u;
  p.tokens = tokens;
  p.vocab = vocab;
  // blocks per row: of at least 2048 logits each, 8 at most
  p.cluster = 1;
  while (p.cluster < kMaxCluster && vocab > 2048 * p.cluster) p.cluster *= 2;
  p.chunk = ((vocab + p.cluster - 1) / p.cluster + 31) / 32 * 32;
  static_assert(kMaxVocab / kMaxCluster <= kMaxChunk, "a row fits in the cluster's shared memory");
  const cudaError_t e = type == SDQ_F32 ? launch_sample<float>(p, rows, dev, (cudaStream_t)stream)
                                        : launch_sample<uint16_t>(p, rows, dev, (cudaStream_t)stream);
  return e == cudaSuccess ? SDQ_OK : SDQ_ERR_CUDA;
}
