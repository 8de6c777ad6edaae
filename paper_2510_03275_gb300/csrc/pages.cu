// Block tables of a step: pages that come back to the pool, pages that the new
// tokens take from it, slots and positions (include/sdq.h).
#include <algorithm>

#include "common.cuh"

namespace sdq {

namespace {

constexpr int kThreads = 1024, kWarps = kThreads / 32;
constexpr uint32_t kMany = 1u << 30;   // sums stop here (above every bound that they are compared with)

struct PagesParams {
  sdq_pages a;
  int shift;   // log2 of the tokens of a page
  int per;     // sequences of a thread
};

__device__ __forceinline__ uint32_t add(uint32_t a, uint32_t b) { return min(a + b, kMany); }

// N exclusive sums over the block's threads, in place; total: of all of them.
template <int N>
__device__ __forceinline__ void scan(uint32_t (&v)[N], uint32_t (&total)[N], uint32_t (*sums)[kWarps]) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t up[N];
#pragma unroll
  for (int k = 0; k < N; ++k) {
    up[k] = v[k];
    for (int d = 1; d < 32; d <<= 1) {
      const uint32_t o = __shfl_up_sync(0xffffffffu, up[k], d);
      if (lane >= d) up[k] = add(up[k], o);
    }
    if (lane == 31) sums[k][warp] = up[k];
    const uint32_t before = __shfl_up_sync(0xffffffffu, up[k], 1);
    v[k] = lane == 0 ? 0 : before;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < N; ++k) {
    uint32_t w = lane < (int)(blockDim.x >> 5) ? sums[k][lane] : 0;   // (every warp on its own)
    for (int d = 1; d < 32; d <<= 1) {
      const uint32_t o = __shfl_up_sync(0xffffffffu, w, d);
      if (lane >= d) w = add(w, o);
    }
    total[k] = __shfl_sync(0xffffffffu, w, 31);
    const uint32_t before = __shfl_sync(0xffffffffu, w, max(warp - 1, 0));
    if (warp > 0) v[k] = add(v[k], before);
  }
  __syncthreads();   // (sums is written again)
}

// A sequence as the call finds it, and what it asks for.
struct Ask {
  int at;                     // its tokens (0 if it is done)
  uint32_t back, fresh, need; // pages that come back, new tokens, pages for them
};

__device__ __forceinline__ Ask ask_of(const PagesParams& p, int s) {
  const sdq_pages& a = p.a;
  const int size = 1 << p.shift;
  const int own = min(max(__ldcg(a.own_len + s), 0), 1 << 30);
  const int n = max(__ldg(a.new_len + s), 0);
  const bool done = a.done && __ldg(a.done + s) != 0;
  Ask r;
  r.back = done ? (uint32_t)min((own + size - 1) >> p.shift, a.page_columns) : 0;
  r.at = done ? 0 : own;
  const uint32_t held = (uint32_t)(r.at + size - 1) >> p.shift, end = ((uint32_t)r.at + (uint32_t)n + (uint32_t)(size - 1)) >> p.shift;
  const bool fits = end <= (uint32_t)a.page_columns;
  r.fresh = fits ? (uint32_t)n : 0;
  r.need = fits ? end - held : 0;
  return r;
}

// Sums over the sequences before one: asked for (tokens, pages), given.
struct Before {
  uint32_t asked_tokens, asked_pages, tokens, pages;
  // Takes sequence `q` in; what it gets: its new tokens, or none.
  __device__ uint32_t take(const Ask& q, uint32_t room, uint32_t available) {
    asked_tokens = add(asked_tokens, q.fresh);
    asked_pages = add(asked_pages, q.need);
    const bool ok = asked_tokens <= room && (q.need == 0 || asked_pages <= available);
    tokens += ok ? q.fresh : 0;
    pages += ok ? q.need : 0;
    return ok ? q.fresh : 0;
  }
};

// One cluster: every thread block sums up all sequences (a thread `per`
// neighbours of them, kOne: one, kept in registers), so that each can place
// any token by itself, and takes its share of the pages that come back and of
// the tokens.  A few thousand integers move; a chain of latencies bounds it.
template <bool kOne>
__global__ void __launch_bounds__(kThreads, 1) pages_kernel(const PagesParams p) {
  __shared__ uint32_t sums[3][kWarps];
  __shared__ Before before[kThreads];            // a thread's first sequence
  __shared__ Ask asks[kOne ? kThreads : 1];
  __shared__ uint32_t starts[kThreads + 1], backs[kThreads + 1];
  const sdq_pages& a = p.a;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, warps = blockDim.x >> 5;
  const int size = 1 << p.shift, blocks = gridDim.x;
  pdl_wait();
  pdl_launch_dependents();
  const int s0 = min(tid * p.per, a.n_seqs), s1 = min(s0 + p.per, a.n_seqs);
  const uint32_t had = (uint32_t)min(max(__ldcg(a.n_free), 0), a.n_pages);
  uint32_t asked[3] = {0, 0, 0}, all[3];         // pages back, tokens, pages
  Ask mine{};
  if (kOne && s0 < s1) {
    mine = ask_of(p, s0);
    asks[tid] = mine;
    asked[0] = mine.back;
    asked[1] = mine.fresh;
    asked[2] = mine.need;
  }
  if (!kOne)
    for (int s = s0; s < s1; ++s) {
      const Ask q = ask_of(p, s);
      asked[0] = add(asked[0], q.back);
      asked[1] = add(asked[1], q.fresh);
      asked[2] = add(asked[2], q.need);
    }
  scan(asked, all, sums);
  const uint32_t available = min(had + all[0], (uint32_t)a.n_pages);
  Before b{asked[1], asked[2], 0, 0};
  if (kOne) b.take(mine, (uint32_t)a.n_tokens, available);   // (one without a sequence asks for nothing)
  else
    for (int s = s0; s < s1; ++s) b.take(ask_of(p, s), (uint32_t)a.n_tokens, available);
  uint32_t given[2] = {b.tokens, b.pages}, taken[2];
  scan(given, taken, sums);
  before[tid] = Before{asked[1], asked[2], given[0], given[1]};
  starts[tid] = given[0];
  backs[tid] = asked[0];
  if (tid == 0) backs[blockDim.x] = all[0];
  __syncthreads();
  // pages that come back, on top of the free ones: a warp takes a thread's sequences
  if (all[0] > 0) {
    for (int c = blockIdx.x * warps + warp; c < (int)blockDim.x; c += blocks * warps) {
      if (backs[c + 1] == backs[c]) continue;
      uint32_t at = had + backs[c];
      for (int s = c * p.per; s < min((c + 1) * p.per, a.n_seqs); ++s) {
        const int n = (int)(kOne ? asks[c] : ask_of(p, s)).back;
        const int32_t* row = a.pages + (int64_t)s * a.page_stride;
#pragma unroll 4
        for (int i = lane; i < n; i += 32)
          if (at + i < (uint32_t)a.n_pages) a.free_pages[at + i] = __ldcg(row + i);
        at = add(at, (uint32_t)n);
      }
    }
    // (the pages go out again below; and nobody writes a table that is read here)
    if (blocks > 1) cluster_sync();
    else __syncthreads();
  }
  for (int t = blockIdx.x * blockDim.x + tid; t < a.n_tokens; t += blocks * blockDim.x) {
    int slot = -1, position = 0;
    if ((uint32_t)t < taken[0]) {
      int c = 0;   // the last thread whose first sequence starts at t or before it
      for (int d = blockDim.x / 2; d; d >>= 1)
        if (starts[c + d] <= (uint32_t)t) c += d;
      Before x = before[c];
      int s = c * p.per;
      Ask q;
      uint32_t first = x.tokens, first_page = x.pages;
      if (kOne) {
        q = asks[c];
      } else {
        uint32_t got;
        do {
          q = ask_of(p, s++);
          first = x.tokens;
          first_page = x.pages;
          got = x.take(q, (uint32_t)a.n_tokens, available);
        } while ((uint32_t)t >= first + got && s < a.n_seqs);
        --s;
      }
      const int place = q.at + (int)((uint32_t)t - first), column = place >> p.shift, held = (q.at + size - 1) >> p.shift;
      int32_t* entry = a.pages + (int64_t)s * a.page_stride + column;
      int page;
      if (column < held) {
        page = __ldcg(entry);
      } else {
        page = __ldcg(a.free_pages + (available - 1 - (first_page + (uint32_t)(column - held))));
        if ((place & (size - 1)) == 0) *entry = page;
      }
      if (page >= 0 && page < a.n_pages) slot = (page << p.shift) + (place & (size - 1));
      position = a.prefix_len + place;
    }
    if (a.slots) a.slots[t] = slot;
    if (a.positions) a.positions[t] = position;
  }
  // lengths last: they may stand where they were read (by every thread block, and,
  // where a thread has several sequences, for the tokens too)
  if (blocks > 1) cluster_sync();
  else if (!kOne) __syncthreads();
  if (blockIdx.x != 0) return;
  uint32_t first = given[0];
  b = before[tid];
  for (int s = s0; s < s1; ++s) {
    const Ask q = kOne ? mine : ask_of(p, s);
    a.token_start[s] = (int32_t)first;
    const uint32_t got = b.take(q, (uint32_t)a.n_tokens, available);
    first += got;
    a.own_out[s] = q.at + (int)got;
  }
  if (tid == 0) {
    a.token_start[a.n_seqs] = (int32_t)taken[0];
    *a.n_free_out = (int32_t)(available - taken[1]);
  }
}

}  // namespace

}  // namespace sdq

using namespace sdq;

extern "C" int sdq_pages_step(const sdq_pages* a, void* stream) {
  if (!a || !a->own_len || !a->new_len || !a->pages || !a->free_pages || !a->n_free || !a->token_start || !a->own_out || !a->n_free_out)
    return SDQ_ERR_INVALID_ARG;
  if (a->page_tokens != 16 && a->page_tokens != 32 && a->page_tokens != 64 && a->page_tokens != 128) return SDQ_ERR_INVALID_ARG;
  if (a->n_pages < 1 || (int64_t)a->n_pages * a->page_tokens >= (1ll << 31)) return SDQ_ERR_INVALID_ARG;
  if (a->n_seqs < 1 || a->n_seqs > 65535 || a->n_tokens < 1 || a->n_tokens > (1 << 20)) return SDQ_ERR_INVALID_ARG;
  if (a->page_columns < 1 || a->page_stride < a->page_columns || (int64_t)a->page_columns * a->page_tokens >= (1ll << 30)) return SDQ_ERR_INVALID_ARG;
  if (a->prefix_len < 0 || a->prefix_len >= (1 << 30)) return SDQ_ERR_INVALID_ARG;
  int dev = -1, sms = 0;
  const int supported = supported_device(&dev, &sms);
  if (supported != SDQ_OK) return supported;
  PagesParams p;
  p.a = *a;
  p.shift = 4;
  while ((1 << p.shift) < a->page_tokens) ++p.shift;
  // Threads for the sequences, a power of 2, and for the tokens; one thread block
  // for every 4096 tokens, or entries that may come back, up to 8.
  int threads = 128;
  while (threads < kThreads && threads < std::max(a->n_seqs, std::min(a->n_tokens, kThreads))) threads *= 2;
  p.per = (a->n_seqs + threads - 1) / threads;
  cudaLaunchConfig_t cfg = {};
  const int64_t moved = std::max<int64_t>(a->n_tokens, a->done ? std::min<int64_t>(a->n_pages, (int64_t)a->n_seqs * a->page_columns) : 0);
  const unsigned blocks = (unsigned)std::min<int64_t>(8, (moved + 4095) / 4096);
  cfg.gridDim = dim3(blocks);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.stream = (cudaStream_t)stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = blocks;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = blocks > 1 ? 2 : 1;
  const cudaError_t e = p.per == 1 ? cudaLaunchKernelEx(&cfg, pages_kernel<true>, p) : cudaLaunchKernelEx(&cfg, pages_kernel<false>, p);
  return e == cudaSuccess ? SDQ_OK : SDQ_ERR_CUDA;
}
