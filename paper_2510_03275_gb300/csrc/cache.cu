// The paged cache of keys and values: its handle, the rotation tables, and the
// kernel that appends a batch's keys and values (include/sdq.h).
#include <cuda.h>
#include <cudaTypedefs.h>

#include <algorithm>
#include <cmath>
#include <new>

#include "cache.cuh"

namespace sdq {

namespace {

constexpr int kThreads = 256;

struct AppendParams {
  sdq_batch b;
  sdq_rope rope;
  const void *q, *k, *v;
  int64_t ldq, ldk, ldv;
  uint16_t *kp, *vp, *q_out;
  int q_heads, kv_heads, dim, page, n_pages;
  int per_part;   // heads of a token that one block of a part takes
  sdq_head_norm norm;
};

// Four consecutive elements in fp32.
__device__ __forceinline__ float4 load4(const float* p) { return __ldg(reinterpret_cast<const float4*>(p)); }
__device__ __forceinline__ float4 load4(const uint16_t* p) {
  const uint2 r = __ldg(reinterpret_cast<const uint2*>(p));
  return make_float4(__uint_as_float(r.x << 16), __uint_as_float(r.x & 0xFFFF0000u), __uint_as_float(r.y << 16),
                     __uint_as_float(r.y & 0xFFFF0000u));
}
// (four of shared memory)
__device__ __forceinline__ float4 shared4(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ float4 shared4(const uint16_t* p) {
  const uint2 r = *reinterpret_cast<const uint2*>(p);
  return make_float4(__uint_as_float(r.x << 16), __uint_as_float(r.x & 0xFFFF0000u), __uint_as_float(r.y << 16),
                     __uint_as_float(r.y & 0xFFFF0000u));
}
__device__ __forceinline__ void store4(uint16_t* p, float4 a) {
  *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(a.x, a.y), pack_bf16x2(a.z, a.w));
}

// A head's elements in a thread's hands (a: 4, b: 4 more), normalised and rotated.
// Every rounding is written down, so that a token's values do not depend on the
// kernel, and so on the batch, that it comes with.
__device__ __forceinline__ float squares(const float4& a, const float4& b) {
  const float x = __fmaf_rn(a.w, a.w, __fmaf_rn(a.z, a.z, __fmaf_rn(a.y, a.y, __fmul_rn(a.x, a.x))));
  const float y = __fmaf_rn(b.w, b.w, __fmaf_rn(b.z, b.z, __fmaf_rn(b.y, b.y, __fmul_rn(b.x, b.x))));
  return __fadd_rn(x, y);
}
// (dim: a power of 2, so that its inverse is exact)
__device__ __forceinline__ void normalise(float4& a, float4& b, float sum_of_squares, int dim, float eps, const float4& wa, const float4& wb) {
  const float r = rsqrtf(__fmaf_rn(sum_of_squares, dim == 128 ? 1.f / 128 : 1.f / 64, eps));
  auto times = [&](const float4& x, const float4& w) {
    return make_float4(__fmul_rn(__fmul_rn(x.x, r), w.x), __fmul_rn(__fmul_rn(x.y, r), w.y), __fmul_rn(__fmul_rn(x.z, r), w.z),
                       __fmul_rn(__fmul_rn(x.w, r), w.w));
  };
  a = times(a, wa);
  b = times(b, wb);
}
// split: a and b are the pairs' first and second elements; else neighbours are.
__device__ __forceinline__ void rotate(float4& a, float4& b, const float4& cs, const float4& sn, bool split) {
  auto first = [](float u, float w, float c, float s) { return __fmaf_rn(u, c, -__fmul_rn(w, s)); };
  auto second = [](float u, float w, float c, float s) { return __fmaf_rn(w, c, __fmul_rn(u, s)); };
  const float4 x = a, y = b;
  if (split) {
    a = make_float4(first(x.x, y.x, cs.x, sn.x), first(x.y, y.y, cs.y, sn.y), first(x.z, y.z, cs.z, sn.z), first(x.w, y.w, cs.w, sn.w));
    b = make_float4(second(x.x, y.x, cs.x, sn.x), second(x.y, y.y, cs.y, sn.y), second(x.z, y.z, cs.z, sn.z), second(x.w, y.w, cs.w, sn.w));
  } else {
    a = make_float4(first(x.x, x.y, cs.x, sn.x), second(x.x, x.y, cs.x, sn.x), first(x.z, x.w, cs.y, sn.y), second(x.z, x.w, cs.y, sn.y));
    b = make_float4(first(y.x, y.y, cs.z, sn.z), second(y.x, y.y, cs.z, sn.z), first(y.z, y.w, cs.w, sn.w), second(y.z, y.w, cs.w, sn.w));
  }
}
// Where a token stands: its page (-1: its key and value are not kept), its place
// among its sequence's tokens, its position.
struct Place {
  int page, at, pos;
};
__device__ __forceinline__ Place place_of(const AppendParams& p, int t, int s) {
  const SeqSpan q = seq_span(p.b, s);
  Place r;
  r.at = q.own - q.count + (t - q.first);
  r.pos = max(0, p.b.prefix_len + min(r.at, q.own - 1));   // (min: a token beyond max_new has no place of its own)
  r.page = -1;
  if (t < q.first + q.count && r.at >= 0 && r.at < q.own) r.page = __ldg(p.b.pages + (int64_t)s * p.b.page_stride + r.at / p.page);
  if (r.page >= p.n_pages) r.page = -1;
  return r;
}

// Every element is read once and written once, rounded to bf16 there; what
// bounds it is HBM for prompts and the launch for single tokens.  A thread
// takes 8 elements of a head: 4 and their 4 partners dim / 2 further on, or
// 8 neighbours, so that both halves of a pair are in its registers, and the same
// ones of every head that it comes to, so that their cosines, sines and weights
// are read once per token (a read for each head, from the L1, cost as much as
// the data).  The next head's elements are under way while one is worked on.
// grid.x: tokens, grid.y: parts of a token's heads.  One token of 64 + 2 x 8 heads of
// 128, fp32: 1.6 us, 2.2 with norms; 256 of four sequences, without norms: 3.9 (a graph of 30 calls).
// kNorm: a head's threads are neighbours in one warp (8 or 16 of them) and add up
// its squares, all in fp32; whole warps stay in the loop for it.
// (Registers: 56 without norms.  Held to 40, so that more thread blocks fit, they
// spill: 1.9 us for the one token, 4.5 for the 256.)
template <class T, bool kNorm>
__global__ void __launch_bounds__(kThreads, kNorm ? 3 : 1) append_kernel(const AppendParams p) {
  pdl_wait();
  pdl_launch_dependents();
  const int t = blockIdx.x, lanes = p.dim / 8, half = p.rope.dim / 2;   // threads of a head
  const int g = threadIdx.x / lanes, c = threadIdx.x - g * lanes, step = kThreads / lanes;
  const bool turn = 8 * c < p.rope.dim, split = turn && !p.rope.interleaved;
  const int ea = split ? 4 * c : 8 * c, eb = split ? 4 * c + half : 8 * c + 4;
  const int n_heads = p.q_heads + 2 * p.kv_heads, last = min(n_heads, ((int)blockIdx.y + 1) * p.per_part) - 1;
  const Place at = place_of(p, t, seq_of_token(p.b.token_start, p.b.n_seqs, t));
  auto source = [&](int h) {
    return (h < p.q_heads                ? static_cast<const T*>(p.q) + t * p.ldq + h * p.dim
            : h < p.q_heads + p.kv_heads ? static_cast<const T*>(p.k) + t * p.ldk + (h - p.q_heads) * p.dim
                                         : static_cast<const T*>(p.v) + t * p.ldv + (h - p.q_heads - p.kv_heads) * p.dim);
  };
  // (kNorm: the heads of a warp, all of them while one is left: a lane past the end only takes part in the sums)
  const int together = kNorm ? 32 / lanes - 1 : 0;
  int h = blockIdx.y * p.per_part + g;
  if ((h & ~together) > last) return;
  const T* src = source(min(h, last));
  float4 xa = load4(src + ea), xb = load4(src + eb), cs = {}, sn = {}, wqa = {}, wqb = {}, wka = {}, wkb = {};
  if (turn) {
    cs = load4(p.rope.cos + (int64_t)at.pos * half + 4 * c);
    sn = load4(p.rope.sin + (int64_t)at.pos * half + 4 * c);
  }
  if (kNorm) {
    if (p.norm.q && !p.norm.q_per_head) wqa = load4(p.norm.q + ea), wqb = load4(p.norm.q + eb);
    if (p.norm.k && !p.norm.k_per_head) wka = load4(p.norm.k + ea), wkb = load4(p.norm.k + eb);
  }
  for (; (h & ~together) <= last; h += step) {
    float4 a = xa, b = xb;
    if (((h + step) & ~together) <= last) {
      src = source(min(h + step, last));
      xa = load4(src + ea);
      xb = load4(src + eb);
    }
    const bool is_q = h < p.q_heads, is_v = h >= p.q_heads + p.kv_heads;
    const int kh = is_q ? h : is_v ? h - p.q_heads - p.kv_heads : h - p.q_heads;
    if (kNorm) {
      float sq = squares(a, b);
      for (int d = 1; d < lanes; d <<= 1) sq += __shfl_xor_sync(0xffffffffu, sq, d);
      if (h > last) break;
      const float* w = is_q ? p.norm.q : is_v ? nullptr : p.norm.k;
      if (w) {
        float4 wa = is_q ? wqa : wka, wb = is_q ? wqb : wkb;
        if (is_q ? p.norm.q_per_head : p.norm.k_per_head) wa = load4(w + kh * p.dim + ea), wb = load4(w + kh * p.dim + eb);
        normalise(a, b, sq, p.dim, p.norm.eps, wa, wb);
      }
    }
    if (turn && !is_v) rotate(a, b, cs, sn, split);
    uint16_t* dst;
    if (is_q) {
      dst = p.q_out + ((int64_t)t * p.q_heads + kh) * p.dim;
    } else {
      if (at.page < 0) continue;
      dst = (is_v ? p.vp : p.kp) + (((int64_t)at.page * p.kv_heads + kh) * p.page + at.at % p.page) * p.dim;
    }
    store4(dst + ea, a);
    store4(dst + eb, b);
  }
}

// Without norms, many tokens: thread blocks enough for every SM to hold several, so
// that what hides the loads is their number and not each one's own next load.  A
// thread holds 8 elements and nothing from one head to the next (38 registers, 6
// thread blocks of an SM against 4).  fp32, us here and by append_kernel: 64 + 2 x 8
// heads of 128, 900 tokens 11.1, 12.8; 2400 25.7 (84 % of the measured copy
// bandwidth), 27.8; 3 x 12 heads of 64, 400 tokens 2.4, 2.8; 2400 8.9, 10.9.
// (append_kernel is ahead once more where its blocks just fill all places, 608 tokens:
// 600 of 64 + 2 x 8 heads 9.0, 8.4; 400 of 8 + 2 heads 2.0, 2.6.  So it takes calls of up
// to two tokens an SM, where it is ahead for all of these but the last: 256 2.0, 2.1.)
template <class T>
__global__ void __launch_bounds__(kThreads) append_many_kernel(const AppendParams p) {
  pdl_wait();
  pdl_launch_dependents();
  const int t = blockIdx.x, lanes = p.dim / 8, half = p.rope.dim / 2;
  const Place at = place_of(p, t, seq_of_token(p.b.token_start, p.b.n_seqs, t));
  const int units = (p.q_heads + 2 * p.kv_heads) * lanes;
  for (int u = threadIdx.x; u < units; u += kThreads) {
    const int h = u / lanes, c = u - h * lanes;
    const bool is_q = h < p.q_heads, is_v = h >= p.q_heads + p.kv_heads;
    const int kh = is_q ? h : is_v ? h - p.q_heads - p.kv_heads : h - p.q_heads;
    const T* src = is_q   ? static_cast<const T*>(p.q) + t * p.ldq + kh * p.dim
                   : is_v ? static_cast<const T*>(p.v) + t * p.ldv + kh * p.dim
                          : static_cast<const T*>(p.k) + t * p.ldk + kh * p.dim;
    const bool turn = !is_v && 8 * c < p.rope.dim, split = turn && !p.rope.interleaved;
    const int ea = split ? 4 * c : 8 * c, eb = split ? 4 * c + half : 8 * c + 4;
    float4 a = load4(src + ea), b = load4(src + eb);
    if (turn) {
      const float4 cs = load4(p.rope.cos + (int64_t)at.pos * half + 4 * c);
      const float4 sn = load4(p.rope.sin + (int64_t)at.pos * half + 4 * c);
      rotate(a, b, cs, sn, split);
    }
    uint16_t* dst;
    if (is_q) {
      dst = p.q_out + ((int64_t)t * p.q_heads + kh) * p.dim;
    } else {
      if (at.page < 0) continue;
      dst = (is_v ? p.vp : p.kp) + (((int64_t)at.page * p.kv_heads + kh) * p.page + at.at % p.page) * p.dim;
    }
    store4(dst + ea, a);
    store4(dst + eb, b);
  }
}

// The same for many tokens with norms, or in bf16.  Loads that wait in registers are too
// few bytes under way here (the arithmetic needs the registers): a warp streams
// pieces of kPiece bytes, some heads of one token's q, k or v, through a ring of its
// own in shared memory, 192 KB of an SM under way at once.  The line of pieces, token
// by token, is cut into equal shares for all warps; what a token needs (its
// place, its cosines and sines) is looked up when a share comes to it.
// 3710 tokens of 64 + 2 x 8 heads of 128, normalised: fp32 42.5 us (79 % of the
// measured copy bandwidth; append_kernel 52), bf16 38.3 (61.6: the sums'
// shuffles, not the bytes); without norms fp32 40.0 (append_many_kernel 37.8, so these
// stay there), bf16 28.8 (34.5).  256 tokens, normalised: fp32 7.5 (6.3), bf16 6.3
// (6.9); 512 of 3 x 12 heads of 64: 4.6 (5.4), 256 of them 4.5 (3.5).
constexpr int kStreamWarps = 16, kPiece = 4096, kStages = 3;
constexpr int64_t kStreamHeads = 24576;   // of q, k and v, from which this kernel takes a call
constexpr int kStreamSmem = kStreamWarps * kStages * kPiece;

template <class T, bool kNorm>
__global__ void __launch_bounds__(32 * kStreamWarps) append_stream_kernel(const AppendParams p) {
  extern __shared__ __align__(16) uint8_t ring[];
  pdl_wait();
  pdl_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint8_t* mine = ring + warp * (kStages * kPiece);
  const int lanes = p.dim / 8, half = p.rope.dim / 2, c = lane & (lanes - 1);
  const bool turn = 8 * c < p.rope.dim, split = turn && !p.rope.interleaved;
  const int ea = split ? 4 * c : 8 * c, eb = split ? 4 * c + half : 8 * c + 4;
  const int hp = kPiece / (p.dim * (int)sizeof(T)), nq = (p.q_heads + hp - 1) / hp, nk = (p.kv_heads + hp - 1) / hp;
  const int64_t per_token = nq + 2 * nk, total = per_token * p.b.n_tokens, warps = (int64_t)gridDim.x * kStreamWarps;
  const int64_t share = (total + warps - 1) / warps, i0 = min(total, ((int64_t)blockIdx.x * kStreamWarps + warp) * share);
  const int n = (int)(min(total, i0 + share) - i0);
  if (n <= 0) return;
  // piece: of token t, the part-th of its pieces
  struct Where {
    int t, part;
  };
  auto next = [&](Where& w) {
    if (++w.part == (int)per_token) w.part = 0, ++w.t;
  };
  // which of q, k, v (0, 1, 2), the first head, how many
  struct Heads {
    int of, first, count;
  };
  auto heads_of = [&](int part) {
    Heads h;
    h.of = part < nq ? 0 : part < nq + nk ? 1 : 2;
    h.first = (part - (h.of == 0 ? 0 : h.of == 1 ? nq : nq + nk)) * hp;
    h.count = min(hp, (h.of == 0 ? p.q_heads : p.kv_heads) - h.first);
    return h;
  };
  Where in{(int)(i0 / per_token), (int)(i0 % per_token)}, at = in;
  int issued = 0;
  auto issue = [&]() {
    if (issued < n) {
      const Heads h = heads_of(in.part);
      const T* src = (h.of == 0   ? static_cast<const T*>(p.q) + in.t * p.ldq
                      : h.of == 1 ? static_cast<const T*>(p.k) + in.t * p.ldk
                                  : static_cast<const T*>(p.v) + in.t * p.ldv) + h.first * p.dim;
      uint8_t* dst = mine + (issued % kStages) * kPiece;
      for (int j = 16 * lane; j < h.count * p.dim * (int)sizeof(T); j += 512) cp_async16(dst + j, reinterpret_cast<const uint8_t*>(src) + j, 16);
      next(in);
    }
    cp_async_commit();
    ++issued;
  };
  for (int k = 0; k < kStages - 1; ++k) issue();
  float4 cs = {}, sn = {}, wqa = {}, wqb = {}, wka = {}, wkb = {};
  if (kNorm) {
    if (p.norm.q && !p.norm.q_per_head) wqa = load4(p.norm.q + ea), wqb = load4(p.norm.q + eb);
    if (p.norm.k && !p.norm.k_per_head) wka = load4(p.norm.k + ea), wkb = load4(p.norm.k + eb);
  }
  int s = -1, s_end = 0, t = -1;   // the sequence, the token behind it, the token that is looked up
  Place place{};
  for (int i = 0; i < n; ++i, next(at)) {
    issue();
    if (at.t != t) {
      t = at.t;
      if (s < 0 || t >= s_end) {
        s = seq_of_token(p.b.token_start, p.b.n_seqs, t);
        s_end = s + 1 < p.b.n_seqs ? __ldg(p.b.token_start + s + 1) : p.b.n_tokens;
      }
      place = place_of(p, t, s);
      if (turn) {
        cs = load4(p.rope.cos + (int64_t)place.pos * half + 4 * c);
        sn = load4(p.rope.sin + (int64_t)place.pos * half + 4 * c);
      }
    }
    cp_async_wait_group<kStages - 1>();
    __syncwarp();
    const Heads h = heads_of(at.part);
    const T* from = reinterpret_cast<const T*>(mine + (i % kStages) * kPiece);
    const float* w = kNorm ? (h.of == 0 ? p.norm.q : h.of == 1 ? p.norm.k : nullptr) : nullptr;
    const bool each = kNorm && (h.of == 0 ? p.norm.q_per_head : p.norm.k_per_head);
    const bool keep = h.of == 0 || place.page >= 0;
    uint16_t* to = h.of == 0 ? p.q_out + ((int64_t)t * p.q_heads + h.first) * p.dim
                             : (h.of == 1 ? p.kp : p.vp) + (((int64_t)max(place.page, 0) * p.kv_heads + h.first) * p.page + place.at % p.page) * p.dim;
    const int64_t ld = h.of == 0 ? p.dim : (int64_t)p.page * p.dim;
    // kBatch heads of a thread at once, so that their chains of shuffles run side by side (whole warps)
    constexpr int kBatch = 4;
    const int mine_first = lane / lanes, step = 32 / lanes;
    for (int g0 = 0; g0 < h.count; g0 += kBatch * step) {
      float4 a[kBatch], b[kBatch];
      float sq[kBatch];
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        const int k = min(g0 + mine_first + u * step, h.count - 1);
        a[u] = shared4(from + k * p.dim + ea);
        b[u] = shared4(from + k * p.dim + eb);
        sq[u] = squares(a[u], b[u]);
      }
      if (kNorm && w) {
        for (int d = 1; d < lanes; d <<= 1) {
#pragma unroll
          for (int u = 0; u < kBatch; ++u) sq[u] += __shfl_xor_sync(0xffffffffu, sq[u], d);
        }
      }
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        const int k = g0 + mine_first + u * step;
        if (k >= h.count || !keep) continue;
        if (kNorm && w) {
          float4 wa = h.of == 0 ? wqa : wka, wb = h.of == 0 ? wqb : wkb;
          if (each) wa = load4(w + (h.first + k) * p.dim + ea), wb = load4(w + (h.first + k) * p.dim + eb);
          normalise(a[u], b[u], sq[u], p.dim, p.norm.eps, wa, wb);
        }
        if (turn && h.of < 2) rotate(a[u], b[u], cs, sn, split);
        store4(to + k * ld + ea, a[u]);
        store4(to + k * ld + eb, b[u]);
      }
    }
    __syncwarp();   // (the piece is read)
  }
  cp_async_wait_all();
}

bool valid_desc(const sdq_cache_desc* d) {
  if (!d || d->kv_heads < 1 || d->kv_heads > 1024 || (d->head_dim != 64 && d->head_dim != 128)) return false;
  if (d->page_tokens != 16 && d->page_tokens != 32 && d->page_tokens != 64 && d->page_tokens != 128) return false;
  return d->n_pages >= 1 && (int64_t)d->n_pages * d->kv_heads * d->page_tokens < (1ll << 31);
}

bool multiple16(const void* p, int64_t ld, int size) {
  return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && (ld * size) % 16 == 0;
}

}  // namespace

int check_cache_device(const sdq_cache_s* c) {
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess) return SDQ_ERR_CUDA;
  return dev == c->device ? SDQ_OK : SDQ_ERR_INVALID_ARG;
}

int check_batch(const sdq_cache_s* c, const sdq_batch* b, int32_t q_heads) {
  if (!c || !b || !b->token_start || !b->own_len || !b->pages) return SDQ_ERR_INVALID_ARG;
  if (q_heads < 1 || q_heads > 4096 || q_heads % c->desc.kv_heads) return SDQ_ERR_INVALID_ARG;
  if (b->n_seqs < 1 || b->n_seqs > 65535 || b->n_tokens < 1 || b->n_tokens > (1 << 20)) return SDQ_ERR_INVALID_ARG;
  if ((int64_t)b->n_tokens * q_heads >= (1ll << 31)) return SDQ_ERR_INVALID_ARG;
  if (b->max_new < 1 || b->max_new > b->n_tokens || b->max_own < 0 || b->max_own >= (1 << 30)) return SDQ_ERR_INVALID_ARG;
  if (b->page_stride < 0 || b->max_own > (int64_t)b->page_stride * c->desc.page_tokens) return SDQ_ERR_INVALID_ARG;
  if (((int64_t)std::max(b->max_own, b->prefix_len) + 64) * c->desc.kv_heads >= (1ll << 31)) return SDQ_ERR_INVALID_ARG;
  if (b->prefix_len < 0 || b->prefix_len >= (1 << 30) || (b->prefix_len > 0 && !b->prefix_pages)) return SDQ_ERR_INVALID_ARG;
  return SDQ_OK;
}

}  // namespace sdq

using namespace sdq;

extern "C" size_t sdq_cache_bytes(const sdq_cache_desc* d) {
  if (!valid_desc(d)) return 0;
  return (size_t)d->n_pages * d->kv_heads * d->page_tokens * d->head_dim * sizeof(uint16_t);
}

extern "C" int sdq_cache_create(const sdq_cache_desc* desc, uint16_t* k_pages, uint16_t* v_pages, sdq_cache* out) {
  if (!out) return SDQ_ERR_INVALID_ARG;
  *out = nullptr;
  if (!valid_desc(desc) || !k_pages || !v_pages) return SDQ_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(k_pages) | reinterpret_cast<uintptr_t>(v_pages)) & 127u) return SDQ_ERR_INVALID_ARG;
  int dev = 0, major = 0, minor = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&minor, cudaDevAttrComputeCapabilityMinor, dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return SDQ_ERR_CUDA;
  if (major != 10 || minor != 3) return SDQ_ERR_UNSUPPORTED;
  auto enc = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(tensor_map_encoder());
  if (!enc) return SDQ_ERR_UNSUPPORTED;
  sdq_cache_s* c = new (std::nothrow) sdq_cache_s();
  if (!c) return SDQ_ERR_ALLOC;
  c->desc = *desc;
  c->device = dev;
  c->sm_count = sms;
  c->k = k_pages;
  c->v = v_pages;
  c->rows = (int64_t)desc->n_pages * desc->kv_heads * desc->page_tokens;
  const cuuint64_t row = (cuuint64_t)desc->head_dim * 2, halves = (cuuint64_t)desc->head_dim / 64;
  const cuuint64_t dims[3] = {(cuuint64_t)desc->head_dim, (cuuint64_t)c->rows, 0}, tdims[3] = {64, (cuuint64_t)c->rows, halves};
  const cuuint64_t strides[2] = {row, 128};
  const cuuint32_t box[2] = {64, (cuuint32_t)cache_box_rows(*desc)}, tbox[3] = {64, 16, (cuuint32_t)halves}, estr[3] = {1, 1, 1};
  for (int i = 0; i < 4; ++i) {
    const bool tile = i >= 2;
    CUtensorMap* map = i == 0 ? &c->kmap : i == 1 ? &c->vmap : i == 2 ? &c->ktile : &c->vtile;
    if (enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, tile ? 3 : 2, i & 1 ? v_pages : k_pages, tile ? tdims : dims, strides,
            tile ? tbox : box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS) {
      delete c;
      return SDQ_ERR_CUDA;
    }
  }
  *out = c;
  return SDQ_OK;
}

extern "C" int sdq_cache_destroy(sdq_cache c) {
  if (!c) return SDQ_ERR_INVALID_ARG;
  delete c;
  return SDQ_OK;
}

extern "C" int sdq_rope_table(int32_t n_pos, int32_t dim, double base, float* cos_host, float* sin_host) {
  if (n_pos < 1 || dim < 2 || dim % 2 || !(base > 0) || !std::isfinite(base) || !cos_host || !sin_host) return SDQ_ERR_INVALID_ARG;
  for (int32_t p = 0; p < n_pos; ++p)
    for (int32_t j = 0; j < dim / 2; ++j) {
      const double a = p * std::pow(base, -2.0 * j / dim);
      cos_host[(size_t)p * (dim / 2) + j] = (float)std::cos(a);
      sin_host[(size_t)p * (dim / 2) + j] = (float)std::sin(a);
    }
  return SDQ_OK;
}

static int append(sdq_cache c, const sdq_batch* b, int32_t q_heads, const void* q, int64_t ldq, const void* k, int64_t ldk,
                  const void* v, int64_t ldv, int32_t type, const sdq_rope* rope, const sdq_head_norm* norm, uint16_t* q_out,
                  void* stream) {
  int st = check_batch(c, b, q_heads);
  if (st != SDQ_OK) return st;
  if ((st = check_cache_device(c)) != SDQ_OK) return st;
  if (!q || !k || !v || !rope || !q_out || (type != SDQ_F32 && type != SDQ_BF16)) return SDQ_ERR_INVALID_ARG;
  const int d = c->desc.head_dim, size = type == SDQ_F32 ? 4 : 2;
  if (ldq < (int64_t)q_heads * d || ldk < (int64_t)c->desc.kv_heads * d || ldv < (int64_t)c->desc.kv_heads * d) return SDQ_ERR_INVALID_ARG;
  if (!multiple16(q, ldq, size) || !multiple16(k, ldk, size) || !multiple16(v, ldv, size) || !multiple16(q_out, 0, 2)) return SDQ_ERR_INVALID_ARG;
  if (rope->dim < 0 || rope->dim > d || rope->dim % 8 || (rope->interleaved != 0 && rope->interleaved != 1)) return SDQ_ERR_INVALID_ARG;
  if (rope->dim > 0) {
    if (!rope->cos || !rope->sin || !multiple16(rope->cos, 0, 4) || !multiple16(rope->sin, 0, 4)) return SDQ_ERR_INVALID_ARG;
    if (rope->n_pos < 1 || rope->n_pos < (int64_t)b->prefix_len + b->max_own) return SDQ_ERR_INVALID_ARG;
  }
  if (norm) {
    if (!multiple16(norm->q, 0, 4) || !multiple16(norm->k, 0, 4)) return SDQ_ERR_INVALID_ARG;
    if ((norm->q_per_head != 0 && norm->q_per_head != 1) || (norm->k_per_head != 0 && norm->k_per_head != 1)) return SDQ_ERR_INVALID_ARG;
    if (!(norm->eps > 0.f) || !std::isfinite(norm->eps)) return SDQ_ERR_INVALID_ARG;
  }
  AppendParams p;
  p.norm = norm ? *norm : sdq_head_norm{};
  p.b = *b;
  p.rope = *rope;
  p.q = q; p.k = k; p.v = v;
  p.ldq = ldq; p.ldk = ldk; p.ldv = ldv;
  p.kp = c->k; p.vp = c->v; p.q_out = q_out;
  p.q_heads = q_heads; p.kv_heads = c->desc.kv_heads; p.dim = d; p.page = c->desc.page_tokens; p.n_pages = c->desc.n_pages;
  const int heads = q_heads + 2 * c->desc.kv_heads, step = kThreads / (d / 8);   // heads that a block has in hand at once
  const int parts = std::max(1, std::min((heads + step - 1) / step, 2 * c->sm_count / b->n_tokens));
  p.per_part = ((heads + parts - 1) / parts + step - 1) / step * step;
  const dim3 grid((unsigned)b->n_tokens, (unsigned)((heads + p.per_part - 1) / p.per_part));
  cudaStream_t cs = (cudaStream_t)stream;
  cudaError_t e;
  if ((norm || type == SDQ_BF16) && (int64_t)b->n_tokens * heads >= kStreamHeads) {
    static std::atomic<int> smem_set[3][64];
    auto run = [&](auto kernel, int which) {
      const cudaError_t set = smem_limit_once(kernel, kStreamSmem, c->device, smem_set[which]);
      if (set != cudaSuccess) return set;
      return launch_pdl(kernel, dim3((unsigned)c->sm_count), dim3(32 * kStreamWarps), (size_t)kStreamSmem, cs, p);
    };
    e = type == SDQ_F32 ? run(append_stream_kernel<float, true>, 0)
        : norm          ? run(append_stream_kernel<uint16_t, true>, 1)
                        : run(append_stream_kernel<uint16_t, false>, 2);
  } else if (!norm && b->n_tokens > 2 * c->sm_count) {   // (grid.y is 1 there)
    const dim3 tokens((unsigned)b->n_tokens);
    e = type == SDQ_F32 ? launch_pdl(append_many_kernel<float>, tokens, dim3(kThreads), 0, cs, p)
                        : launch_pdl(append_many_kernel<uint16_t>, tokens, dim3(kThreads), 0, cs, p);
  } else {
    auto run = [&](auto kernel) { return launch_pdl(kernel, grid, dim3(kThreads), 0, cs, p); };
    e = type == SDQ_F32 ? norm ? run(append_kernel<float, true>) : run(append_kernel<float, false>)
        : norm          ? run(append_kernel<uint16_t, true>)
                        : run(append_kernel<uint16_t, false>);
  }
  return e == cudaSuccess ? SDQ_OK : SDQ_ERR_CUDA;
}

extern "C" int sdq_cache_append(sdq_cache c, const sdq_batch* b, int32_t q_heads, const void* q, int64_t ldq,
                                const void* k, int64_t ldk, const void* v, int64_t ldv, int32_t type,
                                const sdq_rope* rope, uint16_t* q_out, void* stream) {
  return append(c, b, q_heads, q, ldq, k, ldk, v, ldv, type, rope, nullptr, q_out, stream);
}

extern "C" int sdq_cache_append_norm(sdq_cache c, const sdq_batch* b, int32_t q_heads, const void* q, int64_t ldq,
                                     const void* k, int64_t ldk, const void* v, int64_t ldv, int32_t type,
                                     const sdq_rope* rope, const sdq_head_norm* norm, uint16_t* q_out, void* stream) {
  if (!norm) return SDQ_ERR_INVALID_ARG;
  return append(c, b, q_heads, q, ldq, k, ldk, v, ldv, type, rope, norm, q_out, stream);
}
