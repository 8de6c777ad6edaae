// Attention over the paged cache: the kernel for few query rows per key head
// (single and drafted tokens).
#include "attention.cuh"

namespace sdq {

namespace {

// ------------------------------------------------------------ narrow kernel
// Up to 8 NT query rows (new token major, then head of the group) share a key
// head's keys, so HBM bounds it: every key and value is read once.  The work
// is a line of tiles of 16 keys, (sequence, key head) by (sequence, key head),
// cut into equal shares for all resident warps: no share is longer than
// another by more than a tile, whatever the lengths are.  A warp streams its
// share through a ring of its own (TMA, 128-byte swizzle, one copy each for a
// tile's keys and values) and keeps its own maxima, sums and outputs in
// registers: warps meet only at the end, once per thread block, where the
// pieces of a (sequence, head) are joined; those that also lie in other thread
// blocks go through the workspace, and the last to arrive joins them.
//   S^T = K Q^T with the keys as the MMA's 16 rows and 8 queries as its
//   columns (the other way round half of a 16-row tile would be padding), O^T
//   += V^T P^T; K and V fragments come by ldmatrix, P^T is turned from the
//   accumulator's layout into the operand's by movmatrix.
// With a window (kWindow) a unit's tiles are those that some token of the
// sequence sees: of the prefix (unless that is a part of its own) its first keys and the
// window's, then of the sequence's own the same.  What the tokens of a unit see is then not nested, so a
// value that is not finite and not every token's goes to those that see it by an
// addition.  64 sequences of 1 to 16384 tokens, 64 heads, window 1024 and 4 first: 28.8
// us (3.6 TB/s: the ends as above); 2 x 3 tokens, window 32768: 72 us.  Over windows of
// 16352, 32768, 65600 and 131264 that is 33 us and the keys at 7.2 TB/s; as many keys
// without a window 30 and the same rate, one token 13: 24 rows cost that much beside
// their keys, a window 2 to 3.  (A third stage in the scratch's place gains nothing.)
// P is rounded to bf16 for its product (relative 2^-8 at most per weight, as
// the values themselves carry); sums, maxima and outputs are fp32.
// 64 tokens of 64 heads (8 key heads of 128) on 1 to 4096 keys each: 43 us, 4.7
// TB/s; 2 x 3 tokens on 65537 to 131072: 164 us, 5.9 TB/s.  One token on 1037
// keys takes 10.7 us in a graph, a chain of latencies: a block's tables and queries 4000
// cycles, its tiles 2500, its pieces 3300, the ticket 3000 to 6000, the join of
// the blocks 3500.
constexpr int kWarps = 8, kThreads = 32 * kWarps, kTile = 16;
// A (sequence, head) takes as many places of the line as it has tiles, and
// kUnitCost more: its queries, its output and the join cost its warp about as
// much time as that many tiles.
constexpr int kUnitCost = 2;
// Places of a warp's share at least (one sequence of 1037 keys, 8 key heads: 10.7
// us; with 1 instead 11.0, with 3 11.3).
constexpr int64_t kMinShare = 2;

template <int D, int NT> struct NarrowShape {
  static constexpr int kRows = 8 * NT;
  static constexpr int kMat = kTile * D * 2;                   // bytes: K or V of a tile, [half][16 keys][128]
  static constexpr int kStages = D == 128 ? 2 : 4;
  static constexpr int kRing = kStages * 2 * kMat;             // of a warp; holds a piece (kRows x D fp32) at the end
  static constexpr int kScratch = 8 * D * 4;                   // of a warp: 8 rows of its output
  static constexpr int kSmem = 1024 + kWarps * (kRing + kScratch);
  static_assert(kRing >= kRows * D * 4, "a piece fits in a warp's ring");
};

__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];\n"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t (&r)[4], uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];\n"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ uint32_t movmatrix(uint32_t a) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;\n" : "=r"(r) : "r"(a));
  return r;
}
__device__ __forceinline__ void tma_load_3d_warp(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, uint32_t bar) {
  asm volatile(SDQ_ELECT
               "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
               " [%0], [%1, {%2, %3, %4}], [%5];\n}\n" ::"r"(dst),
               "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(bar) : "memory");
}

// a / b for numbers that mostly fit 32 bits (a 64-bit division costs 500 cycles).
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
  return (uint64_t)(a | b) >> 32 ? a / b : (int64_t)((uint32_t)a / (uint32_t)b);
}

// A (sequence, key head), or the whole batch and a key head against the prefix.
struct Unit {
  int s, h;                  // sequence (-1: the batch)
  int first, rows, keys, count;
  int tiles;
  int64_t a;                 // its first place in the line (its tiles', then kUnitCost more)
};

// Row r of a unit: its token (r below 32: exact).
__device__ __forceinline__ int token_of(const AttendParams& p, int r) { return (int)((uint32_t)r * p.group_inverse >> 16); }

// With a window: the tiles of a sequence's unit, first those of the prefix.
struct UnitLine {
  Line prefix, own;
  __device__ int tiles() const { return prefix.tiles + own.tiles; }
  __device__ bool in_prefix(int i) const volatile { return i < prefix.tiles; }
  __device__ int tile(int i) const volatile { return i < prefix.tiles ? prefix.tile(i) : own.tile(i - prefix.tiles); }
};
__device__ __forceinline__ UnitLine unit_line(const AttendParams& p, int count, int own) {
  const int first = position_of(p, own - count);
  return UnitLine{p.apart ? Line{0, 0, 0} : line_of<kTile>(p, p.b.prefix_len, 0, first), line_of<kTile>(p, own, p.b.prefix_len, first)};
}

// The line of units that have tiles.  All of it by whole warps: a lane holds
// the span of one of 32 consecutive sequences.
template <bool kWindow>
struct Walk {
  const AttendParams& p;
  const int part;
  int base = -1;             // of the 32 sequences held
  SeqSpan held;
  __device__ Walk(const AttendParams& p_, int part_) : p(p_), part(part_) {}
  __device__ void hold(int s0) {
    if (s0 == base) return;
    base = s0;
    const int s = s0 + (int)(threadIdx.x & 31);
    held = SeqSpan{0, 0, 0};
    if (s < p.b.n_seqs) held = seq_span(p.b, s);
  }
  __device__ int tiles_of(const SeqSpan& q) const {   // per key head
    if (kWindow) return q.count > 0 ? unit_line(p, q.count, q.own).tiles() : 0;
    return q.count > 0 ? (q.own + kTile - 1) / kTile : 0;
  }
  __device__ static int places_of(int tiles) { return tiles > 0 ? tiles + kUnitCost : 0; }
  // All places.
  __device__ int64_t total() {
    if (part == kPrefix) return (int64_t)p.kv_heads * places_of((p.b.prefix_len + kTile - 1) / kTile);
    int64_t n = 0;
    for (int s0 = (p.b.n_seqs - 1) & ~31; s0 >= 0; s0 -= 32) {   // (the first 32 last: a search begins there)
      hold(s0);
      n += places_of(tiles_of(held));
    }
    if (p.b.n_seqs == 1) return __shfl_sync(0xffffffffu, n, 0) * p.kv_heads;
    for (int d = 16; d; d >>= 1) n += __shfl_xor_sync(0xffffffffu, n, d);
    return n * p.kv_heads;
  }
  __device__ void enter(Unit& u, int s) {
    hold(s & ~31);
    u.s = s;
    u.first = __shfl_sync(0xffffffffu, held.first, s & 31);
    u.count = __shfl_sync(0xffffffffu, held.count, s & 31);
    u.keys = __shfl_sync(0xffffffffu, held.own, s & 31);
    u.rows = u.count * p.group;
    u.tiles = tiles_of(SeqSpan{u.first, u.count, u.keys});
  }
  // The unit of place t, which is below total().
  __device__ Unit find(int64_t t) {
    Unit u;
    if (part == kPrefix) {
      u.s = -1;
      u.first = 0;
      u.count = p.b.n_tokens;
      u.rows = p.b.n_tokens * p.group;
      u.keys = p.b.prefix_len;
      u.tiles = (p.b.prefix_len + kTile - 1) / kTile;
      u.h = (int)((uint32_t)t / (uint32_t)places_of(u.tiles));   // (kv_heads times the places of a head: below 2^31, as below)
      u.a = (int64_t)u.h * places_of(u.tiles);
      return u;
    }
    int64_t before = 0;
    for (int s0 = 0; s0 < p.b.n_seqs; s0 += 32) {
      const int lane = threadIdx.x & 31;
      hold(s0);
      const int64_t n = (int64_t)places_of(tiles_of(held)) * p.kv_heads;
      int64_t end = n;
      for (int d = 1; d < 32 && s0 + d < p.b.n_seqs; d <<= 1) {
        const int64_t o = __shfl_up_sync(0xffffffffu, end, d);
        if (lane >= d) end += o;
      }
      const uint32_t past = __ballot_sync(0xffffffffu, before + end > t);
      if (past) {
        const int l = __ffs(past) - 1;
        const int64_t a = before + __shfl_sync(0xffffffffu, end - n, l);
        enter(u, s0 + l);
        // (a sequence's keys of all heads are fewer than 2^31: check_batch)
        u.h = (int)((uint32_t)(t - a) / (uint32_t)places_of(u.tiles));
        u.a = a + (int64_t)u.h * places_of(u.tiles);
        return u;
      }
      before += __shfl_sync(0xffffffffu, end, 31);
    }
    enter(u, 0);   // (not reached)
    u.h = 0;
    u.a = t;
    return u;
  }
  // The next unit with tiles (there is one).
  __device__ void next(Unit& u) {
    u.a += places_of(u.tiles);
    if (++u.h < p.kv_heads || part == kPrefix) return;
    u.h = 0;
    for (int s = u.s + 1; s < p.b.n_seqs; ++s) {
      enter(u, s);
      if (u.tiles > 0) return;
    }
  }
};

// How the line is cut: `early` thread blocks whose warps take `ahead` places
// more than the others' (AttendParams), all of it if that is enough.
struct Shares {
  int64_t big, small, split;   // places a warp of the first `early` thread blocks, of the others; where the others begin
  int early;
  __device__ Shares(const AttendParams& p, int part, int64_t total, int blocks) {
    early = part == kOwn ? min(p.early, blocks) : 0;
    const int64_t first = (int64_t)early * kWarps, warps = (int64_t)blocks * kWarps, more = first * p.ahead;
    if (early > 0 && total <= more) {
      big = max((int64_t)1, quotient(total + first - 1, first));
      small = 0;
    } else {
      small = max(kMinShare, quotient(total - (early > 0 ? more : 0) + warps - 1, warps));
      big = small + (early > 0 ? p.ahead : 0);
    }
    split = first * big;
  }
  __device__ int64_t begin(int block) const {
    return block <= early ? (int64_t)block * kWarps * big : split + (int64_t)(block - early) * kWarps * small;
  }
  __device__ int64_t of(int block) const { return block < early ? big : small; }
  __device__ int block_of(int64_t place) const {
    return (int)(place < split || small == 0 ? quotient(place, kWarps * big) : early + quotient(place - split, kWarps * small));
  }
};

// Where an output element of a piece stands: row r, column d of kRows x D fp32,
// the 16-byte chunks of a row permuted so that the fragments' scattered
// stores meet no bank twice.
template <int D>
__device__ __forceinline__ int piece_at(int r, int d) {
  return r * D + 4 * ((d >> 2) ^ (2 * ((r >> 1) & 3))) + (d & 3);
}

// Pieces e of a thread block: 2 w the unit that warp w's share ends, 2 w + 1
// the last of its share, 2 kWarps + w a whole unit of it (8 rows at a time).
// open: the units that lie in other thread blocks too, the one from before
// (0) and the one that goes on (1).
constexpr int kPieces = 3 * kWarps;
template <int NT> struct Pieces {
  float m[kPieces][8 * NT], l[kPieces][8 * NT];
  Unit open[2];
  int is_open[2];
};

// What is joined: pieces e0 .. e1 - 1 of this thread block, or parts first ..
// first + n - 1 that thread blocks left in the workspace (e1 == 0).
struct Source {
  int e0, e1;
  int first, n;
};

// Adds n pieces to acc and sum: B pieces' loads under way at once.  ml_of(i):
// maximum and sum, at(i): the row (16-byte chunk c, permuted by `flip`), kFar:
// in global memory, read past the L1 (an overlapping grid's lines may be in it).
template <int K, int B, bool kFar, class Ml, class At>
__device__ __forceinline__ void add_pieces(int n, Ml ml_of, At at, int c, int flip, float top, float4 (&acc)[K], float& sum) {
#pragma unroll 1
  for (int i0 = 0; i0 < n; i0 += B) {
    float f[B];
    float4 v[B][K];
#pragma unroll
    for (int j = 0; j < B; ++j) {
      const int i = min(i0 + j, n - 1);
      const float2 ml = ml_of(i);
      f[j] = i0 + j < n ? exp2_approx(ml.x - top) : 0.f;   // (0 for a piece that saw nothing)
      sum += f[j] > 0.f ? ml.y * f[j] : f[j];
      const float4* from = reinterpret_cast<const float4*>(at(i));
#pragma unroll
      for (int k = 0; k < K; ++k) v[j][k] = kFar ? __ldcg(from + ((c + 4 * k) ^ flip)) : from[(c + 4 * k) ^ flip];
    }
#pragma unroll
    for (int j = 0; j < B; ++j)
#pragma unroll
      for (int k = 0; k < K; ++k)
        if (f[j] != 0.f) {   // (a piece that saw nothing holds anything)
          acc[k].x += f[j] * v[j][k].x;
          acc[k].y += f[j] * v[j][k].y;
          acc[k].z += f[j] * v[j][k].z;
          acc[k].w += f[j] * v[j][k].w;
        }
  }
}

// Rows 8 n .. 8 n + 7 of unit u: the sum of a source's pieces, in the order of
// the keys, written to `out`, or kept for the join with the call's other part;
// or (slot >= 0) kept as part `slot` of the thread blocks' parts.  A warp: 4
// lanes a row, lane c of them 16-byte chunks c, c + 4, ...; K of the D / 16
// chunk groups from k0 on.  (Inlined: as a function of its own, calls cost 15000
// cycles each.)
template <int D, int NT, int K>
__device__ __forceinline__ void finish(const AttendParams& p, const Pieces<NT>& pc, const uint8_t* smem, int part, const Unit& u, int n,
                                    Source src, int64_t slot, int k0) {
  using S = NarrowShape<D, NT>;
  constexpr int R = S::kRows, B = K == 1 ? 4 : 1;   // (4 for K = 8: more code, and up to 3 us more)
  const int lane = threadIdx.x & 31, r = 8 * n + (lane >> 2), c = (lane & 3) + 4 * k0;
  if (r >= u.rows) return;
  const int x = 2 * ((r >> 1) & 3);   // (piece_at)
  // pieces of this thread block: the odd ones in the warps' rings, then at most
  // one that ends its unit (even, in the workspace); or a whole unit's scratch
  const bool whole = src.e0 >= 2 * kWarps;
  const int e0 = whole ? src.e0 : src.e0 | 1, near = whole ? 1 : (src.e1 - e0 + 1) >> 1, step = whole ? 0 : 2;
  const int far = !whole && src.e1 > 0 && (src.e1 & 1) ? src.e1 - 1 : -1;
  const float* near_o = whole ? reinterpret_cast<const float*>(smem + kWarps * S::kRing + (e0 - 2 * kWarps) * S::kScratch) + (r & 7) * D
                              : reinterpret_cast<const float*>(smem + (e0 >> 1) * S::kRing) + r * D;
  const float* far_o = p.warp_o[part] + (((int64_t)blockIdx.x * kWarps + (far >> 1)) * R + r) * D;
  // parts of thread blocks: where the unit began, then continued
  const float2* block_ml = p.block_ml[part] + 2 * (int64_t)src.first * R + r;
  const float* block_o = p.block_o[part] + (2 * (int64_t)src.first * R + r) * D;
  auto near_ml = [&](int i) { return make_float2(pc.m[e0 + step * i][r], pc.l[e0 + step * i][r]); };
  auto far_ml = [&](int) { return make_float2(pc.m[far][r], pc.l[far][r]); };
  auto block_of = [&](int i) { return (int64_t)(2 * i + (i == 0)) * R; };
  auto part_ml = [&](int i) { return __ldcg(block_ml + block_of(i)); };
  float top = -INFINITY;
#pragma unroll 4
  for (int i = 0; i < near; ++i) top = fmaxf(top, near_ml(i).x);
  if (far >= 0) top = fmaxf(top, far_ml(0).x);
#pragma unroll 1
  for (int i0 = 0; i0 < src.n; i0 += 8) {
    float2 ml[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) ml[j] = part_ml(min(i0 + j, src.n - 1));
#pragma unroll
    for (int j = 0; j < 8; ++j) top = fmaxf(top, ml[j].x);
  }
  const float base = top == -INFINITY ? 0.f : top;
  float4 acc[K];
#pragma unroll
  for (int k = 0; k < K; ++k) acc[k] = make_float4(0.f, 0.f, 0.f, 0.f);
  float sum = 0.f;
  add_pieces<K, B, false>(near, near_ml, [&](int i) { return near_o + (step / 2) * i * (S::kRing / 4); }, c, x, base, acc, sum);
  if (far >= 0) add_pieces<K, 1, true>(1, far_ml, [&](int) { return far_o; }, c, x, base, acc, sum);
  add_pieces<K, B, true>(src.n, part_ml, [&](int i) { return block_o + block_of(i) * D; }, c, x, base, acc, sum);
  const int tok = token_of(p, r);
  const int64_t row = (int64_t)(u.first + tok) * p.q_heads + u.h * p.group + r - tok * p.group;
  const bool first = (lane & 3) == 0 && k0 == 0;
  if (slot >= 0 || p.parts > 1) {
    float* dst = slot >= 0 ? p.block_o[part] + (slot * R + r) * D : p.o[part] + row * D;
    const int flip = slot >= 0 ? x : 0;
#pragma unroll
    for (int k = 0; k < K; ++k) *reinterpret_cast<float4*>(dst + 4 * ((c + 4 * k) ^ flip)) = acc[k];
    if (first) *(slot >= 0 ? p.block_ml[part] + slot * R + r : p.ml[part] + row) = make_float2(sum == sum ? top : sum, sum);
    return;
  }
  const float inv = sum > 0.f ? 1.f / sum : sum;   // (0 where nothing is seen; NaN stays)
#pragma unroll
  for (int k = 0; k < K; ++k)
    *reinterpret_cast<uint2*>(p.out + row * D + 4 * (c + 4 * k)) =
        make_uint2(pack_bf16x2(acc[k].x * inv, acc[k].y * inv), pack_bf16x2(acc[k].z * inv, acc[k].w * inv));
  if (p.lse && first) p.lse[row] = natural_lse(top, sum);
}

template <int D, int NT, bool kWindow>
__global__ void __launch_bounds__(kThreads, 1)
    narrow_kernel(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap,
                  const __grid_constant__ AttendParams p, const int part, const int late) {
  using S = NarrowShape<D, NT>;
  constexpr int R = S::kRows, ST = S::kStages, kHalf = kTile * 128;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t full[kWarps][ST];
  __shared__ Pieces<NT> pc;
  __shared__ uint32_t arrived[2];
  __shared__ AttendParams sp;
  constexpr bool kShared = kWindow && NT >= 3;   // (the accumulators leave no registers for the lines: 74 us with them there, not 72)
  __shared__ UnitLine lines[kShared ? kWarps : 1][2];
  const int tid = threadIdx.x, warp = warp_index(), lane = tid & 31;
  const uint32_t sbase = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* smem = smem_raw + (sbase - smem_u32(smem_raw));
  if (tid < kWarps * ST) {
    mbar_init(&full[tid / ST][tid % ST], 1);
    fence_mbar_init();
  }
  if (tid < 2) pc.is_open[tid] = 0;
  static_assert(sizeof(AttendParams) % 4 == 0 && sizeof(AttendParams) / 4 <= kThreads, "copied a word per thread");
  if (tid < (int)(sizeof(AttendParams) / 4)) reinterpret_cast<uint32_t*>(&sp)[tid] = reinterpret_cast<const uint32_t*>(&p)[tid];
  __syncthreads();
  // late: the kernel ahead is this call's own on the prefix, which started
  // once everything before it was complete and shares no memory with this one;
  // it is waited for at the end, so that what follows this kernel follows both
  if (!late) pdl_wait();
  pdl_launch_dependents();
  call_record_start(p.rec, p.call, blockIdx.x == 0 && tid == 0);
  Walk<kWindow> walk(p, part);
  const int64_t total = walk.total();
  const Shares shares(p, part, total, gridDim.x);
  const int64_t share = shares.of(blockIdx.x), ct0 = shares.begin(blockIdx.x), ct1 = min(total, ct0 + kWarps * share);
  const int64_t t0 = ct0 + warp * share, t1 = min(total, t0 + share);
  uint8_t* ring = smem + warp * S::kRing;
  const uint32_t ring_a = sbase + warp * S::kRing;
  float* scratch = reinterpret_cast<float*>(smem + kWarps * S::kRing + warp * S::kScratch);
  bool ok = true;
  Unit head, tail;   // units whose pieces this warp joins: one that ends here, one that goes on behind this share
  bool head_set = false, tail_set = false;
  if (t0 < t1) {
    Unit u = walk.find(t0), ui = u;
    // (a unit that lies in several thread blocks: its ticket gets this call's tag ahead of the arrivals)
    if (warp == 0 && lane == 0 && u.a < ct0) ticket_install(p.tickets[part] + (part == kPrefix ? u.h : (int64_t)u.s * p.kv_heads + u.h), p.call);
    // ---- copies: tile ti of unit ui is the next, if it is one of this share's; `page` of tile pb + lane of sequence ps
    int ti = (int)(t0 - u.a), ki = 0, pb = 0, ps = -2, page = -1;
    UnitLine line_r[2];      // with a window: of u, of ui
    const volatile UnitLine &line = kShared ? lines[warp][0] : line_r[0], &line_i = kShared ? lines[warp][1] : line_r[1];
    auto set_line = [&](int which, const Unit& unit) {
      if (!kShared) {
        line_r[which] = unit_line(p, unit.count, unit.keys);
        return;
      }
      __syncwarp();
      if (lane == 0) lines[warp][which] = unit_line(p, unit.count, unit.keys);
      __syncwarp();
    };
    if (kWindow) set_line(1, ui);
    const int per_page = p.page_shift - 4;   // log2 of tiles per page
    auto issue = [&]() {
      if (ti >= ui.tiles) {
        if (ui.a + walk.places_of(ui.tiles) >= t1) return;
        walk.next(ui);
        ti = 0;
        if (kWindow) set_line(1, ui);
      }
      if (ui.a + ti >= t1) return;
      if (ui.s != ps || ti < pb || ti >= pb + 32) {
        ps = ui.s;
        pb = ti;
        const int32_t* table = part == kPrefix || (kWindow && line_i.in_prefix(ti + lane)) ? p.b.prefix_pages
                                                                                           : p.b.pages + (int64_t)ui.s * p.b.page_stride;
        page = ti + lane < ui.tiles ? __ldg(table + ((kWindow ? line_i.tile(ti + lane) : ti + lane) >> per_page)) : -1;
      }
      const int pg = __shfl_sync(0xffffffffu, page, ti - pb), tile = kWindow ? line_i.tile(ti) : ti;
      // (a page outside the cache: rows outside the arrays, which read as zeros)
      const int y = pg >= 0 && pg < p.n_pages ? ((pg * p.kv_heads + ui.h) << p.page_shift) + ((tile & ((1 << per_page) - 1)) << 4) : -kTile;
      const int st = ki % ST;
      const uint32_t bar = smem_u32(&full[warp][st]), dst = ring_a + st * 2 * S::kMat;
      mbar_expect_tx_warp(&full[warp][st], 2 * S::kMat);
      tma_load_3d_warp(dst, &kmap, 0, y, 0, bar);
      tma_load_3d_warp(dst + S::kMat, &vmap, 0, y, 0, bar);
      ++ti;
      ++ki;
    };
#pragma unroll 1
    for (int i = 0; i < ST; ++i) issue();
    const int g8 = lane >> 2, c2 = 2 * (lane & 3);
    int k = 0;
    for (; u.a < t1; walk.next(u)) {
      const int lo = (int)(max(u.a, t0) - u.a), hi = (int)min((int64_t)u.tiles, t1 - u.a);
      if (lo < hi) {
      // query rows as the products' B operand; rows past the last are zero
      uint32_t qf[NT][D / 16][2];
      int lim[NT][2];   // keys that this lane's two queries of each 8 see
      if (kWindow) set_line(0, u);
      float o[NT][D / 16][4], m[NT][2], l[NT][2];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const int r = 8 * n + g8, tok = token_of(p, r);
        const uint16_t* src = p.q + (int64_t)(u.first + tok) * p.ldq + (int64_t)(u.h * p.group + r - tok * p.group) * D + c2;
#pragma unroll
        for (int d = 0; d < D / 16; ++d)
#pragma unroll
          for (int j = 0; j < 2; ++j) qf[n][d][j] = r < u.rows ? __ldg(reinterpret_cast<const uint32_t*>(src + 16 * d + 8 * j)) : 0u;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int rj = 8 * n + c2 + j;
          lim[n][j] = part == kPrefix || rj >= u.rows ? u.keys : u.keys - u.count + token_of(p, rj) + 1;
          m[n][j] = -INFINITY;
          l[n][j] = 0.f;
        }
#pragma unroll
        for (int d = 0; d < D / 16; ++d)
#pragma unroll
          for (int j = 0; j < 4; ++j) o[n][d][j] = 0.f;
      }
      const int seen_own = part == kPrefix ? u.keys : u.keys - u.count + 1;   // by every row
      const int low_all = kWindow ? position_of(p, u.keys - 1) - p.window + 1 : 0;   // the first position that every row's window has
      for (int i = lo; i < hi; ++i, ++k) {
        // tile t of the unit's keys (of the prefix's or its own), of which there are `end`
        const bool pre = kWindow && line.in_prefix(i);
        const int t = kWindow ? line.tile(i) : i, end = pre ? p.b.prefix_len : u.keys, seen = pre ? end : seen_own;
        const int base = kWindow && !pre ? p.b.prefix_len : 0;      // position of the first
        // with a window: keys from `sinks` up to `low_all - base` are not every row's
        const int sinks = p.sinks - base;
        const bool low_edge = kWindow && t * kTile < low_all - base && (t + 1) * kTile > sinks;
        auto sees = [&](int n, int j, int key) {
          return key < (pre ? end : lim[n][j]) && (!kWindow || key >= position_of(p, lim[n][j] - 1) - p.window + 1 - base || key < sinks);
        };
        const int st = k % ST;
        ok = mbar_wait_warp(&full[warp][st], (k / ST) & 1);
        if (!ok) break;
        const uint32_t kb = ring_a + st * 2 * S::kMat, vb = kb + S::kMat;
        const bool edge = (t + 1) * kTile > seen || low_edge;
        // values from key `from` of the tile's on: zero times them has to be zero
        auto drop = [&](int from) {
#pragma unroll 1
          for (int i = lane; i < kTile * (D / 8); i += 32) {
            const int r = i / (D / 8), c = i % (D / 8);
            if (t * kTile + r >= from) st_shared16(vb + (c >> 3) * kHalf + r * 128 + ((c & 7) << 4), 0, 0, 0, 0);
          }
          fence_proxy_async_smem();   // (before the next copy into this stage)
          __syncwarp();
        };
        bool apart = false;   // a token's value that is not finite, and tokens before it
        if (edge) {
          if ((t + 1) * kTile > end) drop(end);   // past the last key: leftovers (perhaps NaN)
          if (seen < end || low_edge) {
            bool bad = false;
#pragma unroll 1
            for (int i = lane; i < kTile * (D / 8); i += 32) {
              const int r = i / (D / 8), c = i % (D / 8);
              const uint4 v = ld_shared16(vb + (c >> 3) * kHalf + r * 128 + ((c & 7) << 4));
              if (t * kTile + r >= seen || (low_edge && t * kTile + r < low_all - base && t * kTile + r >= sinks)) bad |= some_not_finite(v);
            }
            apart = __any_sync(0xffffffffu, bad);
          }
        }
        float s[NT][2][4];   // even and odd 16 elements, so that the chain of sums is half as long
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int j = 0; j < 4; ++j) s[n][0][j] = s[n][1][j] = 0.f;
        const uint32_t krow = kb + (uint32_t)((lane & 15) * 128), kx = lane & 7, kc = lane >> 4;
#pragma unroll
        for (int d = 0; d < D / 16; ++d) {
          uint32_t a[4];
          const uint32_t c = 2 * d + kc;
          ldmatrix4(a, krow + (c >> 3) * kHalf + (((c & 7) ^ kx) << 4));
#pragma unroll
          for (int n = 0; n < NT; ++n) mma_bf16_16816(s[n][d & 1], a, qf[n][d][0], qf[n][d][1]);
        }
        const int key = t * kTile + g8;   // and key + 8
        uint32_t hidden = 0;   // with a window: which scores are left out (a bit each; worked out behind a branch)
        if (kWindow && edge) {
#pragma unroll
          for (int b = 0; b < 4 * NT; ++b)
            if (!sees(b >> 2, b & 1, key + 8 * (b >> 1 & 1))) hidden |= 1u << b;
        }
        uint32_t pf[NT][2];
        if (kWindow) {
          // The reference of a query's weights is raised only where its maximum
          // passes it by more than 2^8, and then set kAhead above it (weights and
          // sums are floating: nothing is lost by a reference that lies higher);
          // one look for all queries.  (Raised with every larger score, as below, one of 24
          // queries' was on almost every tile: 2 x 3 tokens, window 32768, 77 us, not 74.)
          constexpr float kRaise = 8.f, kAhead = 12.f;
          float x[NT][4], mx[NT][2];
          bool grow = false;
#pragma unroll
          for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              x[n][j] = (s[n][0][j] + s[n][1][j]) * p.scale;
              if (hidden >> (4 * n + j) & 1u) x[n][j] = -INFINITY;
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              mx[n][j] = fmaxf(x[n][j], x[n][j + 2]);
              grow |= mx[n][j] > m[n][j] + kRaise;   // (also from -inf)
            }
          }
          if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              float f[2];
#pragma unroll
              for (int j = 0; j < 2; ++j) {
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) mx[n][j] = fmaxf(mx[n][j], __shfl_xor_sync(0xffffffffu, mx[n][j], d));
                const bool raise = mx[n][j] > m[n][j] + kRaise;
                f[j] = raise ? exp2_approx(m[n][j] - (mx[n][j] + kAhead)) : 1.f;
                if (raise) m[n][j] = mx[n][j] + kAhead;
                l[n][j] *= f[j];
              }
#pragma unroll
              for (int d = 0; d < D / 16; ++d)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[n][d][j] *= f[j & 1];
            }
          }
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            float e[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              e[j] = exp2_approx(x[n][j] - (m[n][j & 1] == -INFINITY ? 0.f : m[n][j & 1]));
              l[n][j & 1] += e[j];
            }
            pf[n][0] = movmatrix(pack_bf16x2(e[0], e[1]));
            pf[n][1] = movmatrix(pack_bf16x2(e[2], e[3]));
          }
        }
#pragma unroll
        for (int n = 0; n < (kWindow ? 0 : NT); ++n) {
          float x[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            x[j] = (s[n][0][j] + s[n][1][j]) * p.scale;
            if (edge && key + 8 * (j >> 1) >= lim[n][j & 1]) x[j] = -INFINITY;
          }
          float mx[2];
#pragma unroll
          for (int j = 0; j < 2; ++j) mx[j] = fmaxf(x[j], x[j + 2]);
          // a query's maximum grows less and less often: looked for across the
          // lanes only where some lane has a larger one
          if (__any_sync(0xffffffffu, mx[0] > m[n][0] || mx[1] > m[n][1])) {
            float f[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
#pragma unroll
              for (int d = 4; d < 32; d <<= 1) mx[j] = fmaxf(mx[j], __shfl_xor_sync(0xffffffffu, mx[j], d));
              mx[j] = fmaxf(mx[j], m[n][j]);
              f[j] = mx[j] == -INFINITY ? 1.f : exp2_approx(m[n][j] - mx[j]);
              m[n][j] = mx[j];
              l[n][j] *= f[j];
            }
#pragma unroll
            for (int d = 0; d < D / 16; ++d)
#pragma unroll
              for (int j = 0; j < 4; ++j) o[n][d][j] *= f[j & 1];
          }
          float e[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            e[j] = exp2_approx(x[j] - (m[n][j & 1] == -INFINITY ? 0.f : m[n][j & 1]));
            l[n][j & 1] += e[j];
          }
          pf[n][0] = movmatrix(pack_bf16x2(e[0], e[1]));
          pf[n][1] = movmatrix(pack_bf16x2(e[2], e[3]));
        }
        const uint32_t vr = ((lane >> 4) << 3) + (lane & 7), vc = (lane >> 3) & 1;
        if (kWindow && apart) {
          // what the tokens see is not a part of what the next one sees: values
          // that are not finite and not every row's go to the rows that see them
          // by an addition, and out of the tile
          auto shared = [&](int kk) { return kk < seen && (kk >= low_all - base || kk < sinks); };
#pragma unroll 1
          for (int r = 0; r < kTile; ++r) {
            const int kk = t * kTile + r;
            if (kk >= end || shared(kk)) continue;
#pragma unroll
            for (int d = 0; d < D / 16; ++d)
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const int c = 2 * d + h;   // 8 elements, of which this lane has number g8
                const uint8_t* at = ring + (vb - ring_a) + (c >> 3) * kHalf + r * 128 + (((c & 7) ^ (r & 7)) << 4) + 2 * g8;
                const uint32_t bits = *reinterpret_cast<const volatile uint16_t*>(at);
                if (!not_finite(bits)) continue;
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                  for (int j = 0; j < 2; ++j)
                    if (sees(n, j, kk)) o[n][d][2 * h + j] += __uint_as_float(bits << 16);
              }
          }
          __syncwarp();
#pragma unroll 1
          for (int i16 = lane; i16 < kTile * (D / 8); i16 += 32) {
            const int r = i16 / (D / 8), c = i16 % (D / 8), kk = t * kTile + r;
            const uint32_t at = vb + (c >> 3) * kHalf + r * 128 + ((c & 7) << 4);
            const uint4 v = ld_shared16(at);
            if (kk < end && !shared(kk) && some_not_finite(v))
              st_shared16(at, v.x & ~not_finite(v.x), v.y & ~not_finite(v.y), v.z & ~not_finite(v.z), v.w & ~not_finite(v.w));
          }
          fence_proxy_async_smem();   // (before the next copy into this stage)
          __syncwarp();
        }
        if (kWindow || !apart) {
#pragma unroll
          for (int d = 0; d < D / 16; ++d) {
            uint32_t a[4];
            const uint32_t c = 2 * d + vc;
            ldmatrix4_trans(a, vb + (c >> 3) * kHalf + vr * 128 + (((c & 7) ^ (vr & 7)) << 4));
#pragma unroll
            for (int n = 0; n < NT; ++n) mma_bf16_16816(o[n][d], a, pf[n][0], pf[n][1]);
          }
          __syncwarp();   // every lane has read the stage
        } else {
          // token by token, the last first, each without the values that it does not see
#pragma unroll 1
          for (int i = u.count - 1; i >= 0; --i) {
            drop(u.keys - u.count + i + 1);
#pragma unroll
            for (int d = 0; d < D / 16; ++d) {
              uint32_t a[4];
              const uint32_t c = 2 * d + vc;
              ldmatrix4_trans(a, vb + (c >> 3) * kHalf + vr * 128 + (((c & 7) ^ (vr & 7)) << 4));
#pragma unroll
              for (int n = 0; n < NT; ++n) {
                float x[4] = {o[n][d][0], o[n][d][1], o[n][d][2], o[n][d][3]};
                mma_bf16_16816(x, a, pf[n][0], pf[n][1]);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                  if (token_of(p, 8 * n + c2 + (j & 1)) == i) o[n][d][j] = x[j];
              }
            }
            __syncwarp();
          }
        }
        issue();
      }
      if (!ok) break;
      // ---- the end of the unit, or of the share
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) l[n][j] += __shfl_xor_sync(0xffffffffu, l[n][j], d);
      const bool starts = lo == 0, ends = hi == u.tiles;
      const bool whole = starts && ends;
      if (whole && p.parts == 1) {
        // a whole unit, nothing to join: O^T is turned by movmatrix as P was, a row's 4 lanes write 16 bytes at a time
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float inv[2];
#pragma unroll
          for (int j = 0; j < 2; ++j) inv[j] = l[n][j] > 0.f ? 1.f / l[n][j] : l[n][j];   // (0 where nothing is seen; NaN stays)
          const int r = 8 * n + g8, tok = token_of(p, r);
          const int64_t row = (int64_t)(u.first + tok) * p.q_heads + u.h * p.group + r - tok * p.group;
#pragma unroll
          for (int d = 0; d < D / 16; ++d)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              const uint32_t v = movmatrix(pack_bf16x2(o[n][d][2 * j] * inv[0], o[n][d][2 * j + 1] * inv[1]));
              if (r < u.rows) *reinterpret_cast<uint32_t*>(p.out + row * D + 16 * d + 8 * j + c2) = v;
            }
          if (p.lse && g8 == 0)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              const int rj = 8 * n + c2 + j, tj = token_of(p, rj);
              if (rj < u.rows)
                p.lse[(int64_t)(u.first + tj) * p.q_heads + u.h * p.group + rj - tj * p.group] = natural_lse(m[n][j], l[n][j]);
            }
        }
        continue;
      }
      // a whole unit leaves 8 rows at a time through the scratch; a piece of the
      // unit that ends here goes into the workspace (the ring is in use), the
      // last one into the ring, whose copies are all read
      const int e = whole ? 2 * kWarps + warp : 2 * warp + (ends ? 0 : 1);
      float* dst = whole  ? scratch
                   : ends ? p.warp_o[part] + ((int64_t)blockIdx.x * kWarps + warp) * (R * D)
                          : reinterpret_cast<float*>(ring);
      __syncwarp();
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const int at = whole ? 0 : 8 * n;
#pragma unroll
        for (int d = 0; d < D / 16; ++d)
#pragma unroll
          for (int j = 0; j < 4; ++j) dst[piece_at<D>(at + c2 + (j & 1), 16 * d + 8 * (j >> 1) + g8)] = o[n][d][j];
        if (g8 == 0) {
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            pc.m[e][8 * n + c2 + j] = l[n][j] == l[n][j] ? m[n][j] : l[n][j];   // (NaN scores leave no maximum)
            pc.l[e][8 * n + c2 + j] = l[n][j];
          }
        }
        if (whole) {
          __syncwarp();
          finish<D, NT, D / 16>(sp, pc, smem, part, u, n, Source{e, e + 1, 0, 0}, -1, 0);
          __syncwarp();
        }
      }
      if (!whole) {
        // the first warp of the thread block that has pieces of the unit joins them below
        if (ends) {
          if (warp == 0) head = u;
          head_set = warp == 0;
        } else if (starts || warp == 0) {
          tail = u;
          tail_set = true;
        }
      }
      }
    }
    // the copies in flight have landed before the thread block ends
    if (!ok)
      for (int i = max(0, ki - ST); i < ki; ++i) mbar_wait_warp(&full[warp][i % ST], (i / ST) & 1);
  }
  // ---- pieces of this thread block
  const bool all_ok = __syncthreads_and(ok);
  if (all_ok) {
    // the units with pieces here, each by one warp.  Those that lie in other
    // thread blocks too are kept as parts
    if (head_set)
      for (int n = 0; n < NT; ++n) finish<D, NT, D / 16>(sp, pc, smem, part, head, n, Source{0, 1, 0, 0}, 2 * (int64_t)blockIdx.x, 0);
    if (tail_set) {
      const bool before = tail.a < ct0, after = tail.a + tail.tiles > ct1;
      int last = warp;   // the last warp with tiles of it
      while (last + 1 < kWarps && ct0 + (last + 1) * share < tail.a + tail.tiles) ++last;
      const Source src{2 * warp + 1, after ? 2 * kWarps : 2 * last + 1, 0, 0};
      const int64_t slot = before || after ? 2 * (int64_t)blockIdx.x + (before ? 0 : 1) : -1;
      for (int n = 0; n < NT; ++n) finish<D, NT, D / 16>(sp, pc, smem, part, tail, n, src, slot, 0);
      if (slot >= 0 && lane == 0) {
        pc.open[before ? 0 : 1] = tail;
        pc.is_open[before ? 0 : 1] = 1;
      }
    }
    if (head_set && lane == 0) {
      pc.open[0] = head;
      pc.is_open[0] = 1;
    }
    __syncthreads();
    if (pc.is_open[0] | pc.is_open[1]) {
      if (tid < 2) {
        arrived[tid] = 0;
        if (pc.is_open[tid]) {
          const Unit& u = pc.open[tid];
          const uint32_t n = (uint32_t)(shares.block_of(u.a + u.tiles - 1) - shares.block_of(u.a) + 1);
          uint64_t* tk = p.tickets[part] + (part == kPrefix ? u.h : (int64_t)u.s * p.kv_heads + u.h);
          const uint32_t got = ticket_take(tk, p.call, n);
          if (got == 0) call_record_fail(p.rec, p.call);
          arrived[tid] = got == n;
        }
      }
      __syncthreads();
      for (int i = 0; i < 2; ++i) {
        if (!arrived[i]) continue;
        // the last to arrive: all thread blocks' parts, a chunk group a warp
        const Unit& u = pc.open[i];
        const int first = shares.block_of(u.a), n = shares.block_of(u.a + u.tiles - 1) - first + 1;
        constexpr int kPer = kWarps / (D / 16);   // warps on a chunk group, each of its own rows
        for (int m = warp % kPer; m < NT; m += kPer)
          finish<D, NT, 1>(sp, pc, smem, part, u, m, Source{0, 0, first, n}, -1, warp / kPer);
      }
    }
    // sequences without keys of their own: 0, or nothing to join.  (Any number of
    // rows, where no sequence has keys: by tokens, whose rows are neighbours)
    if (part == kOwn)
      for (int s = blockIdx.x; s < p.b.n_seqs; s += gridDim.x) {
        const SeqSpan q = seq_span(p.b, s);
        if (q.own > 0 || (kWindow && p.b.prefix_len > 0 && !p.apart)) continue;
        const int64_t r1 = (int64_t)(q.first + q.count) * p.q_heads;
        for (int64_t row = (int64_t)q.first * p.q_heads + warp; row < r1; row += kWarps) {
          const float none[D / 32] = {};
          if (p.parts == 1) write_row<D, D / 32>(p, row, none, -INFINITY, 0.f);
          else if (lane == 0) p.ml[part][row] = make_float2(-INFINITY, 0.f);   // (the join reads no sums of it)
        }
      }
  }
  if (!ok && lane == 0) call_record_fail(p.rec, p.call);
  if (late) pdl_wait();
}

template <int D, int NT, bool kWindow>
cudaError_t launch_kernel(const sdq_cache_s* c, const AttendParams& p, int part, bool late, cudaStream_t st) {
  using S = NarrowShape<D, NT>;
  static std::atomic<int> smem_set[64];
  const cudaError_t e = smem_limit_once(narrow_kernel<D, NT, kWindow>, S::kSmem, c->device, smem_set);
  if (e != cudaSuccess) return e;
  return launch_pdl(narrow_kernel<D, NT, kWindow>, dim3((unsigned)p.ctas), dim3(kThreads), (size_t)S::kSmem, st, c->ktile, c->vtile, p, part,
                    late ? 1 : 0);
}

template <int D, int NT>
cudaError_t launch(const sdq_cache_s* c, const AttendParams& p, int part, bool late, cudaStream_t st) {
  return p.window > 0 ? launch_kernel<D, NT, true>(c, p, part, late, st) : launch_kernel<D, NT, false>(c, p, part, late, st);
}

template <int D>
cudaError_t launch_nt(const sdq_cache_s* c, const AttendParams& p, int part, bool late, cudaStream_t st) {
  switch (narrow_groups(p, part)) {
    case 0:   // (no keys: zeros)
    case 1: return launch<D, 1>(c, p, part, late, st);
    case 2: return launch<D, 2>(c, p, part, late, st);
    case 3: return launch<D, 3>(c, p, part, late, st);
    default: return launch<D, 4>(c, p, part, late, st);
  }
}

}  // namespace

int narrow_groups(const AttendParams& p, int part) {
  if (part == kPrefix ? p.b.prefix_len == 0 : p.b.max_own == 0 && (p.window == 0 || p.b.prefix_len == 0)) return 0;
  return (int)(((int64_t)(part == kPrefix ? p.b.n_tokens : p.b.max_new) * p.group + 7) / 8);
}

int narrow_warps() { return kWarps; }

cudaError_t launch_narrow(const sdq_cache_s* c, const AttendParams& p, int part, bool late, cudaStream_t st) {
  return c->desc.head_dim == 128 ? launch_nt<128>(c, p, part, late, st) : launch_nt<64>(c, p, part, late, st);
}

}  // namespace sdq
