// Attention over the paged cache: the kernel for few query rows per key head
// (single and drafted tokens), the join of partial results, and the host side
// (include/sdq.h).
#include <algorithm>
#include <cmath>

#include "attention.cuh"

namespace sdq {

namespace {

// ------------------------------------------------------------ narrow kernel
// Few query rows share a key head's keys, so HBM bounds it: every key and
// value is read once.  The work is a line of tiles of KT keys, row block by
// row block (prefix first, then sequence by sequence, head by head), cut into
// equal shares for the resident thread blocks: no share is longer than
// another by more than a tile, whatever the lengths.  A share that ends inside
// a row block leaves a partial result.
//   warp W       loads tiles, page by page, into a ring (TMA, 128-byte swizzle)
//   warps 0..W-1 each take 16 keys of every tile: S^T = K Q^T with the keys as
//                the MMA's 16 rows and 8 queries as its columns (the other
//                way round half of a 16-row tile would be padding), a running
//                maximum and sum of their own, O^T += V^T P^T; joined over
//                shared memory once per row block
// K and V fragments come by ldmatrix; P^T is turned from the accumulator's
// layout into the operand's by movmatrix.  P is rounded to bf16 for its
// product (relative 2^-8 at most per weight, as the values themselves carry); sums,
// maxima and outputs are fp32.
template <int D, int NT> struct NarrowShape {
  static constexpr int kWarps = D == 128 && NT == 1 ? 4 : 8;
  static constexpr int kThreads = 32 * (kWarps + 1);
  static constexpr int kTile = 16 * kWarps;                    // keys
  static constexpr int kRows = 8 * NT;
  static constexpr int kHalfTile = kTile * 128;                // bytes: keys x 64 elements
  static constexpr int kMat = (D / 64) * kHalfTile;            // K or V of a tile
  static constexpr int kStage = 2 * kMat;
  static constexpr int kPerSm = NT == 1 ? 2 : 1;
  static constexpr int kRing = kPerSm == 2 ? 3 : (D == 128 ? 3 : 6);
  static constexpr int kBufs = NT <= 2 ? 2 : 1;
  static constexpr int kPitch = D + 4;                         // of the join buffers, in floats
  static constexpr int kQBytes = kRows * D * 2;
  static constexpr int kSmem = 1024 + kRing * kStage + kQBytes + kBufs * kRows * kPitch * 4;
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

// A row block: up to R rows (new token major, then head of the group) of one
// key head of one sequence, or of the whole batch against the prefix.
struct Block {
  int part, s, h, rb;
  int first, rows, keys, count;   // first token, rows of all its blocks, keys, new tokens (kOwn)
  int nrb, tiles;                 // blocks of the (sequence, head), tiles of one block
  int64_t a;                      // first global tile
};

template <int R, int KT>
struct Walk {
  const AttendParams& p;
  int prefix_rb, prefix_tiles;
  int64_t prefix_total;
  __device__ explicit Walk(const AttendParams& p_) : p(p_) {
    prefix_rb = p.narrow[kPrefix] ? (p.b.n_tokens * p.group + R - 1) / R : 0;
    prefix_tiles = p.narrow[kPrefix] ? (p.b.prefix_len + KT - 1) / KT : 0;
    prefix_total = (int64_t)p.kv_heads * prefix_rb * prefix_tiles;
  }
  // Tiles of sequence s over all heads and row blocks.
  __device__ int64_t seq_tiles(int s) const {
    if (s >= p.b.n_seqs) return 0;
    const SeqSpan q = seq_span(p.b, s);
    return (int64_t)p.kv_heads * ((q.count * p.group + R - 1) / R) * ((q.own + KT - 1) / KT);
  }
  // All tiles (a whole warp).
  __device__ int64_t total() const {
    int64_t n = 0;
    if (p.narrow[kOwn])
      for (int s = threadIdx.x & 31; s < p.b.n_seqs; s += 32) n += seq_tiles(s);
    for (int d = 16; d; d >>= 1) n += __shfl_xor_sync(0xffffffffu, n, d);
    return prefix_total + n;
  }
  __device__ void enter(Block& u, int s) const {
    const SeqSpan q = seq_span(p.b, s);
    u.part = kOwn;
    u.s = s;
    u.first = q.first;
    u.count = q.count;
    u.rows = q.count * p.group;
    u.keys = q.own;
    u.nrb = (u.rows + R - 1) / R;
    u.tiles = (q.own + KT - 1) / KT;
  }
  // The row block that holds global tile t (a whole warp); writes the first
  // tile of every sequence up to there to `base` if that is not null.
  __device__ Block find(int64_t t) const {
    Block u;
    if (t < prefix_total) {
      u.part = kPrefix;
      u.s = -1;
      u.first = 0;
      u.count = p.b.n_tokens;
      u.rows = p.b.n_tokens * p.group;
      u.keys = p.b.prefix_len;
      u.nrb = prefix_rb;
      u.tiles = prefix_tiles;
      const int i = (int)(t / prefix_tiles);
      u.h = i / prefix_rb;
      u.rb = i - u.h * prefix_rb;
      u.a = (int64_t)i * prefix_tiles;
      return u;
    }
    int64_t base = prefix_total;
    for (int s0 = 0; s0 < p.b.n_seqs; s0 += 32) {
      const int lane = threadIdx.x & 31;
      const int64_t n = seq_tiles(s0 + lane);
      int64_t end = n;
      for (int d = 1; d < 32; d <<= 1) {
        const int64_t o = __shfl_up_sync(0xffffffffu, end, d);
        if (lane >= d) end += o;
      }
      const uint32_t past = __ballot_sync(0xffffffffu, base + end > t);
      if (past) {
        const int l = __ffs(past) - 1;
        const int64_t a = base + __shfl_sync(0xffffffffu, end - n, l);
        enter(u, s0 + l);
        const int64_t i = (t - a) / u.tiles;
        u.h = (int)(i / u.nrb);
        u.rb = (int)(i - (int64_t)u.h * u.nrb);
        u.a = a + i * u.tiles;
        return u;
      }
      base += __shfl_sync(0xffffffffu, end, 31);
    }
    u.tiles = 0;   // (not reached: t is below total())
    return u;
  }
  // The next row block with tiles; false at the end of the line.
  __device__ bool next(Block& u) const {
    u.a += u.tiles;
    if (++u.rb < u.nrb) return true;
    u.rb = 0;
    if (++u.h < p.kv_heads) return true;
    u.h = 0;
    if (!p.narrow[kOwn]) return false;
    for (int s = u.s + 1; s < p.b.n_seqs; ++s) {
      enter(u, s);
      if (u.tiles > 0 && u.rows > 0) return true;
    }
    return false;
  }
};

template <int D, int NT>
__global__ void __launch_bounds__(NarrowShape<D, NT>::kThreads, NarrowShape<D, NT>::kPerSm)
    narrow_kernel(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap, const AttendParams p) {
  using S = NarrowShape<D, NT>;
  constexpr int W = S::kWarps, KT = S::kTile, R = S::kRows, kCon = 32 * W;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t full[S::kRing], empty[S::kRing];
  __shared__ float row_m[W][R], row_l[W][R];
  const int tid = threadIdx.x, warp = warp_index(), lane = tid & 31;
  const uint32_t sbase = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* ring = smem_raw + (sbase - smem_u32(smem_raw));
  const uint32_t qbase = sbase + S::kRing * S::kStage;
  float* bufs = reinterpret_cast<float*>(ring + S::kRing * S::kStage + S::kQBytes);
  if (tid == 0) {
    for (int i = 0; i < S::kRing; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], W);
    }
    fence_mbar_init();
  }
  __syncthreads();
  pdl_wait();
  pdl_launch_dependents();
  call_record_start(p.rec, p.call, blockIdx.x == 0 && tid == 0);
  const Walk<R, KT> walk(p);
  const int64_t total = walk.total(), share = (total + p.ctas - 1) / p.ctas;
  if (blockIdx.x == 0 && warp == 0 && p.narrow[kOwn]) {   // for the join
    int64_t base = walk.prefix_total;
    for (int s0 = 0; s0 < p.b.n_seqs; s0 += 32) {
      const int64_t n = walk.seq_tiles(s0 + lane);
      int64_t end = n;
      for (int d = 1; d < 32; d <<= 1) {
        const int64_t o = __shfl_up_sync(0xffffffffu, end, d);
        if (lane >= d) end += o;
      }
      if (s0 + lane < p.b.n_seqs) p.base[s0 + lane] = base + end - n;
      base += __shfl_sync(0xffffffffu, end, 31);
    }
    if (lane == 0) p.base[p.b.n_seqs] = total;
  }
  const int64_t t0 = blockIdx.x * share, t1 = min(total, t0 + share);
  if (t0 >= t1) return;
  Block u = walk.find(t0);
  bool ok = true;
  uint32_t it = 0;
  if (warp == W) {
    // ------------------------------------------------------------ loads
    const int box = 1 << p.box_shift, per_page = 1 << (p.page_shift - p.box_shift);
    constexpr uint32_t kRowBytes = (D / 64) * 128 * 2;   // of a key and its value
    do {
      const int lo = (int)(max(u.a, t0) - u.a), hi = (int)(min(u.a + u.tiles, t1) - u.a);
      const int32_t* table = u.part == kPrefix ? p.b.prefix_pages : p.b.pages + (int64_t)u.s * p.b.page_stride;
      const int boxes = (u.keys + box - 1) >> p.box_shift;          // of the whole table
      int at = lo * (KT >> p.box_shift), held = at;                  // box index; first box whose page a lane holds
      int page = at + lane < boxes ? __ldg(table + (at + lane) / per_page) : -1;
      for (int t = lo; t < hi && ok; ++t, ++it) {
        const int st = it % S::kRing, r = it / S::kRing;
        const int n = min(KT >> p.box_shift, boxes - at);
        if (r > 0) ok = mbar_wait_warp(&empty[st], (r - 1) & 1);
        if (!ok) break;
        mbar_expect_tx_warp(&full[st], (uint32_t)(n << p.box_shift) * kRowBytes);
        uint8_t* dst = ring + st * S::kStage;
        for (int i = 0; i < n; ++i, ++at) {
          if (at - held == 32) {
            held = at;
            page = at + lane < boxes ? __ldg(table + (at + lane) / per_page) : -1;
          }
          const int pg = __shfl_sync(0xffffffffu, page, at - held);
          // (a page outside the cache: rows outside the arrays, which read as zeros)
          const int y = pg >= 0 && pg < p.n_pages
                            ? ((pg * p.kv_heads + u.h) << p.page_shift) + ((at & (per_page - 1)) << p.box_shift)
                            : -box;
#pragma unroll
          for (int half = 0; half < D / 64; ++half) {
            tma_load_2d_warp(dst + half * S::kHalfTile + ((i * box) << 7), &kmap, 64 * half, y, &full[st]);
            tma_load_2d_warp(dst + S::kMat + half * S::kHalfTile + ((i * box) << 7), &vmap, 64 * half, y, &full[st]);
          }
        }
      }
    } while (ok && u.a + u.tiles < t1 && walk.next(u));
    // the copies in flight have landed before the thread block ends
    for (uint32_t j = it > S::kRing ? it - S::kRing : 0; j < it; ++j)
      if (!mbar_wait_warp(&full[j % S::kRing], (j / S::kRing) & 1)) ok = false;
    if (!ok && lane == 0) call_record_fail(p.rec, p.call);
    return;
  }

  // ------------------------------------------------------------ products
  const int g8 = lane >> 2, c2 = 2 * (lane & 3);
  do {
    const int lo = (int)(max(u.a, t0) - u.a), hi = (int)(min(u.a + u.tiles, t1) - u.a);
    const int r0 = u.rb * R, nrows = min(R, u.rows - r0);
    // this block's query rows (rows past them zero)
    for (int i = tid; i < R * (D / 8); i += kCon) {
      const int r = i / (D / 8), c = i % (D / 8);
      uint4 v = make_uint4(0, 0, 0, 0);
      if (r < nrows) {
        const int tok = (r0 + r) / p.group, g = r0 + r - tok * p.group;
        v = __ldg(reinterpret_cast<const uint4*>(p.q + (int64_t)(u.first + tok) * p.ldq + (int64_t)(u.h * p.group + g) * D) + c);
      }
      const uint32_t a = qbase + (uint32_t)((c >> 3) * (R * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4));
      asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};\n" ::"r"(a), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
    }
    // keys that this lane's two queries of each 8 see
    int lim[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int r = r0 + 8 * n + c2 + j;
        lim[n][j] = u.part == kPrefix || r >= u.rows ? u.keys : u.keys - u.count + r / p.group + 1;
      }
    const int seen = u.part == kPrefix ? u.keys : u.keys - u.count + r0 / p.group + 1;   // by every row of the block
    float o[NT][D / 16][4], m[NT][2], l[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        m[n][j] = -INFINITY;
        l[n][j] = 0.f;
      }
#pragma unroll
      for (int d = 0; d < D / 16; ++d)
#pragma unroll
        for (int j = 0; j < 4; ++j) o[n][d][j] = 0.f;
    }
    named_bar_sync(1, kCon);
    uint32_t qf[NT == 1 ? D / 32 : 1][4];
    const uint32_t qrow = qbase + (uint32_t)((lane & 7) * 128), qx = lane & 7, qc = lane >> 3;
    if (NT == 1) {
#pragma unroll
      for (int k = 0; k < D / 32; ++k) {
        const uint32_t c = 4 * k + qc;
        ldmatrix4(qf[k], qrow + (c >> 3) * (R * 128) + (((c & 7) ^ qx) << 4));
      }
    }
    for (int t = lo; t < hi && ok; ++t, ++it) {
      const int st = it % S::kRing;
      ok = mbar_wait_warp(&full[st], (it / S::kRing) & 1);
      if (!ok) break;
      const uint32_t kb = sbase + st * S::kStage, vb = kb + S::kMat;
      float s[NT][4];
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[n][j] = 0.f;
      const uint32_t krow = kb + (uint32_t)((16 * warp + (lane & 15)) * 128), kx = lane & 7, kc = lane >> 4;
#pragma unroll
      for (int k = 0; k < D / 32; ++k) {
        uint32_t a0[4], a1[4];
        const uint32_t ca = 4 * k + kc, cb = 4 * k + 2 + kc;
        ldmatrix4(a0, krow + (ca >> 3) * S::kHalfTile + (((ca & 7) ^ kx) << 4));
        ldmatrix4(a1, krow + (cb >> 3) * S::kHalfTile + (((cb & 7) ^ kx) << 4));
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          if (NT > 1) {
            const uint32_t c = 4 * k + qc;
            ldmatrix4(qf[0], qrow + (c >> 3) * (R * 128) + (uint32_t)(n * 1024) + (((c & 7) ^ qx) << 4));
          }
          const uint32_t(&b)[4] = qf[NT == 1 ? k : 0];
          mma_bf16_16816(s[n], a0, b[0], b[1]);
          mma_bf16_16816(s[n], a1, b[2], b[3]);
        }
      }
      const int key = t * KT + 16 * warp + g8;   // and key + 8
      const bool edge = (t + 1) * KT > seen;
      if (edge && t * KT + 16 * warp + 16 > u.keys) {
        // values past the last key are leftovers (perhaps NaN): zero times them has to be zero
        for (int i = lane; i < 16 * (D / 8); i += 32) {
          const int r = 16 * warp + i / (D / 8), c = i % (D / 8);
          if (t * KT + r >= u.keys) {
            const uint32_t a = vb + (uint32_t)((c >> 3) * S::kHalfTile + r * 128 + ((c & 7) << 4));
            asm volatile("st.shared.v4.b32 [%0], {%1,%1,%1,%1};\n" ::"r"(a), "r"(0) : "memory");
          }
        }
        fence_proxy_async_smem();   // (before the next copy into this stage)
        __syncwarp();
      }
      uint32_t pb[NT][2];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          s[n][j] *= p.scale;
          if (edge && key + 8 * (j >> 1) >= lim[n][j & 1]) s[n][j] = -INFINITY;
        }
        float mx[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          mx[j] = fmaxf(s[n][j], s[n][j + 2]);
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) mx[j] = fmaxf(mx[j], __shfl_xor_sync(0xffffffffu, mx[j], d));
          mx[j] = fmaxf(mx[j], m[n][j]);
        }
        if (__any_sync(0xffffffffu, mx[0] > m[n][0] || mx[1] > m[n][1])) {
          float f[2];
#pragma unroll
          for (int j = 0; j < 2; ++j) {
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
          e[j] = exp2_approx(s[n][j] - (m[n][j & 1] == -INFINITY ? 0.f : m[n][j & 1]));
          l[n][j & 1] += e[j];
        }
        pb[n][0] = movmatrix(pack_bf16x2(e[0], e[1]));
        pb[n][1] = movmatrix(pack_bf16x2(e[2], e[3]));
      }
      const uint32_t vr = 16 * warp + ((lane >> 4) << 3) + (lane & 7), vc = (lane >> 3) & 1;
#pragma unroll
      for (int d = 0; d < D / 16; ++d) {
        uint32_t a[4];
        const uint32_t c = 2 * d + vc;
        ldmatrix4_trans(a, vb + (c >> 3) * S::kHalfTile + vr * 128 + (((c & 7) ^ (vr & 7)) << 4));
#pragma unroll
        for (int n = 0; n < NT; ++n) mma_bf16_16816(o[n][d], a, pb[n][0], pb[n][1]);
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&empty[st]);
    }
    // ---------------------------------------------------- join the warps
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) l[n][j] += __shfl_xor_sync(0xffffffffu, l[n][j], d);
        if (g8 == 0) {
          row_m[warp][8 * n + c2 + j] = m[n][j];
          row_l[warp][8 * n + c2 + j] = l[n][j];
        }
      }
    ok = group_and(1, kCon, ok);
    if (!ok) break;
    float f[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < W; ++w) top = fmaxf(top, row_m[w][8 * n + c2 + j]);
        f[n][j] = m[n][j] == -INFINITY ? 0.f : exp2_approx(m[n][j] - top);
      }
#pragma unroll 1
    for (int round = 0; round < W / S::kBufs; ++round) {
      if (warp / S::kBufs == round) {
        float* buf = bufs + (warp % S::kBufs) * (R * S::kPitch);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int d = 0; d < D / 16; ++d)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              float* at = buf + (8 * n + c2 + (j & 1)) * S::kPitch + 16 * d + 8 * (j >> 1) + g8;
              const float v = o[n][d][j] * f[n][j & 1];
              *at = round == 0 ? v : *at + v;
            }
      }
      named_bar_sync(1, kCon);
    }
    const bool head = u.a >= t0, whole = head && u.a + u.tiles <= t1;
    const bool direct = p.direct && whole;
    for (int i = tid; i < nrows * (D / 4); i += kCon) {
      const int r = i / (D / 4), c = i % (D / 4);
      float4 v = *reinterpret_cast<const float4*>(bufs + r * S::kPitch + 4 * c);
      if (S::kBufs == 2) {
        const float4 w = *reinterpret_cast<const float4*>(bufs + (R + r) * S::kPitch + 4 * c);
        v = make_float4(v.x + w.x, v.y + w.y, v.z + w.z, v.w + w.w);
      }
      float top = -INFINITY, sum = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) top = fmaxf(top, row_m[w][r]);
#pragma unroll
      for (int w = 0; w < W; ++w) sum += row_m[w][r] == -INFINITY ? 0.f : row_l[w][r] * exp2_approx(row_m[w][r] - top);
      const int tok = (r0 + r) / p.group, g = r0 + r - tok * p.group;
      const int64_t row = (int64_t)(u.first + tok) * p.q_heads + u.h * p.group + g;
      if (direct) {
        const float k = sum > 0.f ? 1.f / sum : sum;   // (0 where nothing is seen; NaN stays)
        *reinterpret_cast<uint2*>(p.out + row * D + 4 * c) = make_uint2(pack_bf16x2(v.x * k, v.y * k), pack_bf16x2(v.z * k, v.w * k));
        if (p.lse && c == 0) p.lse[row] = top == -INFINITY ? top : (top + log2_approx(sum)) * 0.69314718056f;
      } else {
        float* dst = head ? p.o[u.part] + row * D : p.slot_o + ((int64_t)blockIdx.x * R + r) * D;
        *reinterpret_cast<float4*>(dst + 4 * c) = v;
        if (c == 0) *(head ? p.ml[u.part] + row : p.slot_ml + (int64_t)blockIdx.x * R + r) = make_float2(top, sum);
      }
    }
  } while (ok && u.a + u.tiles < t1 && walk.next(u));
  if (!ok && lane == 0) call_record_fail(p.rec, p.call);
}

// ------------------------------------------------------------------- join
// One warp per row: the weighted sum of its partial results, in the order of
// the keys, so that a call's results do not depend on timing.
template <int D, int R, int KT>
__global__ void __launch_bounds__(256) join_kernel(const AttendParams p) {
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31;
  const int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (row >= (int64_t)p.b.n_tokens * p.q_heads) return;
  const int tok = (int)(row / p.q_heads), hq = (int)(row - (int64_t)tok * p.q_heads), h = hq / p.group, g = hq - h * p.group;
  const int s = seq_of_token(p.b.token_start, p.b.n_seqs, tok);
  const SeqSpan q = seq_span(p.b, s);
  const bool live = tok < q.first + q.count;
  constexpr int V = D / 32;
  float acc[V], top = -INFINITY, sum = 0.f;
#pragma unroll
  for (int i = 0; i < V; ++i) acc[i] = 0.f;
  bool done = false;   // written by the thread block that had the whole row
  const Walk<R, KT> walk(p);
  const int64_t share = p.narrow[kOwn] || p.narrow[kPrefix]
                            ? ((p.narrow[kOwn] ? p.base[p.b.n_seqs] : walk.prefix_total) + p.ctas - 1) / p.ctas : 1;
  for (int part = kPrefix; part >= kOwn; --part) {
    int n = 0, slot0 = 0, r = 0;   // partials: p.splits[part] by row, then slots slot0 ..
    if (p.wide[part]) {
      n = part == kPrefix || (live && (p.chained || q.own > 0)) ? p.splits[part] : 0;
    } else if (p.narrow[part]) {
      int64_t a = 0;
      int tiles = 0, rr = 0;
      if (part == kPrefix) {
        rr = tok * p.group + g;
        tiles = walk.prefix_tiles;
        a = ((int64_t)h * walk.prefix_rb + rr / R) * tiles;
      } else if (live && q.own > 0) {
        rr = (tok - q.first) * p.group + g;
        tiles = (q.own + KT - 1) / KT;
        a = p.base[s] + ((int64_t)h * ((q.count * p.group + R - 1) / R) + rr / R) * tiles;
      }
      r = rr % R;
      if (tiles > 0) {
        slot0 = (int)(a / share) + 1;
        n = (int)((a + tiles - 1) / share) - slot0 + 2;
        if (p.direct && n == 1) done = true;
      }
    }
    if (done) break;
    const int by_row = p.wide[part] ? n : min(n, 1);
    const int64_t rows = (int64_t)p.b.n_tokens * p.q_heads;
    for (int i0 = 0; i0 < n; i0 += 32) {
      float2 ml = make_float2(-INFINITY, 0.f);
      const int i = i0 + lane;
      if (i < n) ml = i < by_row ? p.ml[part][i * rows + row] : p.slot_ml[(int64_t)(slot0 + i - by_row) * R + r];
      float mx = ml.x;
      for (int d = 16; d; d >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
      mx = fmaxf(mx, top);
      const float old = top == -INFINITY ? 0.f : exp2_approx(top - mx);
      const float f = ml.x == -INFINITY ? 0.f : exp2_approx(ml.x - mx);
      float add = ml.y * f;
      if (ml.x == -INFINITY) add = 0.f;
      for (int d = 16; d; d >>= 1) add += __shfl_xor_sync(0xffffffffu, add, d);
      sum = sum * old + add;
      top = mx;
#pragma unroll
      for (int k = 0; k < V; ++k) acc[k] *= old;
      const int m = min(32, n - i0);
#pragma unroll 4
      for (int j = 0; j < m; ++j) {
        const float fj = __shfl_sync(0xffffffffu, f, j);
        const float* src = i0 + j < by_row ? p.o[part] + ((i0 + j) * rows + row) * D
                                           : p.slot_o + ((int64_t)(slot0 + i0 + j - by_row) * R + r) * D;
        if (V == 4) {
          const float4 v = *reinterpret_cast<const float4*>(src + 4 * lane);
          if (fj != 0.f) {
            acc[0] += fj * v.x;
            acc[1] += fj * v.y;
            acc[V - 2] += fj * v.z;
            acc[V - 1] += fj * v.w;
          }
        } else {
          const float2 v = *reinterpret_cast<const float2*>(src + 2 * lane);
          if (fj != 0.f) {
            acc[0] += fj * v.x;
            acc[1] += fj * v.y;
          }
        }
      }
    }
  }
  if (done) return;
  const float k = sum > 0.f ? 1.f / sum : sum;   // (0 where nothing is seen; NaN stays)
  uint32_t* dst = reinterpret_cast<uint32_t*>(p.out + row * D + V * lane);
#pragma unroll
  for (int i = 0; i < V; i += 2) dst[i / 2] = pack_bf16x2(acc[i] * k, acc[i + 1] * k);
  if (p.lse && lane == 0) p.lse[row] = top == -INFINITY ? top : (top + log2_approx(sum)) * 0.69314718056f;
}

// ------------------------------------------------------------------- host
struct Route {
  int nt;              // 8-row groups of the narrow kernel's row blocks (0: not used)
  int rows, ctas;      // its row block, its thread blocks
};

constexpr int kMaxNt = 4;   // the narrow kernel takes up to 32 rows of a key head

// The wide kernel takes the parts with more rows per key head than the narrow
// one's blocks hold.  Where a sequence brings 128 rows and more on the
// average, its row blocks run over the prefix and its own keys in one line;
// below that the batch's rows share blocks against the prefix.
Route route_of(const sdq_cache_s* c, const sdq_batch* b, int q_heads, AttendParams* p) {
  const int group = q_heads / c->desc.kv_heads;
  const int64_t own_rows = b->max_own > 0 ? (int64_t)b->max_new * group : 0;
  const int64_t prefix_rows = b->prefix_len > 0 ? (int64_t)b->n_tokens * group : 0;
  const bool own_wide = own_rows > 8 * kMaxNt;
  p->chained = own_wide && prefix_rows > 0 && prefix_rows >= 128ll * b->n_seqs;
  p->wide[kOwn] = own_wide;
  p->narrow[kOwn] = own_rows > 0 && !own_wide;
  p->wide[kPrefix] = prefix_rows > 8 * kMaxNt && !p->chained;
  p->narrow[kPrefix] = prefix_rows > 0 && prefix_rows <= 8 * kMaxNt;
  for (int part = 0; part < 2; ++part)
    p->splits[part] = p->wide[part] ? wide_splits(c, b, q_heads, part, p->chained) : p->narrow[part];
  const bool both = (p->wide[kOwn] || p->narrow[kOwn]) && (p->wide[kPrefix] || p->narrow[kPrefix]);
  p->direct = !both && p->splits[kOwn] <= 1 && p->splits[kPrefix] <= 1;
  Route r{};
  const int64_t most = std::max(p->narrow[kOwn] ? own_rows : 0, p->narrow[kPrefix] ? prefix_rows : 0);
  r.nt = (int)((most + 7) / 8);
  r.rows = 8 * r.nt;
  r.ctas = c->sm_count * (r.nt == 0 ? 0 : r.nt == 1 ? 2 : 1);
  return r;
}

AttendWs attend_workspace(const sdq_cache_s* c, const sdq_batch* b, int q_heads, const AttendParams& p, const Route& r) {
  const size_t rows = (size_t)b->n_tokens * q_heads, d = c->desc.head_dim;
  AttendWs L{};
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off = (off + bytes + 255) / 256 * 256;
    return at;
  };
  L.rec = take(4 * sizeof(uint64_t));
  L.base = take(sizeof(int64_t) * ((size_t)b->n_seqs + 1));
  for (int part = 0; part < 2; ++part) {
    L.ml[part] = take(sizeof(float2) * p.splits[part] * rows);
    L.o[part] = take(sizeof(float) * p.splits[part] * rows * d);
  }
  L.slot_ml = take(sizeof(float2) * (size_t)r.ctas * r.rows);
  L.slot_o = take(sizeof(float) * (size_t)r.ctas * r.rows * d);
  L.total = off;
  return L;
}

template <int D, int R, int KT>
cudaError_t launch_join(const AttendParams& p, cudaStream_t st) {
  const int64_t rows = (int64_t)p.b.n_tokens * p.q_heads;
  return launch_pdl(join_kernel<D, R, KT>, dim3((unsigned)((rows + 7) / 8)), dim3(256), 0, st, p);
}

template <int D, int NT>
cudaError_t launch_narrow(const sdq_cache_s* c, const AttendParams& p, cudaStream_t st) {
  using S = NarrowShape<D, NT>;
  static std::atomic<int> smem_set[64];
  cudaError_t e = smem_limit_once(narrow_kernel<D, NT>, S::kSmem, c->device, smem_set);
  if (e != cudaSuccess) return e;
  e = launch_pdl(narrow_kernel<D, NT>, dim3((unsigned)p.ctas), dim3(S::kThreads), (size_t)S::kSmem, st, c->kmap, c->vmap, p);
  return e == cudaSuccess ? launch_join<D, S::kRows, S::kTile>(p, st) : e;
}

template <int D>
cudaError_t launch_parts(const sdq_cache_s* c, const AttendParams& p, const Route& r, cudaStream_t st) {
  for (int part = kPrefix; part >= kOwn; --part)
    if (p.wide[part]) {
      const cudaError_t e = launch_wide(c, p, part, st);
      if (e != cudaSuccess) return e;
    }
  switch (r.nt) {
    case 0: return p.direct && (p.wide[kOwn] || p.wide[kPrefix]) ? cudaSuccess : launch_join<D, 8, 64>(p, st);
    case 1: return launch_narrow<D, 1>(c, p, st);
    case 2: return launch_narrow<D, 2>(c, p, st);
    case 3: return launch_narrow<D, 3>(c, p, st);
    default: return launch_narrow<D, 4>(c, p, st);
  }
}

int log2_of(int v) {
  int s = 0;
  while ((1 << s) < v) ++s;
  return s;
}

}  // namespace

}  // namespace sdq

using namespace sdq;

extern "C" size_t sdq_attention_workspace_bytes(sdq_cache c, const sdq_batch* b, int32_t q_heads) {
  if (check_batch(c, b, q_heads) != SDQ_OK) return 0;
  AttendParams p{};
  const Route r = route_of(c, b, q_heads, &p);
  return attend_workspace(c, b, q_heads, p, r).total;
}

extern "C" int sdq_attention(sdq_cache c, const sdq_batch* b, int32_t q_heads, const uint16_t* q, int64_t ldq, float scale,
                             uint16_t* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
  int st = check_batch(c, b, q_heads);
  if (st != SDQ_OK) return st;
  if ((st = check_cache_device(c)) != SDQ_OK) return st;
  if (!q || !out || !ws || !(scale > 0.f) || !std::isfinite(scale)) return SDQ_ERR_INVALID_ARG;
  const int d = c->desc.head_dim;
  if (ldq < (int64_t)q_heads * d || ldq % 8) return SDQ_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out)) & 15u) return SDQ_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(ws) & 255u) || (reinterpret_cast<uintptr_t>(lse) & 3u)) return SDQ_ERR_INVALID_ARG;
  AttendParams p{};
  const Route r = route_of(c, b, q_heads, &p);
  const AttendWs L = attend_workspace(c, b, q_heads, p, r);
  if (ws_bytes < L.total) return SDQ_ERR_WORKSPACE;
  uint8_t* w = static_cast<uint8_t*>(ws);
  p.b = *b;
  p.q = q; p.ldq = ldq; p.out = out; p.lse = lse;
  p.scale = scale * 1.44269504089f;
  p.q_heads = q_heads; p.kv_heads = c->desc.kv_heads; p.group = q_heads / c->desc.kv_heads;
  p.page_shift = log2_of(c->desc.page_tokens);
  p.box_shift = log2_of(cache_box_rows(c->desc));
  p.n_pages = c->desc.n_pages;
  p.rec = reinterpret_cast<uint64_t*>(w + L.rec);
  p.call = call_tag(next_call_number());
  p.base = reinterpret_cast<int64_t*>(w + L.base);
  for (int part = 0; part < 2; ++part) {
    p.o[part] = reinterpret_cast<float*>(w + L.o[part]);
    p.ml[part] = reinterpret_cast<float2*>(w + L.ml[part]);
  }
  p.slot_o = reinterpret_cast<float*>(w + L.slot_o);
  p.slot_ml = reinterpret_cast<float2*>(w + L.slot_ml);
  p.ctas = r.ctas;
  const cudaError_t e = d == 128 ? launch_parts<128>(c, p, r, (cudaStream_t)stream) : launch_parts<64>(c, p, r, (cudaStream_t)stream);
  return e == cudaSuccess ? SDQ_OK : SDQ_ERR_CUDA;
}

extern "C" int sdq_attention_status(const void* ws, void* stream) {
  if (!ws) return SDQ_ERR_INVALID_ARG;
  uint64_t rec[2] = {0, 0};   // last failed call, last call
  cudaError_t e = cudaMemcpyAsync(rec, ws, sizeof(rec), cudaMemcpyDeviceToHost, (cudaStream_t)stream);
  if (e == cudaSuccess) e = cudaStreamSynchronize((cudaStream_t)stream);
  if (e != cudaSuccess) return SDQ_ERR_CUDA;
  return rec[1] != 0 && rec[0] == rec[1] ? SDQ_ERR_TIMEOUT : SDQ_OK;
}
