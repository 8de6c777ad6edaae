// Attention over the paged cache: the kernel for many query rows per key head
// (prompts, and a batch's rows against the shared prefix).
#include <algorithm>

#include "attention.cuh"

namespace sdq {

namespace {

// ----------------------------------------------------------- wide kernel
// A thread block takes 256 query rows of one key head (new token major, then
// head of the group) and a line of key tiles (128 keys each: the prefix's,
// then the sequence's own, or one of the two); the tensor cores bound it, 2 x
// 128 x 128 x head_dim products a tile and 128 rows:
//   warps 0-3, 4-7  rows 0-127, 128-255, a row per thread: S from tensor
//                   memory 64 keys at a time, running maximum and sum, P (bf16)
//                   back into S's place; O is rescaled there only when a row's
//                   maximum has grown by more than 2^8 (weights stay below
//                   2^8, sums in fp32 lose nothing by it)
//   warp 8          S = Q K^T (both from shared memory) and O += P V (P from
//                   tensor memory, V as the transposed operand) on tcgen05;
//                   the first 64 keys' product runs while the row's thread
//                   works on the other 64, and one half's products while the
//                   other's softmax runs
//   warp 9          K and V tiles, page by page, into a ring (TMA, 128-byte
//                   swizzle); warps 10 and 11 only complete its warpgroup
// The MMAs of a thread block run in the order of their issue, so that S of the
// next tile may overwrite P once the product that reads it is issued.
// Few row blocks: several thread blocks share the line of one, write their sums
// to the workspace, and the kernel that joins a call's parts takes them all.  (As
// clusters that joined at the end of this kernel, in the workspace or in their
// shared memory, they took 4 to 10 us longer, and the device holds fewer.)
// A tile takes 2320 cycles (2048 of products), a thread block's start 5000, its
// output 3000 (6500 as fp32 sums).  Prompts of 400 to 2500 tokens behind 1021,
// 64 heads: 200 us, 67 % of the measured bf16 rate (196 without the look for
// values that are not finite); 64 tokens of 64 heads against 8199 keys alone: 28
// us.
// Registers: 384 threads hold 168 each at launch; the first two warpgroups go
// to 224 once the third has gone down to 56 (224 + 224 + 56 = 3 x 168).
constexpr int kWideThreads = 384;
constexpr int kKeys = 128;             // of a tile
constexpr int kSub = 64;               // keys of one P
constexpr int kHalf = kKeys * 128;     // bytes: 128 rows x 64 elements

template <int D> struct WideShape {
  static constexpr int kMat = (D / 64) * kHalf;              // 128 rows of Q, K or V
  static constexpr int kRing = D == 128 ? 5 : 8;
  static constexpr int kSmem = 1024 + (2 + kRing) * kMat;
  static_assert(256 * D * 4 <= (2 + kRing) * kMat, "256 fp32 rows fit over the operands");
};

__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
        "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
        "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr));
}

// Two fp32 in a 64-bit register, and arithmetic on both at once.
__device__ __forceinline__ uint64_t pair_of(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};\n" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpair(uint64_t p, float& a, float& b) {
  asm("mov.b64 {%0, %1}, %2;\n" : "=f"(a), "=f"(b) : "l"(p));
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;\n" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;\n" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;\n" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;\n" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// Operand with its second dimension contiguous (V: keys x 64 elements per
// 128-byte row, 128-byte swizzle): 8-key groups 1024 bytes apart, the next 64
// elements kHalf bytes on.
__device__ __forceinline__ uint64_t sw128_mn_desc(uint32_t saddr) {
  uint64_t d = 0;
  d |= (uint64_t)((saddr & 0x3FFFFu) >> 4);
  d |= (uint64_t)(kHalf >> 4) << 16;
  d |= (uint64_t)(1024 >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}

// What a thread block works on.
struct WideItem {
  int first, rows, r0;       // first token, rows of the (sequence, head) or of the batch, first row of the block
  int h, split;
  int s;                     // sequence, -1: the whole batch
  int own, count;            // its own tokens and new tokens
  int prefix_tiles, t0, t1;  // of the line: the prefix's tiles, this block's [t0, t1)
};

// (a whole warp; false: nothing to do)
__device__ __forceinline__ bool wide_item(const AttendParams& p, int part, WideItem* w) {
  const int splits = p.splits[part];
  const int id = blockIdx.x / (p.kv_heads * splits), rest = blockIdx.x % (p.kv_heads * splits);
  w->h = rest / splits;
  w->split = rest % splits;
  const int ptiles = (p.b.prefix_len + kKeys - 1) / kKeys;
  int tiles;
  if (part == kPrefix) {
    w->s = -1;
    w->first = 0;
    w->rows = p.b.n_tokens * p.group;
    w->r0 = id * 256;
    w->own = w->count = 0;
    w->prefix_tiles = tiles = ptiles;
    if (w->r0 >= w->rows) return false;
  } else {
    // block `id` counted over the sequences' row blocks
    const int lane = threadIdx.x & 31;
    int base = 0, s = -1, rb = 0;
    SeqSpan q{0, 0, 0};
    for (int s0 = 0; s0 < p.b.n_seqs && s < 0; s0 += 32) {
      SeqSpan x{0, 0, 0};
      if (s0 + lane < p.b.n_seqs) x = seq_span(p.b, s0 + lane);
      const int n = (x.count * p.group + 255) / 256;
      int end = n;
      for (int d = 1; d < 32 && s0 + d < p.b.n_seqs; d <<= 1) {
        const int o = __shfl_up_sync(0xffffffffu, end, d);
        if (lane >= d) end += o;
      }
      const uint32_t past = __ballot_sync(0xffffffffu, base + end > id);
      if (past) {
        const int l = __ffs(past) - 1;
        s = s0 + l;
        rb = id - base - __shfl_sync(0xffffffffu, end - n, l);
        rb = __shfl_sync(0xffffffffu, n, l) - 1 - rb;   // the blocks that see the most keys first
        q = SeqSpan{__shfl_sync(0xffffffffu, x.first, l), __shfl_sync(0xffffffffu, x.count, l), __shfl_sync(0xffffffffu, x.own, l)};
      }
      base += __shfl_sync(0xffffffffu, end, 31);
    }
    if (s < 0) return false;
    w->s = s;
    w->first = q.first;
    w->count = q.count;
    w->own = q.own;
    w->rows = q.count * p.group;
    w->r0 = rb * 256;
    w->prefix_tiles = p.chained ? ptiles : 0;
    const int last = min(w->rows, w->r0 + 256) - 1;   // its last row sees the most
    tiles = w->prefix_tiles + (max(0, q.own - q.count + last / p.group + 1) + kKeys - 1) / kKeys;
  }
  const int per = (tiles + splits - 1) / splits;
  w->t0 = min(tiles, w->split * per);
  w->t1 = min(tiles, w->t0 + per);
  return true;
}

template <int D>
__global__ void __launch_bounds__(kWideThreads, 1)
    wide_kernel(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap, const AttendParams p,
                const int part) {
  using S = WideShape<D>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t full[S::kRing], empty[S::kRing], q_full, s_full[2], p_full[2][2], pv_done[2], mma_done;
  __shared__ uint32_t tmem_base;
  __shared__ volatile int tainted;   // a value that is not finite was taken out
  const int tid = threadIdx.x, warp = warp_index(), lane = tid & 31;
  const uint32_t sbase = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t ring = sbase + 2 * S::kMat;
  uint8_t* ring_ptr = smem_raw + (ring - smem_u32(smem_raw));
  if (tid == 0) {
    for (int i = 0; i < S::kRing; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], 1);
    }
    mbar_init(&q_full, 256);
    for (int i = 0; i < 2; ++i) {
      mbar_init(&s_full[i], 1);
      for (int j = 0; j < 2; ++j) mbar_init(&p_full[i][j], 128);
      mbar_init(&pv_done[i], 1);
    }
    mbar_init(&mma_done, 1);
    tainted = 0;
    fence_mbar_init();
  }
  if (warp == 8) {
    tmem_alloc(&tmem_base, 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_wait();
  pdl_launch_dependents();
  call_record_start(p.rec, p.call, blockIdx.x == 0 && tid == 0);
  WideItem w;
  if (!wide_item(p, part, &w)) {   // (all warps alike)
    if (warp == 8) tmem_dealloc(tmem_base, 512);
    return;
  }
  const int n = w.t1 - w.t0, halves = w.rows - w.r0 > 128 ? 2 : 1;
  // at the end: fp32 sums for the join, or rows of the output
  const bool joins = p.splits[part] > 1 || p.parts > 1;
  const uint32_t tmem = tmem_base;
  bool ok = true;
  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 56;\n");
    if (warp == 9) {
      // ------------------------------------------------------------ loads
      const int box = 1 << p.box_shift, per_page = 1 << (p.page_shift - p.box_shift), per_tile = kKeys >> p.box_shift;
      const int32_t* own_table = p.b.pages + (int64_t)(w.s < 0 ? 0 : w.s) * p.b.page_stride;
      // the page of the lane's box of line tile t (-1: past the last token), and the tile's boxes
      auto boxes_of = [&](int t) {
        const int keys = t < w.prefix_tiles ? p.b.prefix_len : w.own, at = (t < w.prefix_tiles ? t : t - w.prefix_tiles) * per_tile;
        return max(0, min(per_tile, ((keys + box - 1) >> p.box_shift) - at));
      };
      auto row_of = [&](int t) {
        const int at = (t < w.prefix_tiles ? t : t - w.prefix_tiles) * per_tile + lane;
        const int pg = t < w.t1 && lane < boxes_of(t) ? __ldg((t < w.prefix_tiles ? p.b.prefix_pages : own_table) + at / per_page) : -1;
        // (a page outside the cache: rows outside the arrays, which read as zeros)
        return pg >= 0 && pg < p.n_pages ? ((pg * p.kv_heads + w.h) << p.page_shift) + ((at & (per_page - 1)) << p.box_shift) : -box;
      };
      int y_next = row_of(w.t0), slot = 0;
      for (int t = w.t0; t < w.t1 && ok; ++t) {
        const int y = y_next, nb = boxes_of(t);
        y_next = row_of(t + 1);
#pragma unroll
        for (int kv = 0; kv < 2; ++kv, ++slot) {
          const int st = slot % S::kRing, r = slot / S::kRing;
          if (r > 0 && !mbar_wait_warp(&empty[st], (r - 1) & 1)) {
            ok = false;
            break;
          }
          mbar_expect_tx_warp(&full[st], (uint32_t)((nb << p.box_shift) * 128 * (D / 64)));
          for (int i = 0; i < nb; ++i) {
            const int yi = __shfl_sync(0xffffffffu, y, i);
#pragma unroll
            for (int half = 0; half < D / 64; ++half)
              tma_load_2d_warp(ring_ptr + st * S::kMat + half * kHalf + ((i * box) << 7), kv ? &vmap : &kmap, 64 * half, yi, &full[st]);
          }
        }
      }
      // the copies in flight have landed before the thread block ends
      for (int j = max(0, slot - S::kRing); j < slot; ++j)
        if (!mbar_wait_warp(&full[j % S::kRing], (j / S::kRing) & 1)) ok = false;
    } else if (warp == 8) {
      // --------------------------------------------------------- products
      constexpr uint32_t kF32Bf16 = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(128 >> 4) << 24);   // M = 128
      // (64 keys an MMA for S would read Q twice as often: shared memory would bound it, 128 bytes a cycle)
      constexpr uint32_t qk_idesc = kF32Bf16 | ((uint32_t)(kKeys >> 3) << 17);
      constexpr uint32_t pv_idesc = kF32Bf16 | ((uint32_t)(D >> 3) << 17) | (1u << 16);   // B with its N contiguous
      auto scores = [&](int half, int st) {
        const uint64_t a = sw128_desc(sbase + half * S::kMat), b = sw128_desc(ring + st * S::kMat);
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const uint64_t off = (uint64_t)((k >> 2) * (kHalf >> 4) + 2 * (k & 3));
          umma_bf16_warp(tmem + 128 * half, a + off, b + off, qk_idesc, k > 0);
        }
        umma_commit_warp(&s_full[half]);
      };
      if (n > 0) {
        ok = mbar_wait_warp(&q_full, 0) && mbar_wait_warp(&full[0], 0);
        tc_fence_after();
        if (ok) {
          for (int half = 0; half < halves; ++half) scores(half, 0);
          umma_commit_warp(&empty[0]);
        }
        for (int i = 0; i < n && ok; ++i) {
          const int kn = 2 * i + 2, vs = (2 * i + 1) % S::kRing, ks = kn % S::kRing;
          for (int half = 0; half < halves && ok; ++half) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              if (ok) ok = mbar_wait_warp(&p_full[half][j], i & 1);
              if (ok && j + half == 0) ok = mbar_wait_warp(&full[vs], ((2 * i + 1) / S::kRing) & 1);
              if (!ok) break;
              tc_fence_after();
              const uint64_t b = sw128_mn_desc(ring + vs * S::kMat + j * (kSub * 128));
#pragma unroll
              for (int k = 0; k < kSub / 16; ++k)
                umma_bf16_ts_warp(tmem + 256 + D * half, tmem + 128 * half + kSub * j + 8 * k, b + (uint64_t)(k * (2048 >> 4)),
                                  pv_idesc, (i | j | k) != 0);
              if (j == 0) umma_commit_warp(&pv_done[half]);
            }
            if (half == halves - 1) umma_commit_warp(&empty[vs]);
            if (i + 1 < n) {
              if (ok && half == 0) ok = mbar_wait_warp(&full[ks], (kn / S::kRing) & 1);
              if (!ok) break;
              tc_fence_after();
              scores(half, ks);
              if (half == halves - 1) umma_commit_warp(&empty[ks]);
            }
          }
        }
        umma_commit_warp(&mma_done);
        if (!mbar_wait_warp(&mma_done, 0)) ok = false;
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 224;\n");
    if ((warp >> 2) < halves) {
      // ---------------------------------------------------------- softmax
      const int half = warp >> 2, wtid = tid & 127;
      const uint32_t qb = sbase + half * S::kMat;
      const int row = w.r0 + 128 * half + wtid, tok = row / p.group, g = row - tok * p.group;
      const bool live = row < w.rows;
      {
        // a warp its 32 rows, a row's chunks by neighbouring lanes (rows past the last: zeros)
        constexpr int kChunks = D / 8;
        const uint16_t* mine = p.q + (live ? (int64_t)(w.first + tok) * p.ldq + (int64_t)(w.h * p.group + g) * D : 0);
        const uint32_t bytes = live ? 16u : 0u;
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {
          const int l = (32 / kChunks) * i + lane / kChunks, r = 32 * (warp & 3) + l, c = lane % kChunks;
          const uint16_t* src = reinterpret_cast<const uint16_t*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(mine), l));
          cp_async16(smem_raw + (qb - smem_u32(smem_raw)) + (c >> 3) * kHalf + r * 128 + (((c & 7) ^ (r & 7)) << 4), src + 8 * c,
                     __shfl_sync(0xffffffffu, bytes, l));
        }
      }
      cp_async_wait_all();
      fence_proxy_async_smem();
      mbar_arrive(&q_full);
      // own keys that this row sees, and that every row of its half does
      const int lim = live ? w.own - w.count + tok + 1 : w.own;
      const int all = w.own - w.count + (w.r0 + 128 * half) / p.group + 1;
      // and that every row of the block does.  Values of later ones that are not
      // finite are taken out of the tile, as zero times them is not zero, and added
      // at the end to the rows that see them
      const int all_rows = max(0, w.own - w.count + w.r0 / p.group + 1);
      const uint32_t ts = tmem + ((uint32_t)(32 * (warp & 3)) << 16) + 128 * half;
      const uint32_t to = tmem + ((uint32_t)(32 * (warp & 3)) << 16) + 256 + D * half;
      float m = -INFINITY;        // reference maximum (log2 units)
      uint64_t l2 = 0;            // two sums
      const uint64_t scale2 = pair_of(p.scale, p.scale);
      for (int q = 0; q < 2 * n; ++q) {
        const int i = q >> 1, j = q & 1;
        if (j == 0 && !mbar_wait_warp(&s_full[half], i & 1)) {
          ok = false;
          break;
        }
        tc_fence_after();
        uint32_t x[kSub];
        tmem_ld32(ts + kSub * j, x);
        tmem_ld32(ts + kSub * j + 32, x + 32);
        tmem_ld_wait();
        const int t = w.t0 + i;
        const bool pre = t < w.prefix_tiles;
        const int k0 = (pre ? t : t - w.prefix_tiles) * kKeys + kSub * j, keys = pre ? p.b.prefix_len : w.own;
        if (k0 + kSub > (pre ? keys : all)) {
          const int see = (pre ? keys : lim) - k0;   // of these 64
#pragma unroll
          for (int c = 0; c < kSub; ++c)
            if (c >= see) x[c] = 0xFF800000u;
        }
        if (half == 0 && k0 + kSub > (pre ? keys : min(keys, all_rows))) {
          // (for both halves: the second's product is issued after the first's)
          // values past the last key are leftovers (perhaps NaN): zero times them has to be zero too
          const int vs = (2 * i + 1) % S::kRing, from = 8 * max(0, (pre ? keys : min(keys, all_rows)) - k0);
          if (!mbar_wait_warp(&full[vs], ((2 * i + 1) / S::kRing) & 1)) {
            ok = false;
            break;
          }
          const uint32_t at = ring + vs * S::kMat + (kSub * j) * 128;   // 16-byte pieces c of the rows
#pragma unroll 1
          for (int c = from + wtid; c < 8 * kSub; c += 256) {
            uint4 v[2][D / 64];
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
              for (int d = 0; d < D / 64; ++d) v[k][d] = ld_shared16(at + d * kHalf + 16 * min(c + 128 * k, 8 * kSub - 1));
            bool any = false;
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
              for (int d = 0; d < D / 64; ++d) any |= some_not_finite(v[k][d]);
            if (!any) continue;
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
              for (int d = 0; d < D / 64; ++d) {
                const uint4 x = v[k][d];
                if (c + 128 * k >= 8 * kSub || !some_not_finite(x)) continue;
                if (k0 + ((c + 128 * k) >> 3) < keys) tainted = 1;
                st_shared16(at + d * kHalf + 16 * (c + 128 * k), x.x & ~not_finite(x.x), x.y & ~not_finite(x.y), x.z & ~not_finite(x.z),
                            x.w & ~not_finite(x.w));
              }
          }
          fence_proxy_async_smem();
        }
        float mx[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) mx[c] = max3(__uint_as_float(x[3 * c]), __uint_as_float(x[3 * c + 1]), __uint_as_float(x[3 * c + 2]));
#pragma unroll
        for (int c = 12; c < kSub; c += 2) mx[(c >> 1) & 3] = max3(mx[(c >> 1) & 3], __uint_as_float(x[c]), __uint_as_float(x[c + 1]));
        const float top = max3(mx[0], mx[1], fmaxf(mx[2], mx[3])) * p.scale;
        const bool grow = top > m + 8.f;   // (also from -inf)
        if (__any_sync(0xffffffffu, grow)) {
          const float f = grow ? exp2_approx(m - top) : 1.f;
          if (grow) m = top;
          l2 = mul2(l2, pair_of(f, f));
          if (q > 0) {   // once the products so far are in O (those of the tiles before are, with this one's S)
            if (j == 1 && !mbar_wait_warp(&pv_done[half], i & 1)) {
              ok = false;
              break;
            }
            tc_fence_after();
#pragma unroll
            for (int c = 0; c < D / 32; ++c) {
              uint32_t o[32];
              tmem_ld32(to + 32 * c, o);
              tmem_ld_wait();
#pragma unroll
              for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * f);
              tmem_st32(to + 32 * c, o);
            }
          }
        }
        const float neg = m == -INFINITY ? 0.f : -m;
        const uint64_t neg2 = pair_of(neg, neg);
        uint64_t sum[2] = {0, 0};
        uint32_t e[kSub / 2];
#pragma unroll
        for (int c = 0; c < kSub / 2; ++c) {
          float a, b;
          unpair(fma2(pair_of(__uint_as_float(x[2 * c]), __uint_as_float(x[2 * c + 1])), scale2, neg2), a, b);
          a = exp2_approx(a);
          b = exp2_approx(b);
          sum[c & 1] = add2(sum[c & 1], pair_of(a, b));
          e[c] = pack_bf16x2(a, b);
        }
        tmem_st32(ts + kSub * j, e);
        l2 = add2(l2, add2(sum[0], sum[1]));
        tmem_st_wait();
        tc_fence_before();
        mbar_arrive(&p_full[half][j]);
      }
      float l, lb;
      unpair(l2, l, lb);
      l += lb;
      // ------------------------------------------------------------- out
      if (n > 0 && ok) ok = mbar_wait_warp(&mma_done, 0);
      tc_fence_after();
      if (n > 0 && ok && tainted) {
#pragma unroll 1
        for (int c = 0; c < D / 32; ++c) {
          uint32_t o[32];
          tmem_ld32(to + 32 * c, o);
          tmem_ld_wait();
#pragma unroll 1
          for (int key = all_rows; live && key < lim; ++key) {
            const int pg = __ldg(p.b.pages + (int64_t)w.s * p.b.page_stride + (key >> p.page_shift));
            if (pg < 0 || pg >= p.n_pages) continue;
            const uint32_t* v = reinterpret_cast<const uint32_t*>(
                p.v + ((((int64_t)pg * p.kv_heads + w.h) << p.page_shift) + (key & ((1 << p.page_shift) - 1))) * D + 32 * c);
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              const uint32_t x = __ldg(v + j), bad = not_finite(x);
              if (bad & 0xFFFFu) o[2 * j] = __float_as_uint(__uint_as_float(o[2 * j]) + __uint_as_float(x << 16));
              if (bad >> 16) o[2 * j + 1] = __float_as_uint(__uint_as_float(o[2 * j + 1]) + __uint_as_float(x & 0xFFFF0000u));
            }
          }
          __syncwarp();
          tmem_st32(to + 32 * c, o);
        }
        tmem_st_wait();
      }
      if (joins) {
        // fp32 rows through shared memory, over operands that nothing reads any
        // more (nor has still to arrive: the barrier is behind all copies of Q)
        named_bar_sync(1, 128 * halves);
        const int64_t at = (int64_t)(w.first + tok) * p.q_heads + w.h * p.group + g;
        const bool split = p.splits[part] > 1;
        const int64_t slot = (split ? (int64_t)w.split * p.b.n_tokens * p.q_heads : 0) + at;
        const uint32_t stage = sbase + (uint32_t)((128 * half + 32 * (warp & 3)) * 4 * D), mine = stage + (uint32_t)(lane * 4 * D);
        const uint32_t lives = __ballot_sync(0xffffffffu, live);
        const unsigned long long dst = reinterpret_cast<unsigned long long>((split ? p.split_o[part] : p.o[part]) + slot * D);
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          uint32_t o[32];
          if (n > 0) {
            tmem_ld32(to + 32 * c, o);
            tmem_ld_wait();
          } else {
#pragma unroll
            for (int j = 0; j < 32; ++j) o[j] = 0;
          }
#pragma unroll
          for (int j = 0; j < 8; ++j)
            st_shared16(mine + (((8 * c + j) ^ (lane & 7)) << 4), o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]);
        }
        __syncwarp();
        constexpr int kChunks = D / 4, kAt = 32 / kChunks;   // 16-byte pieces of a row, rows at once
#pragma unroll 8
        for (int i = 0; i < kChunks; ++i) {
          const int r = kAt * i + lane / kChunks, c = lane % kChunks;
          uint4* to_row = reinterpret_cast<uint4*>(__shfl_sync(0xffffffffu, dst, r)) + c;
          const uint4 v = ld_shared16(stage + (uint32_t)(r * 4 * D) + ((c ^ (r & 7)) << 4));
          if (lives >> r & 1) *to_row = v;
        }
        if (live) (split ? p.split_ml[part] : p.ml[part])[slot] = make_float2(l == l ? m : l, l);   // (NaN scores leave no maximum)
      } else if (ok) {
        // rows to memory over the place of Q, which nothing reads any more: a
        // thread's row would go out in 16-byte pieces, 32 rows at a time.  (Nor
        // has Q still to arrive: the products began behind all copies of it; where
        // there was none, a warp's place may be the target of another's copies)
        if (n == 0) named_bar_sync(1, 128 * halves);
        const int64_t at = (int64_t)(w.first + tok) * p.q_heads + w.h * p.group + g;
        const float k = l > 0.f ? 1.f / l : l;       // (0 where nothing is seen; NaN stays)
        constexpr int kChunks = D / 8;
        const uint32_t stage = qb + (uint32_t)(32 * (warp & 3) * 2 * D);
        const uint32_t mine = stage + (uint32_t)(lane * 2 * D);
        const uint32_t lives = __ballot_sync(0xffffffffu, live);
        unsigned long long dst = reinterpret_cast<unsigned long long>(p.out + at * D);
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          uint32_t o[32];
          if (n > 0) {
            tmem_ld32(to + 32 * c, o);
            tmem_ld_wait();
          } else {
#pragma unroll
            for (int j = 0; j < 32; ++j) o[j] = 0;
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t v0 = pack_bf16x2(__uint_as_float(o[8 * j]) * k, __uint_as_float(o[8 * j + 1]) * k);
            const uint32_t v1 = pack_bf16x2(__uint_as_float(o[8 * j + 2]) * k, __uint_as_float(o[8 * j + 3]) * k);
            const uint32_t v2 = pack_bf16x2(__uint_as_float(o[8 * j + 4]) * k, __uint_as_float(o[8 * j + 5]) * k);
            const uint32_t v3 = pack_bf16x2(__uint_as_float(o[8 * j + 6]) * k, __uint_as_float(o[8 * j + 7]) * k);
            st_shared16(mine + (((4 * c + j) ^ (lane & 7)) << 4), v0, v1, v2, v3);
          }
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {
          const int r = (32 / kChunks) * i + lane / kChunks, c = lane % kChunks;
          uint4* to_row = reinterpret_cast<uint4*>(__shfl_sync(0xffffffffu, dst, r)) + c;
          const uint4 v = ld_shared16(stage + (uint32_t)(r * 2 * D) + ((c ^ (r & 7)) << 4));
          if (lives >> r & 1) *to_row = v;
        }
        if (live && p.lse) p.lse[at] = natural_lse(m, l);
      }
    }
    else mbar_arrive(&q_full);
  }
  if (!ok && lane == 0) call_record_fail(p.rec, p.call);
  tc_fence_before();
  __syncthreads();
  if (warp == 8) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

// Row blocks that the grid has to hold: of all tokens, or at most those of the
// sequences (each ends in a block of its own).
int64_t wide_blocks(const sdq_batch* b, int group, int part) {
  const int64_t rows = (int64_t)b->n_tokens * group;
  return part == kPrefix ? (rows + 255) / 256 : rows / 256 + std::min(b->n_seqs, b->n_tokens);
}

template <int D>
cudaError_t launch(const sdq_cache_s* c, const AttendParams& p, int part, cudaStream_t st) {
  static std::atomic<int> smem_set[64];
  const cudaError_t e = smem_limit_once(wide_kernel<D>, WideShape<D>::kSmem, c->device, smem_set);
  if (e != cudaSuccess) return e;
  return launch_pdl(wide_kernel<D>, dim3((unsigned)wide_grid(c, p, part)), dim3(kWideThreads), (size_t)WideShape<D>::kSmem, st, c->kmap,
                    c->vmap, p, part);
}

}  // namespace

int64_t wide_grid(const sdq_cache_s* c, const AttendParams& p, int part) {
  return wide_blocks(&p.b, p.group, part) * c->desc.kv_heads * p.splits[part];
}

// us, over waves of thread blocks: a tile (256 rows) takes 1.3 us, a thread
// block's two ends 5 us.
double wide_time(const sdq_cache_s* c, const sdq_batch* b, int q_heads, int part, bool chained, int s) {
  const int64_t blocks = wide_blocks(b, q_heads / c->desc.kv_heads, part) * c->desc.kv_heads * s;
  const int64_t tiles = (part == kPrefix || chained ? ((int64_t)b->prefix_len + kKeys - 1) / kKeys : 0) +
                        (part == kOwn ? ((int64_t)b->max_own + kKeys - 1) / kKeys : 0);
  return (double)((blocks + c->sm_count - 1) / c->sm_count) * (5.0 + 1.3 * (double)((tiles + s - 1) / s));
}

// The least of: its time; the join of the parts' sums, a launch (3 us) and 4
// TB/s; and what the narrow kernel beside it, where that takes the other part,
// needs longer: kNarrowStart and its reading (40 bytes a ns and SM) on the SMs
// left free, or on all of them afterwards.  (The lengths are not known here, only
// their bound: a sixth of it stands for them, the mean of lengths spread over
// their logarithm.)  64 sequences of 8 heads a key head behind 8199 keys, own
// lengths up to 512, 7 parts by this rule, us for 3, 5, 6, 7, 8 parts: lengths
// over their logarithm 45, 35, 33, 31, 41; all at the bound 50, 52, 52, 53, 57;
// all of 1 but one 44, 34, 32, 31, 31.  16 of 32 heads behind 2051, up to 300,
// 3 parts, us for 2, 3, 4: 21, 19, 24; at the bound 34, 33, 37; 21, 19, 23.
int wide_splits(const sdq_cache_s* c, const sdq_batch* b, int q_heads, int part, bool chained, bool narrow) {
  const double own = narrow ? (double)b->n_seqs * c->desc.kv_heads * b->max_own / 6 * c->desc.head_dim * 4 : 0.0;   // bytes
  auto time = [&](int s) {
    const double t = wide_time(c, b, q_heads, part, chained, s);
    const int64_t grid = wide_blocks(b, q_heads / c->desc.kv_heads, part) * c->desc.kv_heads * s;
    const double free = 40e3 * (double)std::max<int64_t>(0, c->sm_count - grid);   // bytes a us
    const double both = own <= free * t ? std::max(t, kNarrowStart + own / std::max(1.0, free))
                                        : t + kNarrowStart + (own - free * t) / (40e3 * c->sm_count);
    return both + (s > 1 ? 3.0 + (double)b->n_tokens * q_heads * c->desc.head_dim * 4.0 * s / 4e6 : 0.0);
  };
  int best = 1;
  for (int s = 2; s <= kMaxWideSplits; ++s)
    if (time(s) < time(best)) best = s;
  return best;
}

cudaError_t launch_wide(const sdq_cache_s* c, const AttendParams& p, int part, cudaStream_t st) {
  return c->desc.head_dim == 128 ? launch<128>(c, p, part, st) : launch<64>(c, p, part, st);
}

}  // namespace sdq
