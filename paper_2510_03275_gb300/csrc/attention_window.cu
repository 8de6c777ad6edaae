// Attention over the paged cache with a window of positions: the kernel for many
// query rows per key head (prompts).
#include <algorithm>

#include "attention_wide.cuh"

namespace sdq {

namespace {

// --------------------------------------------------------- window kernel
// Row blocks of 256 query rows of one key head, as in the wide kernel, and the same
// division of labour; but what they see is a dozen tiles or two, so that a
// block's ends (its search, its queries, its first keys, its output) would
// cost as much as a third of its products.  So one thread block per SM stays and takes
// items (a row block, a key head, a share of its keys) one after another, whose
// ends run beside each other:
//   warp 10         looks the next item up, into one of two places
//   warp 9          streams the keys and values of item after item
//   warp 11         looks at the values of keys that not all rows see, and passes
//                   every tile of values on
//   warp 8          starts the next scores behind the last product of an item,
//                   while its output is still being written
//   warps 0-3, 4-7  rows 0-127, 128-255: softmax and output; they copy the next
//                   item's queries over the last ones' as soon as the last scores are
//                   there, ahead of their softmax (by one warp beside them: 2.5 us an
//                   item more)
// The other kind of items: all of the batch's rows against what the sequences see
// of the prefix (part kPrefix), each row from where its own window begins.
// An item's line is of 64-key pieces, two to a tile, so that what is left out,
// first keys apart from the window, and the ends cost half a tile at most.
// Prompts of 13757 tokens, 64 heads of 128, window 1024 and 4 first tokens, behind
// 515: 422 us, 1070 TFLOP/s of what the rows see (58 % of the measured bf16 rate).  An
// item takes 18.5 us: 9.0 tiles, of which the rows see 7.75, are 12.3 of them at that
// rate (1.7 for what nobody sees of the tiles at the edges), the rest are its ends and
// the waits between products.
// P is rounded to bf16 for its product with bf16 values, as in the other kernels (relative
// 2^-8 at most per weight, as the values themselves carry); sums, maxima and outputs are
// fp32, the output rounded once.
// Registers: 384 threads hold 168 each at launch; the third warpgroup goes down to
// 72, the first two up to 216 (2 x 216 + 72 = 3 x 168).

// Stages of keys and of values (apart, so that whoever waits for the values has
// waited for every use of a stage before).
template <int D> constexpr int kStagesK = WideShape<D>::kRing / 2;
template <int D> constexpr int kStagesV = WideShape<D>::kRing - kStagesK<D>;

struct Item {
  int valid;                 // 0: there are no more
  int first, rows, r0;       // first token, rows of the (sequence, head), first row of the block
  int h, split, s;           // key head, share, sequence (-1: the whole batch)
  int own, count;            // its own tokens and new tokens
  int piece, n, n_pieces;    // first piece of the line, tiles and pieces from there on
  int all_rows, low_rows;    // own keys that every row of the block sees, the first position that all of their windows have
  Line prefix, mine;         // which pieces of the prefix's and of the own keys the line holds
};
// Piece q of an item: is it the prefix's, its first key.
struct Piece {
  bool pre;
  int k0;
};
__device__ __forceinline__ Piece piece_at(const volatile Item& w, int q) {
  const int c = w.piece + q, i = c - w.prefix.tiles;
  if (i < 0) return Piece{true, w.prefix.tile(c) * kSub};
  return Piece{false, w.mine.tile(i) * kSub};
}

// Does a piece hold keys that not all rows of the block see?  Values there that
// are not finite are taken out of the tile, as zero times them is not zero, and
// added at the end to the rows that see them.
__device__ __forceinline__ bool partial(const AttendParams& p, const volatile Item& w, const Piece& c) {
  const int keys = c.pre ? p.b.prefix_len : min(w.own, w.all_rows), base = c.pre ? 0 : p.b.prefix_len;
  return c.k0 + kSub > keys || (c.k0 < w.low_rows - base && c.k0 + kSub > p.sinks - base);
}

// What depends on the part that a call's kernel takes: picked on the host, so that
// the kernel indexes none of its parameters at run time (by value, as the others have
// them, they would be copied to local memory for that).
struct WindowPart {
  int prefix;    // all of the batch's rows against the prefix
  int splits;
  int joins;     // fp32 sums for the join, or rows of the output
  float* o;
  float2* ml;
};

// Item `id` (a whole warp; false: there are no more).  at, before: the 32
// sequences of the last search and the row blocks before them.
__device__ __forceinline__ bool find_item(const AttendParams& p, const WindowPart& part, int64_t id, int& at, int& before, Item* out) {
  const int splits = part.splits, lane = threadIdx.x & 31;
  const int64_t block = id / (p.kv_heads * splits);
  const int rest = (int)(id % (p.kv_heads * splits));
  // the line's shares: which of its pieces the item takes
  auto share = [&](Item& w) {
    const int pieces = w.prefix.tiles + w.mine.tiles, tiles = (pieces + 1) / 2, per = (tiles + splits - 1) / splits;
    const int t0 = min(tiles, w.split * per), t1 = min(tiles, t0 + per);
    w.piece = 2 * t0;
    w.n = t1 - t0;
    w.n_pieces = max(0, min(2 * w.n, pieces - 2 * t0));
  };
  if (part.prefix) {
    if (lane == 0) {
      Item w;
      w.valid = 1;
      w.s = -1;
      w.first = w.count = w.own = w.all_rows = 0;
      w.rows = p.b.n_tokens * p.group;
      w.r0 = (int)block * 256;
      w.h = rest / splits;
      w.split = rest % splits;
      w.prefix = line_of<kSub>(p, p.b.prefix_len, 0, position_of(p, -1));   // (no token stands before that)
      w.mine = Line{0, 0, 0};
      w.low_rows = p.b.prefix_len;   // (some may see nothing of a piece but first keys)
      share(w);
      *out = w;
    }
    return true;
  }
  for (; at < p.b.n_seqs; at += 32) {
    SeqSpan x{0, 0, 0};
    if (at + lane < p.b.n_seqs) x = seq_span(p.b, at + lane);
    const int n = (x.count * p.group + 255) / 256;
    int end = n;
    for (int d = 1; d < 32; d <<= 1) {
      const int o = __shfl_up_sync(0xffffffffu, end, d);
      if (lane >= d) end += o;
    }
    const uint32_t past = __ballot_sync(0xffffffffu, before + end > block);
    if (!past) {
      before += __shfl_sync(0xffffffffu, end, 31);
      continue;
    }
    const int l = __ffs(past) - 1;
    if (lane != l) return true;
    Item w;
    w.valid = 1;
    w.s = at + l;
    const int rb = n - 1 - (int)(block - (before + end - n));   // the blocks that see the most keys first
    w.first = x.first;
    w.count = x.count;
    w.own = x.own;
    w.rows = x.count * p.group;
    w.r0 = rb * 256;
    w.h = rest / splits;
    w.split = rest % splits;
    const int last = min(w.rows, w.r0 + 256) - 1;   // its last row sees up to the latest position
    const int keys = max(0, x.own - x.count + last / p.group + 1), first = position_of(p, x.own - x.count + w.r0 / p.group);
    w.prefix = line_of<kSub>(p, p.b.prefix_len, 0, first);
    w.mine = line_of<kSub>(p, keys, p.b.prefix_len, first);
    share(w);
    w.all_rows = max(0, x.own - x.count + w.r0 / p.group + 1);
    w.low_rows = position_of(p, x.own - x.count + last / p.group) - p.window + 1;
    *out = w;
    return true;
  }
  return false;
}

template <int D>
__global__ void __launch_bounds__(kWideThreads, 1)
    window_kernel(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap, const AttendParams p,
                  const WindowPart part, const int64_t items) {
  using S = WideShape<D>;
  extern __shared__ uint8_t smem_raw[];
  constexpr int NK = kStagesK<D>, NV = kStagesV<D>;
  __shared__ __align__(8) uint64_t full_k[NK], empty_k[NK], full_v[NV], clean[NV], empty_v[NV], q_full[2], s_full[2], p_full[2][2], pv_done[2], o_full[2], o_free[2],
      item_full[2], item_empty[2], mma_done;
  __shared__ uint32_t tmem_base;
  __shared__ Item item_s[2];
  __shared__ volatile int tainted[2];   // 1 + the item that a value that is not finite was taken out of
  const int tid = threadIdx.x, warp = warp_index(), lane = tid & 31;
  const uint32_t sbase = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t k_ring = sbase + 2 * S::kMat, v_ring = k_ring + NK * S::kMat;
  uint8_t* ring_ptr = smem_raw + (k_ring - smem_u32(smem_raw));
  if (tid == 0) {
    for (int i = 0; i < NK; ++i) {
      mbar_init(&full_k[i], 1);
      mbar_init(&empty_k[i], 1);
    }
    for (int i = 0; i < NV; ++i) {
      mbar_init(&full_v[i], 1);
      mbar_init(&clean[i], 1);
      mbar_init(&empty_v[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&q_full[i], 128);
      mbar_init(&s_full[i], 1);
      for (int j = 0; j < 2; ++j) mbar_init(&p_full[i][j], 128);
      mbar_init(&pv_done[i], 1);
      mbar_init(&o_full[i], 1);
      mbar_init(&o_free[i], 128);
      mbar_init(&item_full[i], 1);
      mbar_init(&item_empty[i], 11);
      tainted[i] = 0;
    }
    mbar_init(&mma_done, 1);
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
  const uint32_t tmem = tmem_base;
  bool ok = true;
  // (the it-th item of this thread block; false: a wait ran out)
  auto item_ready = [&](int it) { return mbar_wait_warp(&item_full[it & 1], (it >> 1) & 1); };
  auto item_done = [&](int it) {
    __syncwarp();
    if (lane == 0) mbar_arrive(&item_empty[it & 1]);
  };
  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 72;\n");
    if (warp == 10) {
      // ------------------------------------------------------------ items
      int at = 0, before = 0;
      for (int it = 0; ok; ++it) {
        if (it >= 2 && !mbar_wait_warp(&item_empty[it & 1], ((it >> 1) - 1) & 1)) {
          ok = false;
          break;
        }
        const int64_t id = blockIdx.x + (int64_t)it * gridDim.x;
        const bool is = id < items && find_item(p, part, id, at, before, &item_s[it & 1]);
        if (!is && lane == 0) item_s[it & 1].valid = 0;
        __syncwarp();
        if (lane == 0) mbar_arrive(&item_full[it & 1]);
        if (!is) break;
      }
    } else if (warp == 11) {
      // ------------------------------------------------------------ values
      for (int it = 0, tile = 0; ok; ++it) {   // tile: of all items so far
        if (!item_ready(it)) {
          ok = false;
          break;
        }
        const volatile Item& w = item_s[it & 1];
        if (!w.valid) break;
        const int n = w.n, n_pieces = w.n_pieces;
        for (int i = 0; i < n && ok; ++i, ++tile) {
          const int vs = tile % NV;
          int look = 0;
          for (int j = 0; j < 2; ++j)
            if (2 * i + j < n_pieces && partial(p, w, piece_at(w, 2 * i + j))) look |= 1 << j;
          ok = mbar_wait_warp(&full_v[vs], (tile / NV) & 1);
          if (!ok) break;
          for (int j = 0; j < 2; ++j) {
            if (!(look >> j & 1)) continue;
            const Piece c = piece_at(w, 2 * i + j);
            const int keys = c.pre ? p.b.prefix_len : w.own;
            const uint32_t at = v_ring + vs * S::kMat + (kSub * j) * 128;   // 16-byte pieces of the rows
            constexpr int kAhead = 8;
#pragma unroll 1
            for (int b = lane; b < 8 * kSub * (D / 64); b += 32 * kAhead) {
              uint4 v[kAhead];
              bool any = false;
#pragma unroll
              for (int k = 0; k < kAhead; ++k) {
                const int e = b + 32 * k;
                v[k] = ld_shared16(at + (e / (8 * kSub)) * kHalf + 16 * (e % (8 * kSub)));
                any |= some_not_finite(v[k]);
              }
              if (!any) continue;
#pragma unroll
              for (int k = 0; k < kAhead; ++k) {
                if (!some_not_finite(v[k])) continue;
                const int e = b + 32 * k;
                if (c.k0 + ((e % (8 * kSub)) >> 3) < keys) tainted[it & 1] = it + 1;
                st_shared16(at + (e / (8 * kSub)) * kHalf + 16 * (e % (8 * kSub)), v[k].x & ~not_finite(v[k].x), v[k].y & ~not_finite(v[k].y),
                            v[k].z & ~not_finite(v[k].z), v[k].w & ~not_finite(v[k].w));
              }
            }
          }
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) mbar_arrive(&clean[vs]);
        }
        item_done(it);
      }
    } else if (warp == 9) {
      // ------------------------------------------------------------ loads
      const int box = 1 << p.box_shift, per_page = 1 << (p.page_shift - p.box_shift), per_piece = kSub >> p.box_shift;
      int tile = 0, issued_k = 0, issued_v = 0;   // of all items so far
      for (int it = 0; ok; ++it) {
        if (!item_ready(it)) {
          ok = false;
          break;
        }
        const volatile Item& w = item_s[it & 1];
        if (!w.valid) break;
        const int n = w.n, n_pieces = w.n_pieces, own = w.own, h = w.h;
        const int32_t* own_table = p.b.pages + (int64_t)max(w.s, 0) * p.b.page_stride;
        // of the lane's box of tile t: is it one (not past the last key), its rows
        auto row_of = [&](int t, bool* is) {
          const int q = 2 * t + lane / per_piece;
          *is = false;
          if (lane >= 2 * per_piece || q >= n_pieces) return -box;
          const Piece c = piece_at(w, q);
          const int at = (c.k0 >> p.box_shift) + lane % per_piece;
          *is = at < (((c.pre ? p.b.prefix_len : own) + box - 1) >> p.box_shift);
          const int pg = *is ? __ldg((c.pre ? p.b.prefix_pages : own_table) + at / per_page) : -1;
          // (a page outside the cache: rows outside the arrays, which read as zeros)
          return pg >= 0 && pg < p.n_pages ? ((pg * p.kv_heads + h) << p.page_shift) + ((at & (per_page - 1)) << p.box_shift) : -box;
        };
        bool is_next = false;
        int y_next = row_of(0, &is_next);
        for (int t = 0; t < n && ok; ++t, ++tile) {
          const int y = y_next;
          const uint32_t boxes = __ballot_sync(0xffffffffu, is_next);
          y_next = row_of(t + 1, &is_next);
#pragma unroll
          for (int kv = 0; kv < 2; ++kv) {
            const int stages = kv ? NV : NK, st = tile % stages, r = tile / stages;
            uint64_t* bar = (kv ? full_v : full_k) + st;
            if (r > 0 && !mbar_wait_warp((kv ? empty_v : empty_k) + st, (r - 1) & 1)) {
              ok = false;
              break;
            }
            mbar_expect_tx_warp(bar, (uint32_t)((__popc(boxes) << p.box_shift) * 128 * (D / 64)));
            (kv ? issued_v : issued_k) = tile + 1;
            for (uint32_t left = boxes; left; left &= left - 1) {
              const int i = __ffs(left) - 1, yi = __shfl_sync(0xffffffffu, y, i);
#pragma unroll
              for (int half = 0; half < D / 64; ++half)
                tma_load_2d_warp(ring_ptr + ((kv ? NK : 0) + st) * S::kMat + half * kHalf + ((i * box) << 7), kv ? &vmap : &kmap, 64 * half, yi, bar);
            }
          }
        }
        item_done(it);
      }
      // the copies in flight have landed before the thread block ends
      for (int j = max(0, issued_k - NK); j < issued_k; ++j)
        if (!mbar_wait_warp(&full_k[j % NK], (j / NK) & 1)) ok = false;
      for (int j = max(0, issued_v - NV); j < issued_v; ++j)
        if (!mbar_wait_warp(&full_v[j % NV], (j / NV) & 1)) ok = false;
    } else if (warp == 8) {
      // --------------------------------------------------------- products
      constexpr uint32_t kF32Bf16 = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(128 >> 4) << 24);   // M = 128
      constexpr uint32_t qk_idesc = kF32Bf16 | ((uint32_t)(kKeys >> 3) << 17);
      constexpr uint32_t pv_idesc = kF32Bf16 | ((uint32_t)(D >> 3) << 17) | (1u << 16);   // B with its N contiguous
      auto scores = [&](int half, int st) {
        const uint64_t a = sw128_desc(sbase + half * S::kMat), b = sw128_desc(k_ring + st * S::kMat);
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const uint64_t off = (uint64_t)((k >> 2) * (kHalf >> 4) + 2 * (k & 3));
          umma_bf16_warp(tmem + 128 * half, a + off, b + off, qk_idesc, k > 0);
        }
        umma_commit_warp(&s_full[half]);
      };
      auto keys_there = [&](int t) { return mbar_wait_warp(&full_k[t % NK], (t / NK) & 1); };
      int tile = 0, tiles[2] = {0, 0}, blocks[2] = {0, 0};   // of all items so far; of a half: tiles, items with tiles
      for (int it = 0; ok; ++it) {
        if (!item_ready(it)) {
          ok = false;
          break;
        }
        const volatile Item& w = item_s[it & 1];
        if (!w.valid) break;
        const int n = w.n, n_pieces = w.n_pieces, halves = w.rows - w.r0 > 128 ? 2 : 1;
        if (n > 0) {
          for (int half = 0; half < halves && ok; ++half) ok = mbar_wait_warp(&q_full[half], blocks[half] & 1);
          if (ok) ok = keys_there(tile);
          if (!ok) break;
          tc_fence_after();
          for (int half = 0; half < halves; ++half) scores(half, tile % NK);
          umma_commit_warp(&empty_k[tile % NK]);
          for (int i = 0; i < n && ok; ++i) {
            const int t = tile + i, vs = t % NV, ks = (t + 1) % NK;
            for (int half = 0; half < halves && ok; ++half) {
              // (the output of the item before has been read)
              if (i == 0 && blocks[half] > 0) ok = mbar_wait_warp(&o_free[half], (blocks[half] - 1) & 1);
#pragma unroll
              for (int j = 0; j < 2; ++j) {
                if (ok) ok = mbar_wait_warp(&p_full[half][j], (tiles[half] + i) & 1);
                if (ok && j + half == 0) ok = mbar_wait_warp(&clean[vs], (t / NV) & 1);
                if (!ok) break;
                tc_fence_after();
                const uint64_t b = sw128_mn_desc(v_ring + vs * S::kMat + j * (kSub * 128));
                if (2 * i + j < n_pieces)   // (the last tile may have one piece)
#pragma unroll
                  for (int k = 0; k < kSub / 16; ++k)
                    umma_bf16_ts_warp(tmem + 256 + D * half, tmem + 128 * half + kSub * j + 8 * k, b + (uint64_t)(k * (2048 >> 4)),
                                      pv_idesc, (i | j | k) != 0);
                if (j == 0) umma_commit_warp(&pv_done[half]);
              }
              if (!ok) break;
              if (half == halves - 1) umma_commit_warp(&empty_v[vs]);
              if (i + 1 < n) {
                if (half == 0) ok = keys_there(t + 1);
                if (!ok) break;
                tc_fence_after();
                scores(half, ks);
                if (half == halves - 1) umma_commit_warp(&empty_k[ks]);
              } else {
                umma_commit_warp(&o_full[half]);
              }
            }
          }
          tile += n;
          for (int half = 0; half < halves; ++half) {
            tiles[half] += n;
            ++blocks[half];
          }
        }
        item_done(it);
      }
      umma_commit_warp(&mma_done);
      if (!mbar_wait_warp(&mma_done, 0)) ok = false;
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 216;\n");
    // ------------------------------------------------------------- softmax
    const int half = warp >> 2, wtid = tid & 127;
    const uint32_t qb = sbase + half * S::kMat;
    const uint32_t ts = tmem + ((uint32_t)(32 * (warp & 3)) << 16) + 128 * half;
    const uint32_t to = tmem + ((uint32_t)(32 * (warp & 3)) << 16) + 256 + D * half;
    const uint64_t scale2 = pair_of(p.scale, p.scale);
    const bool wide_rows = (reinterpret_cast<uintptr_t>(p.out) & 31u) == 0;   // (32 bytes a store)
    bool loading = false;
    // Item it's queries, if this half has some: a warp its 32 rows, a row's
    // chunks by neighbouring lanes (rows past the last: zeros).
    auto load_queries = [&](int it) {
      loading = false;
      if (!item_ready(it)) return false;
      const volatile Item& w = item_s[it & 1];
      const int rows = w.rows, r0 = w.r0, row = r0 + 128 * half + wtid;
      if (!w.valid || w.n == 0 || rows - r0 <= 128 * half) return true;
      loading = true;
      const bool live = row < rows;
      const int tok = row / p.group, g = row - tok * p.group;
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
      return true;
    };
    auto queries_there = [&]() {
      if (!loading) return;
      cp_async_wait_all();
      fence_proxy_async_smem();
      mbar_arrive(&q_full[half]);
    };
    ok = load_queries(0);
    queries_there();
    int tiles = 0, blocks = 0;   // as the products'
    for (int it = 0; ok; ++it) {
      const volatile Item& w = item_s[it & 1];   // (load_queries has waited for it)
      if (!w.valid) break;
      const int n = w.n, n_pieces = w.n_pieces, rows = w.rows, r0 = w.r0;
      if (rows - r0 <= 128 * half) {   // (the second half of a short row block)
        ok = load_queries(it + 1);
        queries_there();
        item_done(it);
        continue;
      }
      const int row = r0 + 128 * half + wtid, tok = row / p.group, g = row - tok * p.group;
      const bool live = row < rows;
      const int own = w.own, behind = own - w.count;   // the place of token 0 of the item's
      // own keys that this row sees, that every row of its half does
      const int lim = live ? behind + tok + 1 : own, all = behind + (r0 + 128 * half) / p.group + 1;
      // the first position of this row's window, and of that of the last row of its half (the latest one); where the
      // rows are several sequences', of its warp's latest
      const int last = min(rows, r0 + 128 * half + 128) - 1;
      auto low_of = [&](int t) { return position_of(p, behind + t) - p.window + 1; };
      int low = 0, low_half;
      if (part.prefix) {
        if (live) {
          const SeqSpan x = seq_span(p.b, seq_of_token(p.b.token_start, p.b.n_seqs, tok));
          low = position_of(p, x.own - x.count + (tok - x.first)) - p.window + 1;
        }
        low_half = __reduce_max_sync(0xffffffffu, low);
      } else {
        if (live) low = low_of(tok);
        low_half = low_of(last / p.group);
      }
      // does piece q need a look at what its keys are?  (Of both pieces of a tile before its scores are waited for:
      // between the scores and the weights every instruction counts)
      auto edge_of = [&](int q) {
        const Piece c = piece_at(w, q);
        const int base = c.pre ? 0 : p.b.prefix_len;
        return c.k0 + kSub > (c.pre ? p.b.prefix_len : all) || (c.k0 < low_half - base && c.k0 + kSub > p.sinks - base);
      };
      int edge = 0;
      float m = -INFINITY;        // reference maximum (log2 units)
      uint64_t l2 = 0;            // two sums
      if (n == 0) ok = load_queries(it + 1);
      for (int q = 0; q < 2 * n && ok; ++q) {
        const int i = q >> 1, j = q & 1;
        if (j == 0) {
          edge = (int)edge_of(q) | (int)edge_of(q + 1) << 1;
          ok = mbar_wait_warp(&s_full[half], (tiles + i) & 1);
          // (the last scores are there: nothing reads the queries any more)
          if (ok && i == n - 1) ok = load_queries(it + 1);
          if (!ok) break;
        }
        if (q >= n_pieces) {      // (a tile of one piece)
          mbar_arrive(&p_full[half][1]);
          break;
        }
        tc_fence_after();
        uint32_t x[kSub];
        tmem_ld32(ts + kSub * j, x);
        tmem_ld32(ts + kSub * j + 32, x + 32);
        tmem_ld_wait();
        if (edge >> j & 1) {
          const Piece c = piece_at(w, q);
          const int k0 = c.k0, keys = c.pre ? p.b.prefix_len : own, base = c.pre ? 0 : p.b.prefix_len;
          if (k0 + kSub > (c.pre ? keys : all)) {
            const int see = (c.pre ? keys : lim) - k0;   // of these 64
#pragma unroll
            for (int k = 0; k < kSub; ++k)
              if (k >= see) x[k] = 0xFF800000u;
          }
          if (k0 < low_half - base && k0 + kSub > p.sinks - base) {
            const int from = p.sinks - base - k0, to_key = low - base - k0;   // of these 64
#pragma unroll
            for (int k = 0; k < kSub; ++k)
              if (k >= from && k < to_key) x[k] = 0xFF800000u;
          }
        }
        float mx[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) mx[c] = max3(__uint_as_float(x[3 * c]), __uint_as_float(x[3 * c + 1]), __uint_as_float(x[3 * c + 2]));
#pragma unroll
        for (int c = 12; c < kSub; c += 2) mx[(c >> 1) & 3] = max3(mx[(c >> 1) & 3], __uint_as_float(x[c]), __uint_as_float(x[c + 1]));
        const float top = max3(mx[0], mx[1], fmaxf(mx[2], mx[3])) * p.scale;
        // The reference is raised where a row's maximum passes it by more than 2^8,
        // and then set kAhead above the maximum: the first keys of a window are few
        // for many rows, and later ones larger.  (Weights and sums are floating:
        // nothing is lost by a reference that lies higher.)
        const bool grow = top > m + 8.f;   // (also from -inf)
        if (__any_sync(0xffffffffu, grow)) {
          constexpr float kAhead = 12.f;
          const float f = grow ? exp2_approx(m - (top + kAhead)) : 1.f;
          if (grow) m = top + kAhead;
          l2 = mul2(l2, pair_of(f, f));
          if (q > 0) {   // once the products so far are in O (those of the tiles before are, with this one's S)
            if (j == 1) ok = mbar_wait_warp(&pv_done[half], (tiles + i) & 1);
            if (!ok) break;
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
      // the next item's scores may begin
      queries_there();
      float l, lb;
      unpair(l2, l, lb);
      l += lb;
      // --------------------------------------------------------------- out
      if (n > 0 && ok) ok = mbar_wait_warp(&o_full[half], blocks & 1);
      if (!ok) break;
      tc_fence_after();
      const bool taint = n > 0 && tainted[it & 1] == it + 1;
      const int64_t at = (int64_t)(w.first + tok) * p.q_heads + w.h * p.group + g;
      const int64_t place = (int64_t)w.split * p.b.n_tokens * p.q_heads + at;
      const float k = l > 0.f ? 1.f / l : l;       // (0 where nothing is seen; NaN stays)
      // (written straight from registers, 32 bytes a store: the place of the
      // queries, through which rows could go, holds the next ones by now)
#pragma unroll 1
      for (int c = 0; c < D / 32; ++c) {
        uint32_t o[32];
        if (n > 0) {
          tmem_ld32(to + 32 * c, o);
          tmem_ld_wait();
          if (c == D / 32 - 1) {
            tc_fence_before();
            mbar_arrive(&o_free[half]);
          }
        } else {
#pragma unroll
          for (int j = 0; j < 32; ++j) o[j] = 0;
        }
        if (taint && live) {
#pragma unroll 1
          for (int q = 0; q < n_pieces; ++q) {
            const Piece pc = piece_at(w, q);
            if (!partial(p, w, pc)) continue;
            const int base = pc.pre ? 0 : p.b.prefix_len, end = min(pc.k0 + kSub, pc.pre ? p.b.prefix_len : lim);
            const int32_t* table = pc.pre ? p.b.prefix_pages : p.b.pages + (int64_t)max(w.s, 0) * p.b.page_stride;
#pragma unroll 1
            for (int key = pc.k0; key < end; ++key) {
              if (key < low - base && key >= p.sinks - base) continue;
              const int pg = __ldg(table + (key >> p.page_shift));
              if (pg < 0 || pg >= p.n_pages) continue;
              const uint32_t* v = reinterpret_cast<const uint32_t*>(
                  p.v + ((((int64_t)pg * p.kv_heads + w.h) << p.page_shift) + (key & ((1 << p.page_shift) - 1))) * D + 32 * c);
#pragma unroll
              for (int j = 0; j < 16; ++j) {
                const uint32_t y = __ldg(v + j), bad = not_finite(y);
                if (bad & 0xFFFFu) o[2 * j] = __float_as_uint(__uint_as_float(o[2 * j]) + __uint_as_float(y << 16));
                if (bad >> 16) o[2 * j + 1] = __float_as_uint(__uint_as_float(o[2 * j + 1]) + __uint_as_float(y & 0xFFFF0000u));
              }
            }
          }
        }
        if (live && part.joins) {
          float* dst = part.o + place * D + 32 * c;
#pragma unroll
          for (int j = 0; j < 4; ++j) st_global32(dst + 8 * j, o + 8 * j);
        } else if (live) {
          uint32_t r[16];
#pragma unroll
          for (int j = 0; j < 16; ++j) r[j] = pack_bf16x2(__uint_as_float(o[2 * j]) * k, __uint_as_float(o[2 * j + 1]) * k);
          uint16_t* dst = p.out + at * D + 32 * c;
          if (wide_rows) {
            st_global32(dst, r);
            st_global32(dst + 16, r + 8);
          } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) reinterpret_cast<uint4*>(dst)[j] = make_uint4(r[4 * j], r[4 * j + 1], r[4 * j + 2], r[4 * j + 3]);
          }
        }
        __syncwarp();   // (whole warps read tensor memory)
      }
      if (live && part.joins) part.ml[place] = make_float2(l == l ? m : l, l);   // (NaN scores leave no maximum)
      if (live && !part.joins && p.lse) p.lse[at] = natural_lse(m, l);
      if (n > 0) {
        tiles += n;
        ++blocks;
      }
      item_done(it);
    }
    cp_async_wait_all();
  }
  if (!ok && lane == 0) call_record_fail(p.rec, p.call);
  tc_fence_before();
  __syncthreads();
  if (warp == 8) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

template <int D>
cudaError_t launch(const sdq_cache_s* c, const AttendParams& p, int part, int64_t items, cudaStream_t st) {
  const bool split = p.splits[part] > 1;
  const WindowPart w{part == kPrefix, p.splits[part], split || p.parts > 1, split ? p.split_o[part] : p.o[part],
                     split ? p.split_ml[part] : p.ml[part]};
  static std::atomic<int> smem_set[64];
  const cudaError_t e = smem_limit_once(window_kernel<D>, WideShape<D>::kSmem, c->device, smem_set);
  if (e != cudaSuccess) return e;
  return launch_pdl(window_kernel<D>, dim3((unsigned)std::min<int64_t>(items, c->sm_count)), dim3(kWideThreads),
                    (size_t)WideShape<D>::kSmem, st, c->kmap, c->vmap, p, w, items);
}

}  // namespace

cudaError_t launch_window(const sdq_cache_s* c, const AttendParams& p, int part, int64_t items, cudaStream_t st) {
  return c->desc.head_dim == 128 ? launch<128>(c, p, part, items, st) : launch<64>(c, p, part, items, st);
}

}  // namespace sdq
