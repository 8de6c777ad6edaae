// Attention over the paged cache: which kernel takes what, the workspace, the
// entry points (include/sdq.h).
#include <algorithm>
#include <cmath>

#include "attention.cuh"

namespace sdq {

namespace {

// One warp per row: the prefix's results, then the own part's, one for each
// thread block that shared a row block's keys, in this order; kBatch pieces under
// way at once.  L2 bounds it, or the launch: 4096 rows of 7 + 1 parts 5 us.
template <int D>
__global__ void __launch_bounds__(256) join_kernel(const AttendParams p) {
  pdl_wait();
  pdl_launch_dependents();
  constexpr int V = D / 32, kBatch = 4;
  const int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5), rows = (int64_t)p.b.n_tokens * p.q_heads;
  if (row >= rows) return;
  // (a token that no sequence counts as its own has no own result: seq_span)
  const int tok = (int)(row / p.q_heads);
  const SeqSpan q = seq_span(p.b, seq_of_token(p.b.token_start, p.b.n_seqs, tok));
  const bool own = tok < q.first + q.count;
  const int np = p.narrow[kPrefix] + max(p.wide[kPrefix], p.splits[kPrefix]);
  const int n = np + (own ? p.narrow[kOwn] + max(p.wide[kOwn], p.splits[kOwn]) : 0);
  float acc[V], sum = 0.f, top = -INFINITY;
#pragma unroll
  for (int k = 0; k < V; ++k) acc[k] = 0.f;
#pragma unroll 1
  for (int i0 = 0; i0 < n; i0 += kBatch) {
    float2 ml[kBatch];
    float v[kBatch][V];
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const int i = min(i0 + j, n - 1), part = i < np ? kPrefix : kOwn, at = i < np ? i : i - np;
      const bool split = p.splits[part] > 1;
      const int64_t place = (split ? at * rows : 0) + row;
      ml[j] = __ldcg((split ? p.split_ml[part] : p.ml[part]) + place);
      load_row<D, V>((split ? p.split_o[part] : p.o[part]) + place * D, v[j]);
    }
    float now = top;
#pragma unroll
    for (int j = 0; j < kBatch; ++j) now = fmaxf(now, ml[j].x);
    const float base = now == -INFINITY ? 0.f : now, old = exp2_approx(top - base);   // (0 before the first)
    top = now;
    sum *= old;
#pragma unroll
    for (int k = 0; k < V; ++k) acc[k] *= old;
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const float f = i0 + j < n ? exp2_approx(ml[j].x - base) : 0.f;
      if (f == 0.f) continue;   // (a part that saw nothing holds anything)
      sum += ml[j].y * f;
#pragma unroll
      for (int k = 0; k < V; ++k) acc[k] += f * v[j][k];
    }
  }
  write_row<D, V>(p, row, acc, top, sum);
}

// ------------------------------------------------------------------- host
// A prefix's rows go to the wide kernel from 9 on (16 rows of 32 heads against
// 2051 keys: 15.6 us, 20.6 on the narrow one, whose warps then hold 16 rows each
// and spend more on them than on the keys), a sequence's from 33 on, since the wide
// kernel takes a thread block for every 256 of them, or fewer.  Where a sequence
// brings 128 rows and more on the average, its row blocks run over the prefix
// and its own keys in one line; below that the batch's rows share blocks against
// the prefix, and the two parts' results are joined.
constexpr int kPrefixNarrowRows = 8;

void set_route(const sdq_cache_s* c, const sdq_batch* b, int q_heads, AttendParams* p) {
  const int group = q_heads / c->desc.kv_heads;
  const int64_t own_rows = b->max_own > 0 ? (int64_t)b->max_new * group : 0;
  const int64_t prefix_rows = b->prefix_len > 0 ? (int64_t)b->n_tokens * group : 0;
  const bool own_wide = own_rows > kNarrowRows;
  p->b = *b;
  p->group = group;
  p->group_inverse = 65536u / (uint32_t)group + 1;
  p->chained = own_wide && prefix_rows > 0 && prefix_rows >= 128ll * b->n_seqs;
  p->wide[kOwn] = own_wide;
  // (a call without any keys goes through the narrow kernel too: it writes the zeros)
  p->narrow[kOwn] = !own_wide && (own_rows > 0 || prefix_rows == 0);
  p->wide[kPrefix] = prefix_rows > kPrefixNarrowRows && !p->chained;
  p->narrow[kPrefix] = prefix_rows > 0 && prefix_rows <= kPrefixNarrowRows;
  p->parts = p->wide[kOwn] + p->narrow[kOwn] + p->wide[kPrefix] + p->narrow[kPrefix];
  for (int part = 0; part < 2; ++part) {
    p->splits[part] = p->wide[part] ? wide_splits(c, b, q_heads, part, p->chained, part == kPrefix && p->narrow[kOwn]) : 0;
  }
  p->ctas = c->sm_count;
  // Beside a wide kernel that leaves SMs free, the narrow one's first thread
  // blocks start at once and the others as the wide kernel's end: the first
  // take ahead what they can read until then (40 bytes a ns and SM).
  if (p->wide[kPrefix] && p->narrow[kOwn]) {
    p->early = c->sm_count - (int)std::min<int64_t>(wide_grid(c, *p, kPrefix), c->sm_count);
    p->ahead = (int)((wide_time(c, b, q_heads, kPrefix, false, p->splits[kPrefix]) + kNarrowStart) * 40e3 / (64.0 * c->desc.head_dim * narrow_warps()));
  }
}

AttendWs attend_workspace(const sdq_cache_s* c, const sdq_batch* b, int q_heads, const AttendParams& p) {
  const size_t rows = (size_t)b->n_tokens * q_heads, d = c->desc.head_dim;
  AttendWs L{};
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off = (off + bytes + 255) / 256 * 256;
    return at;
  };
  L.rec = take(4 * sizeof(uint64_t));
  L.tickets[kOwn] = take(p.narrow[kOwn] ? sizeof(uint64_t) * b->n_seqs * c->desc.kv_heads : 0);
  L.tickets[kPrefix] = take(p.narrow[kPrefix] ? sizeof(uint64_t) * c->desc.kv_heads : 0);
  for (int part = 0; part < 2; ++part) {
    L.ml[part] = take(p.parts > 1 && p.splits[part] <= 1 ? sizeof(float2) * rows : 0);
    L.o[part] = take(p.parts > 1 && p.splits[part] <= 1 ? sizeof(float) * rows * d : 0);
    L.split_ml[part] = take(p.splits[part] > 1 ? sizeof(float2) * p.splits[part] * rows : 0);
    L.split_o[part] = take(p.splits[part] > 1 ? sizeof(float) * p.splits[part] * rows * d : 0);
    const size_t slots = p.narrow[part] ? (size_t)p.ctas * 8 * narrow_groups(b, p.group, part) : 0;
    L.warp_o[part] = take(sizeof(float) * slots * narrow_warps() * d);
    L.block_ml[part] = take(sizeof(float2) * 2 * slots);
    L.block_o[part] = take(sizeof(float) * 2 * slots * d);
  }
  L.total = off;
  return L;
}

template <int D>
cudaError_t launch_join(const AttendParams& p, cudaStream_t st) {
  const int64_t rows = (int64_t)p.b.n_tokens * p.q_heads;
  return launch_pdl(join_kernel<D>, dim3((unsigned)((rows + 7) / 8)), dim3(256), 0, st, p);
}

cudaError_t launch_parts(const sdq_cache_s* c, const AttendParams& p, cudaStream_t st) {
  cudaError_t e = cudaSuccess;
  for (int part = kPrefix; part >= kOwn && e == cudaSuccess; --part) {
    if (p.wide[part]) e = launch_wide(c, p, part, st);
    else if (p.narrow[part]) e = launch_narrow(c, p, part, part == kOwn && p.parts > 1, st);
  }
  if (e != cudaSuccess || (p.parts == 1 && p.splits[kOwn] <= 1 && p.splits[kPrefix] <= 1)) return e;
  return c->desc.head_dim == 128 ? launch_join<128>(p, st) : launch_join<64>(p, st);
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
  set_route(c, b, q_heads, &p);
  return attend_workspace(c, b, q_heads, p).total;
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
  set_route(c, b, q_heads, &p);
  const AttendWs L = attend_workspace(c, b, q_heads, p);
  if (ws_bytes < L.total) return SDQ_ERR_WORKSPACE;
  uint8_t* w = static_cast<uint8_t*>(ws);
  p.q = q; p.v = c->v; p.ldq = ldq; p.out = out; p.lse = lse;
  p.scale = scale * 1.44269504089f;
  p.q_heads = q_heads; p.kv_heads = c->desc.kv_heads;
  p.page_shift = log2_of(c->desc.page_tokens);
  p.box_shift = log2_of(cache_box_rows(c->desc));
  p.n_pages = c->desc.n_pages;
  p.rec = reinterpret_cast<uint64_t*>(w + L.rec);
  p.call = call_tag(next_call_number());
  for (int part = 0; part < 2; ++part) {
    p.tickets[part] = reinterpret_cast<uint64_t*>(w + L.tickets[part]);
    p.o[part] = reinterpret_cast<float*>(w + L.o[part]);
    p.ml[part] = reinterpret_cast<float2*>(w + L.ml[part]);
    p.split_o[part] = reinterpret_cast<float*>(w + L.split_o[part]);
    p.split_ml[part] = reinterpret_cast<float2*>(w + L.split_ml[part]);
    p.warp_o[part] = reinterpret_cast<float*>(w + L.warp_o[part]);
    p.block_o[part] = reinterpret_cast<float*>(w + L.block_o[part]);
    p.block_ml[part] = reinterpret_cast<float2*>(w + L.block_ml[part]);
  }
  const cudaError_t e = launch_parts(c, p, (cudaStream_t)stream);
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
