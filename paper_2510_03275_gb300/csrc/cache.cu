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
  int per_part;   // 8-element units of a token that one block of a part takes
};

// Four consecutive elements in fp32.
__device__ __forceinline__ float4 load4(const float* p) { return __ldg(reinterpret_cast<const float4*>(p)); }
__device__ __forceinline__ float4 load4(const uint16_t* p) {
  const uint2 r = __ldg(reinterpret_cast<const uint2*>(p));
  return make_float4(__uint_as_float(r.x << 16), __uint_as_float(r.x & 0xFFFF0000u), __uint_as_float(r.y << 16),
                     __uint_as_float(r.y & 0xFFFF0000u));
}
__device__ __forceinline__ void store4(uint16_t* p, float4 a) {
  *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(a.x, a.y), pack_bf16x2(a.z, a.w));
}

// Every element is read once and written once, rounded to bf16 there; what
// bounds it is HBM for prompts and the launch for single tokens.  A thread
// takes 8 elements of one head: 4 and their 4 partners dim / 2 further on, or
// 8 neighbours, so that both halves of a pair are in its registers.  grid.x:
// tokens, grid.y: parts of a token's heads.  2566 tokens of 64 + 2 x 8 heads of
// 128, fp32: 28 us (84 % of the measured copy bandwidth); one token: 1.8 us (a
// graph of 30 calls).
template <class T>
__global__ void __launch_bounds__(kThreads) append_kernel(AppendParams p) {
  pdl_wait();
  pdl_launch_dependents();
  const int t = blockIdx.x, per_head = p.dim / 8, half = p.rope.dim / 2;
  const int s = seq_of_token(p.b.token_start, p.b.n_seqs, t);
  const SeqSpan q = seq_span(p.b, s);
  const int at = q.own - q.count + (t - q.first);
  const int pos = max(0, p.b.prefix_len + min(at, q.own - 1));   // (min: a token beyond max_new has no place of its own)
  int page = -1;
  if (t < q.first + q.count && at >= 0 && at < q.own) page = __ldg(p.b.pages + (int64_t)s * p.b.page_stride + at / p.page);
  const bool keep = page >= 0 && page < p.n_pages;
  const int units = (p.q_heads + 2 * p.kv_heads) * per_head;
  const int end = min(units, ((int)blockIdx.y + 1) * p.per_part);
  for (int u = blockIdx.y * p.per_part + threadIdx.x; u < end; u += kThreads) {
    const int h = u / per_head, c = u - h * per_head;
    const bool is_q = h < p.q_heads, is_v = h >= p.q_heads + p.kv_heads;
    const int kh = is_v ? h - p.q_heads - p.kv_heads : h - p.q_heads;
    const T* src = is_q   ? static_cast<const T*>(p.q) + t * p.ldq + h * p.dim
                   : is_v ? static_cast<const T*>(p.v) + t * p.ldv + kh * p.dim
                          : static_cast<const T*>(p.k) + t * p.ldk + kh * p.dim;
    const bool turn = !is_v && 8 * c < p.rope.dim;
    const bool split = turn && !p.rope.interleaved;
    const int ea = split ? 4 * c : 8 * c, eb = split ? 4 * c + half : 8 * c + 4;
    float4 a = load4(src + ea), b = load4(src + eb);
    if (turn) {
      const float4 cs = load4(p.rope.cos + (int64_t)pos * half + 4 * c);
      const float4 sn = load4(p.rope.sin + (int64_t)pos * half + 4 * c);
      if (split) {
        const float4 x = a, y = b;
        a = make_float4(x.x * cs.x - y.x * sn.x, x.y * cs.y - y.y * sn.y, x.z * cs.z - y.z * sn.z, x.w * cs.w - y.w * sn.w);
        b = make_float4(y.x * cs.x + x.x * sn.x, y.y * cs.y + x.y * sn.y, y.z * cs.z + x.z * sn.z, y.w * cs.w + x.w * sn.w);
      } else {
        const float4 x = a, y = b;
        a = make_float4(x.x * cs.x - x.y * sn.x, x.y * cs.x + x.x * sn.x, x.z * cs.y - x.w * sn.y, x.w * cs.y + x.z * sn.y);
        b = make_float4(y.x * cs.z - y.y * sn.z, y.y * cs.z + y.x * sn.z, y.z * cs.w - y.w * sn.w, y.w * cs.w + y.z * sn.w);
      }
    }
    uint16_t* dst;
    if (is_q) {
      dst = p.q_out + ((int64_t)t * p.q_heads + h) * p.dim;
    } else {
      if (!keep) continue;
      dst = (is_v ? p.vp : p.kp) + (((int64_t)page * p.kv_heads + kh) * p.page + at % p.page) * p.dim;
    }
    store4(dst + ea, a);
    store4(dst + eb, b);
  }
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

extern "C" int sdq_cache_append(sdq_cache c, const sdq_batch* b, int32_t q_heads, const void* q, int64_t ldq,
                                const void* k, int64_t ldk, const void* v, int64_t ldv, int32_t type,
                                const sdq_rope* rope, uint16_t* q_out, void* stream) {
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
  AppendParams p;
  p.b = *b;
  p.rope = *rope;
  p.q = q; p.k = k; p.v = v;
  p.ldq = ldq; p.ldk = ldk; p.ldv = ldv;
  p.kp = c->k; p.vp = c->v; p.q_out = q_out;
  p.q_heads = q_heads; p.kv_heads = c->desc.kv_heads; p.dim = d; p.page = c->desc.page_tokens; p.n_pages = c->desc.n_pages;
  const int units = (q_heads + 2 * c->desc.kv_heads) * (d / 8);
  const int parts = std::max(1, std::min((units + kThreads - 1) / kThreads, 2 * c->sm_count / b->n_tokens));
  p.per_part = ((units + parts - 1) / parts + kThreads - 1) / kThreads * kThreads;
  const dim3 grid((unsigned)b->n_tokens, (unsigned)((units + p.per_part - 1) / p.per_part));
  const cudaError_t e = type == SDQ_F32
                            ? launch_pdl(append_kernel<float>, grid, dim3(kThreads), 0, (cudaStream_t)stream, p)
                            : launch_pdl(append_kernel<uint16_t>, grid, dim3(kThreads), 0, (cudaStream_t)stream, p);
  return e == cudaSuccess ? SDQ_OK : SDQ_ERR_CUDA;
}
