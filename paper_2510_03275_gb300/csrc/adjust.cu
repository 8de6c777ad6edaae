// Logits before the choice of a token: penalties for repeated tokens, biases, a
// grammar's allowed tokens (include/sdq.h).
#include <cmath>
#include <type_traits>

#include "common.cuh"

namespace sdq {

namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kMaxBiases = 4096;
constexpr uint32_t kCount = 0x7FFFFFFFu;   // of a token's word: how often it was answered; the bit above: it has been seen

struct AdjustParams {
  sdq_adjust a;
  const void* in;
  void* out;
  int64_t ld, ldo;
  int vocab;
};

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
template <class T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ uint16_t from_float<uint16_t>(float x) { return (uint16_t)pack_bf16x2(x, 0.f); }

// What a row's tokens meet.
struct Row {
  float repetition, frequency, presence;
  const uint32_t* allowed;   // null: everything is
  __device__ bool may(int t) const { return !allowed || (__ldg(allowed + (t >> 5)) >> (t & 31) & 1u); }
  __device__ float penalized(float z, uint32_t word) const {
    if (word == 0) return z;
    z = z > 0.f ? z / repetition : z * repetition;
    return word & kCount ? z - (frequency * (float)(word & kCount) + presence) : z;
  }
};

// A thread block takes kThreads * kV 16-byte pieces of a row of logits (places
// e of the row, whose first logit is at place `lead` behind a 16-byte
// boundary).  Each logit is read and written once: HBM bounds it.  What the
// history says of the block's tokens is counted in shared memory first (a word
// per token; whole numbers, so that no order of atomics shows); every block of a
// row looks through all of its history, 4 tokens a load.  The few tokens
// with a bias are worked out one by a thread, the list's entries for one token
// added up in their order, and written behind the others.  96 x 128255 fp32
// logits (a copy: 17 us): 34 us, 11 of them for histories of 100 to 32768 tokens
// (their length, their tokens, the logits: chains of latencies that two thread
// blocks per SM hide in part; 16-bit counters, for three, gain nothing), 4 for
// 300 biases, 2 for the grammar; in place 36 (less is written, but a block reads a piece only
// once it knows that it changes); one row of 32000: 3.5.
template <class T, int kV, bool kInPlace>
__global__ void __launch_bounds__(kThreads, kV * 16 / (int)sizeof(T) >= 32 ? 2 : 3) adjust_kernel(const AdjustParams p) {
  constexpr int kVec = 16 / sizeof(T), kChunk = kThreads * kV * kVec;
  extern __shared__ __align__(16) uint32_t smem[];
  uint32_t* seen = smem;                                    // [kChunk]
  int* tok = reinterpret_cast<int*>(smem + kChunk);         // of the biases in this block's range: the token,
  float* add = reinterpret_cast<float*>(tok + p.a.n_bias);  // the bias
  float* res = add + p.a.n_bias;                            // and the logit that comes of it
  __shared__ int counts[kWarps];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int row = blockIdx.x;   // (a row's common tokens, mostly its low ones, are counted first: the last blocks have least to do)
  const T* in = static_cast<const T*>(p.in) + row * p.ld;
  T* out = static_cast<T*>(p.out) + row * p.ldo;
  const int lead = (int)((reinterpret_cast<uintptr_t>(in) & 15u) / sizeof(T));
  const bool even = ((reinterpret_cast<uintptr_t>(in) ^ reinterpret_cast<uintptr_t>(out)) & 15u) == 0;
  const int t0 = (int)blockIdx.y * kChunk - lead, t1 = min(p.vocab, t0 + kChunk);   // tokens (those below 0: none)
  pdl_wait();
  pdl_launch_dependents();
  auto whole = [&](int t) { return even && t >= 0 && t + kVec <= p.vocab; };
  // what the block waits for first, all of it under way at once
  const int set = p.a.allowed ? (p.a.allowed_row ? __ldg(p.a.allowed_row + row) : row) : -1;
  const int len = !p.a.history || t0 >= t1 ? 0 : p.a.history_len ? min(max(__ldg(p.a.history_len + row), 0), p.a.history_max) : p.a.history_max;
  const int prompt = p.a.prompt_len ? __ldg(p.a.prompt_len + row) : 0;
  Row r;
  r.repetition = p.a.repetition ? __ldg(p.a.repetition + row) : 1.f;
  r.frequency = p.a.frequency ? __ldg(p.a.frequency + row) : 0.f;
  r.presence = p.a.presence ? __ldg(p.a.presence + row) : 0.f;
  r.allowed = set >= 0 && set < p.a.n_allowed ? p.a.allowed + set * p.a.allowed_stride : nullptr;
  // the history: places 0 .. head - 1 lie before a 16-byte boundary, the last ones behind whole pieces
  const int32_t* h = p.a.history + row * p.a.history_stride;
  const int head = min(len, (int)(-(reinterpret_cast<uintptr_t>(h) >> 2) & 3u)), pieces = (len - head) / 4;
  const int4* h4 = reinterpret_cast<const int4*>(h + head);
  constexpr int kAhead = 4;
  int4 ids[kAhead];
  auto load_ids = [&](int i0) {
#pragma unroll
    for (int k = 0; k < kAhead; ++k) ids[k] = i0 + k * kThreads < pieces ? __ldg(h4 + i0 + k * kThreads) : make_int4(-1, -1, -1, -1);
  };
  load_ids(tid);
  // of this thread's logits, which the grammar allows: kVec bits for each piece
  uint32_t open = ~0u;
  static_assert(kV * kVec <= 32, "a word per thread");
  if (r.allowed) {
    open = 0;
    const int last = (p.vocab - 1) >> 5;
#pragma unroll
    for (int v = 0; v < kV; ++v) {
      const int t = t0 + (v * kThreads + tid) * kVec, b = min(max(t, 0) >> 5, last);
      const uint32_t lo = __ldg(r.allowed + b), hi = __ldg(r.allowed + min(b + 1, last));
      open |= ((t >= 0 ? __funnelshift_r(lo, hi, t & 31) : lo << (-t & 31)) & ((1u << kVec) - 1)) << (kVec * v);
    }
  }
  if (p.a.history) {
    for (int i = tid; i < kChunk / 4; i += kThreads) reinterpret_cast<uint4*>(seen)[i] = make_uint4(0, 0, 0, 0);
    __syncthreads();
    const uint32_t width = (uint32_t)max(t1 - max(t0, 0), 0), low = (uint32_t)max(t0, 0);
    auto count = [&](int i, int t) {
      if ((uint32_t)t - low >= width) return;   // (also below 0)
      if (i < prompt) atomicOr(seen + (t - t0), ~kCount);
      else atomicAdd(seen + (t - t0), 1u);
    };
    for (int i0 = tid; i0 < pieces; i0 += kAhead * kThreads, load_ids(i0)) {
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int i = head + 4 * (i0 + k * kThreads);
        count(i, ids[k].x);
        count(i + 1, ids[k].y);
        count(i + 2, ids[k].z);
        count(i + 3, ids[k].w);
      }
    }
    if (tid < head) count(tid, __ldg(h + tid));
    const int i = head + 4 * pieces + tid - 4;
    if (tid >= 4 && i < len) count(i, __ldg(h + i));
  }
  // biases of tokens in this block's range, in the list's order
  int n = 0;
  for (int i0 = 0; i0 < p.a.n_bias; i0 += kThreads) {
    const int i = i0 + tid, t = i < p.a.n_bias ? __ldg(p.a.bias_ids + row * p.a.bias_ids_stride + i) : -1;
    const bool here = t >= 0 && t >= t0 && t < t1;
    const uint32_t which = __ballot_sync(0xffffffffu, here);
    __syncthreads();   // (counts of the pieces before are read)
    if (lane == 0) counts[warp] = __popc(which);
    __syncthreads();
    int at = n;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      if (w < warp) at += counts[w];
      n += counts[w];
    }
    if (here) {
      at += __popc(which & ((1u << lane) - 1));
      tok[at] = t;
      add[at] = __ldg(p.a.bias + row * p.a.bias_stride + i);
    }
  }
  __syncthreads();
  for (int e = tid; e < n; e += kThreads) {
    const int t = tok[e];
    const float z = to_float(in[t]);
    float sum = 0.f;
#pragma unroll 8
    for (int k = 0; k < n; ++k)
      if (tok[k] == t) sum += add[k];
    res[e] = r.may(t) ? r.penalized(z, p.a.history ? seen[t - t0] : 0) + sum : -INFINITY;   // (entries of one token: the same)
  }
  if (n > 0) __syncthreads();
  // (4 pieces of the logits under way at once: held from the kernel's start they
  // cost registers, and with them thread blocks of an SM: 2 of them for large
  // chunks, 3 for small ones; 32 x 50272 in bf16 7.2 us, with 2 or 4 8.5)
  constexpr int kAtOnce = kV < 4 ? kV : 4;
#pragma unroll 1
  for (int v0 = 0; v0 < kV; v0 += kAtOnce) {
    uint4 x[kAtOnce];
    if (!kInPlace) {
#pragma unroll
      for (int v = 0; v < kAtOnce; ++v) {
        const int t = t0 + ((v0 + v) * kThreads + tid) * kVec;
        if (whole(t)) x[v] = __ldg(reinterpret_cast<const uint4*>(in + t));
      }
    }
#pragma unroll
    for (int v = 0; v < kAtOnce; ++v) {
      const int at = ((v0 + v) * kThreads + tid) * kVec, t = t0 + at;
      if (t >= t1 || t + kVec <= 0) continue;
      uint32_t w[kVec], any = 0;
#pragma unroll
      for (int j = 0; j < kVec; j += 4) {
        const uint4 q = p.a.history ? *reinterpret_cast<const uint4*>(seen + at + j) : make_uint4(0, 0, 0, 0);
        w[j] = q.x;
        w[j + 1] = q.y;
        w[j + 2] = q.z;
        w[j + 3] = q.w;
        any |= q.x | q.y | q.z | q.w;
      }
      const uint32_t bits = open >> (kVec * (v0 + v));
      const bool all = (~bits & ((1u << kVec) - 1)) == 0;
      if (kInPlace && any == 0 && all) continue;
      if (whole(t)) {
        if (kInPlace) x[v] = *reinterpret_cast<const uint4*>(in + t);
        if (any != 0 || !all) {
          T z[kVec];
          memcpy(z, &x[v], 16);
#pragma unroll
          for (int j = 0; j < kVec; ++j) {
            if (w[j]) z[j] = from_float<T>(r.penalized(to_float(z[j]), w[j]));
            if (!(bits >> j & 1u)) z[j] = from_float<T>(-INFINITY);
          }
          memcpy(&x[v], z, 16);
        }
        *reinterpret_cast<uint4*>(out + t) = x[v];
      } else {
#pragma unroll
        for (int j = 0; j < kVec; ++j) {
          if (t + j < 0 || t + j >= p.vocab) continue;
          T z = in[t + j];
          if (w[j]) z = from_float<T>(r.penalized(to_float(z), w[j]));
          if (!(bits >> j & 1u)) z = from_float<T>(-INFINITY);
          out[t + j] = z;
        }
      }
    }
  }
  if (n > 0) __syncthreads();
  for (int e = tid; e < n; e += kThreads) out[tok[e]] = from_float<T>(res[e]);
}

template <class T, int kV, bool kInPlace>
cudaError_t launch(const AdjustParams& p, int rows, int device, cudaStream_t st) {
  constexpr int kVec = 16 / sizeof(T), kChunk = kThreads * kV * kVec;
  static std::atomic<int> smem_set[64];
  const cudaError_t e = smem_limit_once(adjust_kernel<T, kV, kInPlace>, 4 * kChunk + 12 * kMaxBiases, device, smem_set);
  if (e != cudaSuccess) return e;
  const dim3 grid((unsigned)rows, (unsigned)((p.vocab + kVec - 1 + kChunk - 1) / kChunk));
  return launch_pdl(adjust_kernel<T, kV, kInPlace>, grid, dim3(kThreads), 4 * (size_t)kChunk + 12 * (size_t)p.a.n_bias, st, p);
}

}  // namespace

}  // namespace sdq

using namespace sdq;

extern "C" int sdq_adjust_logits(const void* logits, int32_t type, int32_t rows, int32_t vocab, int64_t ld, const sdq_adjust* a,
                                 void* out, int64_t ldo, void* stream) {
  if (!logits || !a || !out || (type != SDQ_F32 && type != SDQ_BF16)) return SDQ_ERR_INVALID_ARG;
  if (rows < 1 || rows > 65535 || vocab < 1 || vocab > 393216 || ld < vocab || ldo < vocab) return SDQ_ERR_INVALID_ARG;
  const uintptr_t size = type == SDQ_F32 ? 4 : 2, in_at = reinterpret_cast<uintptr_t>(logits), out_at = reinterpret_cast<uintptr_t>(out);
  if (in_at % size || out_at % size) return SDQ_ERR_INVALID_ARG;
  const bool in_place = in_at == out_at && (rows == 1 || ld == ldo);
  if (!in_place && in_at < out_at + size * ((uintptr_t)(rows - 1) * ldo + vocab) &&
      out_at < in_at + size * ((uintptr_t)(rows - 1) * ld + vocab))
    return SDQ_ERR_INVALID_ARG;
  if (a->history_stride < 0 || a->bias_ids_stride < 0 || a->bias_stride < 0 || a->allowed_stride < 0) return SDQ_ERR_INVALID_ARG;
  if ((a->history && a->history_max < 0) || a->n_bias < 0 || a->n_bias > kMaxBiases) return SDQ_ERR_INVALID_ARG;
  if (a->n_bias > 0 && (!a->bias_ids || !a->bias)) return SDQ_ERR_INVALID_ARG;
  if (a->allowed && a->n_allowed < (a->allowed_row ? 1 : rows)) return SDQ_ERR_INVALID_ARG;
  int dev = -1, sms = 0;
  const int supported = supported_device(&dev, &sms);
  if (supported != SDQ_OK) return supported;
  AdjustParams p;
  p.a = *a;
  p.in = logits; p.out = out;
  p.ld = ld; p.ldo = ldo;
  p.vocab = vocab;
  cudaStream_t st = (cudaStream_t)stream;
  // 16384 logits a thread block where the rows fill the device with that, else 4096
  const bool large = (int64_t)rows * ((vocab + 16383) / 16384) >= 2 * sms;
  auto run = [&](auto zero, auto place) {
    using T = decltype(zero);
    constexpr int kVec = 16 / sizeof(T);
    constexpr bool kInPlace = decltype(place)::value;
    return large ? launch<T, 16384 / kVec / kThreads, kInPlace>(p, rows, dev, st) : launch<T, 4096 / kVec / kThreads, kInPlace>(p, rows, dev, st);
  };
  const std::true_type yes;
  const std::false_type no;
  const cudaError_t e = type == SDQ_F32 ? in_place ? run(0.f, yes) : run(0.f, no) : in_place ? run((uint16_t)0, yes) : run((uint16_t)0, no);
  return e == cudaSuccess ? SDQ_OK : SDQ_ERR_CUDA;
}
