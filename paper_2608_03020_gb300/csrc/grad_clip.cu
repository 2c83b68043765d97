// Global norm of many gradient tensors and their clipping:
//   norm = sqrt(sum_t sum_i g_t[i]^2),  out_t = f g_t,  f = max_norm / norm if norm > max_norm, else 1
//
// Two launches per up to kMany tensors, whatever their number and sizes: the list of tensors travels
// in the kernel's parameters, cut into chunks of kChunk elements that the blocks take in turn, each
// thread with its part of a chunk in registers before it uses the first of it.
//   k_clip_sumsq   squares summed in fp32 over the (at most 34) elements of a thread and chunk, everything
//                  above in fp64, in a fixed order; a thread whose fp32 sum leaves the range in which it
//                  is exact enough (overflow, squares near the smallest normal) sums them again in fp64
//   k_clip_scale   every block adds the partial sums in the same order and scales its chunks, the last
//                  ones first: they are the ones still in L2.  In place with f = 1 nothing is written
// Bound: HBM, one read for the norm, and the second read (as far as L2 does not hold it) and one write
// for the clipping; launch latency below a few MB.  15.7 million fp32 and 101 million bf16 elements: 131 us
// for three passes over 264 MB (6.0 TB/s), in place 124 us, 63 with f = 1; 48 tensors of 7168 fp32 elements
// 5.9 us.  An output that shares no 16-byte boundary with its input: 81 million bf16 88 us, 77 with one.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstring>

#include "loca_internal.h"
#include "tc_ptx.cuh"

namespace loca {
namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 8192;
constexpr int kSumBlocks = 4, kScaleBlocks = 6;  // resident blocks per SM
constexpr int kFew = 64;     // tensors of one launch: a small list keeps the launch short
constexpr int kMany = 1000;  // 28 KB of parameters

template <int kCap>
struct List {
  const void* in[kCap];
  void* out[kCap];
  int64_t numel_type[kCap];   // 2 numel + (1 if bf16)
  int32_t chunk_end[kCap];    // chunks up to and including this tensor's
  int32_t n;
  int32_t chunks;
};

static_assert(sizeof(List<kMany>) + 64 <= 32764, "a launch's parameters");

struct Chunk {
  int t;
  int64_t first;
  int count;
  bool bf16;
};
template <int kCap>
__device__ __forceinline__ Chunk chunk_of(const List<kCap>& l, int c) {
  int lo = 0, hi = l.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    if (l.chunk_end[mid] > c) hi = mid;
    else lo = mid + 1;
  }
  Chunk k;
  k.t = lo;
  k.bf16 = (l.numel_type[lo] & 1) != 0;
  const int64_t numel = l.numel_type[lo] >> 1;
  k.first = int64_t(c - (lo ? l.chunk_end[lo - 1] : 0)) * kChunk;
  k.count = int(numel - k.first < kChunk ? numel - k.first : kChunk);
  if (!LOCA_CHECK_SPAN(k.first, k.count, numel)) k.count = 0;
  return k;
}

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }

// This thread's share of a chunk: 16-byte vectors, all loaded before the first is used, and the single
// elements before and behind them.
template <class T>
struct Share {
  static constexpr int kVec = 16 / sizeof(T);
  static constexpr int kIter = kChunk / (kVec * kThreads);
  const T* p;
  int count, head, vecs;
  uint4 q[kIter];

  __device__ __forceinline__ Share(const T* p_, int count_) : p(p_), count(count_) {
    head = int((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / int(sizeof(T));
    if (head > count) head = count;
    vecs = (count - head) / kVec;
#pragma unroll
    for (int j = 0; j < kIter; ++j) {
      const int i = j * kThreads + int(threadIdx.x);
      q[j] = i < vecs ? __ldg(reinterpret_cast<const uint4*>(p + head) + i) : make_uint4(0, 0, 0, 0);
    }
  }
  // f(index) over this thread's single elements
  template <class F>
  __device__ __forceinline__ void singles(F&& f) const {
    for (int i = threadIdx.x; i < head; i += kThreads) f(i);
    for (int i = head + vecs * kVec + int(threadIdx.x); i < count; i += kThreads) f(i);
  }
};

template <class T>
__device__ __forceinline__ double sum_squares(const T* p, int count) {
  const Share<T> c(p, count);
  float s = 0.f;
#pragma unroll
  for (int j = 0; j < Share<T>::kIter; ++j) {
    const T* v = reinterpret_cast<const T*>(&c.q[j]);
#pragma unroll
    for (int i = 0; i < Share<T>::kVec; ++i) s = fmaf(to_f(v[i]), to_f(v[i]), s);
  }
  c.singles([&](int i) { s = fmaf(to_f(p[i]), to_f(p[i]), s); });
  if (s >= 1e-30f && s <= 1e38f) return double(s);
  double d = 0.0;
  for (int j = 0; j < Share<T>::kIter; ++j) {
    const T* v = reinterpret_cast<const T*>(&c.q[j]);
    for (int i = 0; i < Share<T>::kVec; ++i) d = fma(double(to_f(v[i])), double(to_f(v[i])), d);
  }
  c.singles([&](int i) { d = fma(double(to_f(p[i])), double(to_f(p[i])), d); });
  return d;
}

__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// sqrt(s) and the factor.  The chip adds two doubles a cycle and SM: a double square root and division in
// every block took 15 us of 25 at 4 million elements.  The root is taken of the leading 24 bits of
// s 4^-e in [1, 4), and one Newton step with the exact remainder leaves it, and likewise the quotient,
// within 2^-40 before its one rounding to fp32.
__device__ __forceinline__ void norm_and_factor(double s, float max_norm, float& norm, float& f) {
  f = 1.f;
  if (!(s < INFINITY)) {  // infinite: every finite element becomes 0; NaN: nothing is scaled
    norm = float(s);
    if (s > 0.0) f = max_norm < INFINITY ? 0.f : 1.f;
    return;
  }
  norm = 0.f;
  if (!(s > 0.0)) return;
  const int e = ((__double2hiint(s) >> 20) - 1023) >> 1;  // s is a normal double: squares of fp32 values
  const double m = __hiloint2double(__double2hiint(s) - e * (1 << 21), __double2loint(s));
  const float mh = float(m), ml = float(m - double(mh));
  const float r = sqrtf(mh);
  const float lo = (fmaf(-r, r, mh) + ml) / (2.f * r);
  norm = ldexpf(r + lo, e);
  if (s > double(max_norm) * double(max_norm)) {
    const float q = max_norm / r;
    f = ldexpf(q + (fmaf(-q, r, max_norm) - q * lo) / r, -e);
  }
}

template <int kCap>
__global__ void __launch_bounds__(kThreads, kSumBlocks) k_clip_sumsq(const __grid_constant__ List<kCap> l, double* part) {
  __shared__ double sh[kThreads];
  tc::wait_for_previous();
  tc::launch_dependents();
  double s = 0.0;
  for (int c = blockIdx.x; c < l.chunks; c += gridDim.x) {
    const Chunk k = chunk_of(l, c);
    s += k.bf16 ? sum_squares(static_cast<const __nv_bfloat16*>(l.in[k.t]) + k.first, k.count)
                : sum_squares(static_cast<const float*>(l.in[k.t]) + k.first, k.count);
  }
  sh[threadIdx.x] = s;
  __syncthreads();
  if (threadIdx.x >= 32) return;
  s = 0.0;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) s += sh[32 * w + threadIdx.x];
  s = warp_sum(s);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

template <class T>
__device__ __forceinline__ T from_f(float x);
template <>
__device__ __forceinline__ float from_f<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

template <class T>
__device__ __forceinline__ uint4 scaled(uint4 q, float f) {
  T* v = reinterpret_cast<T*>(&q);
#pragma unroll
  for (int e = 0; e < 16 / int(sizeof(T)); ++e) v[e] = from_f<T>(f * to_f(v[e]));
  return q;
}

template <class T>
__device__ __forceinline__ void scale_chunk(const T* p, T* o, int count, float f) {
  using S = Share<T>;
  const int apart = int((reinterpret_cast<uintptr_t>(p) - reinterpret_cast<uintptr_t>(o)) & 15);
  if (apart != 0) {
    // The two do not share 16-byte boundaries (tensors of odd sizes behind one another in a buffer):
    // each vector of the output comes from the two aligned vectors of the input that it lies across.
    // All of both lies inside the chunk.
    int head = int((16 - (reinterpret_cast<uintptr_t>(o) & 15)) & 15) / int(sizeof(T));
    if (head * int(sizeof(T)) < apart) head += S::kVec;
    if (head > count) head = count;
    int vecs = ((count - head) * int(sizeof(T)) + apart) / 16 - 1;
    if (vecs < 0) vecs = 0;
    // p + head is `apart` bytes behind a boundary
    const uint4* src = reinterpret_cast<const uint4*>(reinterpret_cast<uintptr_t>(p + head) - apart);
    constexpr int kAhead = 2;  // vectors on the way at once
    for (int i0 = threadIdx.x; i0 < vecs; i0 += kAhead * kThreads) {
      uint4 a[kAhead], b[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int i = i0 + j * kThreads;
        a[j] = b[j] = make_uint4(0, 0, 0, 0);
        if (i < vecs) {
          a[j] = __ldg(src + i);
          b[j] = __ldg(src + i + 1);
        }
      }
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int i = i0 + j * kThreads;
        const uint32_t w[8] = {a[j].x, a[j].y, a[j].z, a[j].w, b[j].x, b[j].y, b[j].z, b[j].w};
        uint32_t r[4];
        const unsigned bits = 8u * unsigned(apart & 3);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t lo = apart < 4 ? w[e] : apart < 8 ? w[e + 1] : apart < 12 ? w[e + 2] : w[e + 3];
          const uint32_t hi = apart < 4 ? w[e + 1] : apart < 8 ? w[e + 2] : apart < 12 ? w[e + 3] : w[e + 4];
          r[e] = __funnelshift_r(lo, hi, bits);
        }
        if (i < vecs) __stcs(reinterpret_cast<uint4*>(o + head) + i, scaled<T>(make_uint4(r[0], r[1], r[2], r[3]), f));
      }
    }
    for (int i = threadIdx.x; i < head; i += kThreads) o[i] = from_f<T>(f * to_f(p[i]));
    for (int i = head + vecs * S::kVec + int(threadIdx.x); i < count; i += kThreads) o[i] = from_f<T>(f * to_f(p[i]));
    return;
  }
  S c(p, count);
#pragma unroll
  for (int j = 0; j < S::kIter; ++j) {
    const int i = j * kThreads + int(threadIdx.x);
    const uint4 q = scaled<T>(c.q[j], f);
    if (i < c.vecs) __stcs(reinterpret_cast<uint4*>(o + c.head) + i, q);
  }
  c.singles([&](int i) { o[i] = from_f<T>(f * to_f(p[i])); });
}

template <int kCap>
__global__ void __launch_bounds__(kThreads, kScaleBlocks)
    k_clip_scale(const __grid_constant__ List<kCap> l, const double* part, int parts, float max_norm, float* norm) {
  __shared__ float factor;
  tc::wait_for_previous();
  tc::launch_dependents();
  if (threadIdx.x < 32) {
    double s = 0.0;
    constexpr int kAhead = 8;
    for (int i0 = threadIdx.x; i0 < parts; i0 += 32 * kAhead) {
      double v[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) v[j] = i0 + 32 * j < parts ? part[i0 + 32 * j] : 0.0;
#pragma unroll
      for (int j = 0; j < kAhead; ++j) s += v[j];
    }
    s = warp_sum(s);
    if (threadIdx.x == 0) {
      float n;
      norm_and_factor(s, max_norm, n, factor);
      if (blockIdx.x == 0) *norm = n;
    }
  }
  __syncthreads();
  const float f = factor;
  for (int c = l.chunks - 1 - int(blockIdx.x); c >= 0; c -= int(gridDim.x)) {
    const Chunk k = chunk_of(l, c);
    if (f == 1.f && l.in[k.t] == l.out[k.t]) continue;
    if (k.bf16)
      scale_chunk(static_cast<const __nv_bfloat16*>(l.in[k.t]) + k.first, static_cast<__nv_bfloat16*>(l.out[k.t]) + k.first,
                  k.count, f);
    else
      scale_chunk(static_cast<const float*>(l.in[k.t]) + k.first, static_cast<float*>(l.out[k.t]) + k.first, k.count, f);
  }
}

int blocks_of(int chunks, int per_sm) {
  const int most = per_sm * sm_count();
  return chunks < 1 ? 1 : chunks < most ? chunks : most;
}

template <int kCap>
void fill(List<kCap>& l, const void* const* grads, void* const* out, const int64_t* numel, const int32_t* dtype, int n) {
  int64_t chunks = 0;
  for (int i = 0; i < n; ++i) {
    l.in[i] = grads[i];
    l.out[i] = out ? out[i] : const_cast<void*>(grads[i]);
    l.numel_type[i] = 2 * numel[i] + (dtype[i] == LOCA_BF16 ? 1 : 0);
    chunks += (numel[i] + kChunk - 1) / kChunk;
    l.chunk_end[i] = int32_t(chunks);
  }
  l.n = n;
  l.chunks = int32_t(chunks);
}

struct Args {
  const void* const* grads;
  void* const* out;
  const int64_t* numel;
  const int32_t* dtype;
  int n;
};

template <class... P, class... A>
cudaError_t launch_early(void (*kernel)(P...), int blocks, cudaStream_t s, A... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(blocks));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = s;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// Squares of one list: adds its blocks to `parts`.
template <int kCap>
cudaError_t sumsq(const Args& a, double* part, int& parts, cudaStream_t s) {
  List<kCap> l;
  fill(l, a.grads, a.out, a.numel, a.dtype, a.n);
  const int blocks = blocks_of(l.chunks, kSumBlocks);
  double* to = part + parts;
  parts += blocks;
  return launch_early(k_clip_sumsq<kCap>, blocks, s, l, to);
}

template <int kCap>
cudaError_t scale(const Args& a, const double* part, int parts, float max_norm, float* norm, cudaStream_t s) {
  List<kCap> l;
  fill(l, a.grads, a.out, a.numel, a.dtype, a.n);
  const int blocks = blocks_of(l.chunks, kScaleBlocks);
  return launch_early(k_clip_scale<kCap>, blocks, s, l, part, parts, max_norm, norm);
}

Args part_of(const Args& a, int first) {
  Args b = a;
  b.n = a.n - first < kMany ? a.n - first : kMany;
  b.grads += first;
  if (b.out) b.out += first;
  b.numel += first;
  b.dtype += first;
  return b;
}

}  // namespace

int64_t grad_clip_max_numel() { return int64_t(kChunk) * 2000000; }

size_t grad_clip_workspace_bytes(int n) {
  const size_t launches = n < 1 ? 1 : (size_t(n) + kMany - 1) / kMany;
  return align256(launches * size_t(kSumBlocks) * size_t(sm_count()) * sizeof(double));
}

cudaError_t launch_grad_clip(const void* const* grads, void* const* out, const int64_t* numel, const int32_t* dtype,
                             int n, float max_norm, float* norm, void* workspace, cudaStream_t s) {
  const Args all{grads, out, numel, dtype, n};
  double* part = static_cast<double*>(workspace);
  int parts = 0;
  for (int i = 0; i < n || i == 0; i += kMany) {
    const Args a = part_of(all, i);
    const cudaError_t e = a.n <= kFew ? sumsq<kFew>(a, part, parts, s) : sumsq<kMany>(a, part, parts, s);
    if (e != cudaSuccess) return e;
  }
  for (int i = 0; i < n || i == 0; i += kMany) {
    const Args a = part_of(all, i);
    const cudaError_t e = a.n <= kFew ? scale<kFew>(a, part, parts, max_norm, norm, s)
                                      : scale<kMany>(a, part, parts, max_norm, norm, s);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace loca
