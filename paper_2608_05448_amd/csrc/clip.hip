// The global norm of a set of gradients and their clipping. Both are streams over the tensors: the norm
// reads every element once, clipping reads and writes every element once (nothing where the norm is
// within the limit and the gradients are clipped in place).
//
// The tensors' addresses travel in the kernel's arguments (no table in device memory, so that a call
// needs no copy and can be captured), up to kNormSet or kClipSet a launch. The tensors of a launch are cut into chunks
// of kChunk elements, which the workgroups take in turn. The squares are formed and summed in binary64:
// exact products, no overflow or underflow of a square for any binary32 or bfloat16 value, and a sum
// whose error does not grow with the number of elements. Each workgroup writes one partial sum, which
// one more workgroup adds in a fixed order, so the norm does not change from run to run.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.hpp"

namespace dbl {
namespace {

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef __bf16 bf16x8u __attribute__((ext_vector_type(8), aligned(2)));

constexpr int kClipSet = 130;        // tensors a launch (kNormSet for the norm)
constexpr int64_t kChunk = 16384;    // elements

// Tensors of one launch: addresses, sizes and, for each, the number of chunks before it.
struct NormSet {
  const void* g[kNormSet];
  int64_t n[kNormSet];
  int32_t first[kNormSet + 1];
  uint8_t bf16[kNormSet];
};
struct ClipSet {
  const void* g[kClipSet];
  void* out[kClipSet];
  int64_t n[kClipSet];
  int32_t first[kClipSet + 1];
  uint8_t bf16[kClipSet];
};
static_assert(sizeof(NormSet) <= 3900 && sizeof(ClipSet) <= 3900, "4 KB of kernel arguments");

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}
// Sum over a workgroup of 256, in every thread's hands.
__device__ __forceinline__ double group_sum(double v) {
  __shared__ double red[4];
  v = wave_sum(v);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return (red[0] + red[1]) + (red[2] + red[3]);
}

__device__ __forceinline__ void add_square(double& s, float x) {
  const double y = static_cast<double>(x);
  s = fma(y, y, s);
}

// The tensor of chunk c: the last one whose first chunk is not past it (by halves: walking the list, a
// scalar load a tensor, took most of the time of many small tensors).
template <class Set>
__device__ __forceinline__ int tensor_of(const Set& s, int count, int c) {
  int lo = 0, hi = count;  // first[lo] <= c < first[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (s.first[mid] <= c) lo = mid;
    else hi = mid;
  }
  return lo;
}

// STREAM: non-temporal loads. A set that the 256 MB Infinity Cache cannot hold until it is clipped is read
// faster so (3.0 GB 514 -> 453 us); one that it can hold is then clipped from it (52 MB 18.2 us, 20.8 with
// the norm's loads non-temporal). More workgroups or loads in flight, smaller and larger chunks and
// non-temporal accesses in the clipping gained nothing.
constexpr int64_t kStreamBytes = int64_t(512) << 20;
template <bool STREAM, class T>
__device__ __forceinline__ T load(const T* p) {
  if constexpr (STREAM) return __builtin_nontemporal_load(p);
  return *p;
}

template <bool STREAM>
__global__ __launch_bounds__(256) void norm_part_kernel(const NormSet s, int count, int chunks,
                                                        double* __restrict__ part) {
  const int tid = threadIdx.x;
  double acc[4] = {0.0, 0.0, 0.0, 0.0};
  int t = tensor_of(s, count, blockIdx.x);
  for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
    while (c >= s.first[t + 1]) ++t;
    const int64_t at = (c - s.first[t]) * kChunk;
    const int64_t left = s.n[t] - at;
    const int n = static_cast<int>(left < kChunk ? left : kChunk);
    if (s.bf16[t]) {
      const __bf16* g = static_cast<const __bf16*>(s.g[t]) + at;
#pragma unroll 4
      for (int i = 8 * tid; i < (n & ~7); i += 2048) {
        const bf16x8u v = load<STREAM>(reinterpret_cast<const bf16x8u*>(g + i));
#pragma unroll
        for (int j = 0; j < 8; ++j) add_square(acc[j & 3], static_cast<float>(v[j]));
      }
      if (tid < (n & 7)) add_square(acc[0], static_cast<float>(g[(n & ~7) + tid]));
    } else {
      const float* g = static_cast<const float*>(s.g[t]) + at;
#pragma unroll 4
      for (int i = 4 * tid; i < (n & ~3); i += 1024) {
        const f32x4u v = load<STREAM>(reinterpret_cast<const f32x4u*>(g + i));
#pragma unroll
        for (int j = 0; j < 4; ++j) add_square(acc[j], v[j]);
      }
      if (tid < (n & 3)) add_square(acc[0], g[(n & ~3) + tid]);
    }
  }
  const double v = group_sum((acc[0] + acc[1]) + (acc[2] + acc[3]));
  if (tid == 0) part[blockIdx.x] = v;
}

__global__ __launch_bounds__(256) void norm_finish_kernel(const double* __restrict__ part, int64_t n,
                                                          float* __restrict__ norm) {
  double v = 0.0;
  for (int64_t i = threadIdx.x; i < n; i += 256) v += part[i];
  v = group_sum(v);
  if (threadIdx.x == 0) *norm = static_cast<float>(sqrt(v));
}

// g * scale in fp32, rounded once to the tensor's type. `same`: whether the outputs are the gradients
// themselves, which a scale of 1 leaves alone.
__global__ __launch_bounds__(256) void clip_kernel(const ClipSet s, int count, int chunks, int same,
                                                   const float* __restrict__ norm, float max_norm) {
  const float value = *norm;
  // No limit scales by 1 under an infinite norm too, where the quotient would be inf / inf.
  const float ratio = max_norm == INFINITY && value == value ? 1.0f : max_norm / (value + 1e-6f);
  const float scale = ratio > 1.0f ? 1.0f : ratio;  // NaN stays
  if (same && scale == 1.0f) return;
  const int tid = threadIdx.x;
  int t = tensor_of(s, count, blockIdx.x);
  for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
    while (c >= s.first[t + 1]) ++t;
    const int64_t at = (c - s.first[t]) * kChunk;
    const int64_t left = s.n[t] - at;
    const int n = static_cast<int>(left < kChunk ? left : kChunk);
    if (s.bf16[t]) {
      const __bf16* g = static_cast<const __bf16*>(s.g[t]) + at;
      __bf16* o = static_cast<__bf16*>(s.out[t]) + at;
#pragma unroll 4
      for (int i = 8 * tid; i < (n & ~7); i += 2048) {
        bf16x8u v = *reinterpret_cast<const bf16x8u*>(g + i);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = static_cast<__bf16>(static_cast<float>(v[j]) * scale);
        *reinterpret_cast<bf16x8u*>(o + i) = v;
      }
      if (tid < (n & 7)) {
        const int i = (n & ~7) + tid;
        o[i] = static_cast<__bf16>(static_cast<float>(g[i]) * scale);
      }
    } else {
      const float* g = static_cast<const float*>(s.g[t]) + at;
      float* o = static_cast<float*>(s.out[t]) + at;
#pragma unroll 4
      for (int i = 4 * tid; i < (n & ~3); i += 1024) {
        f32x4u v = *reinterpret_cast<const f32x4u*>(g + i);
        v *= scale;
        *reinterpret_cast<f32x4u*>(o + i) = v;
      }
      if (tid < (n & 3)) o[(n & ~3) + tid] = g[(n & ~3) + tid] * scale;
    }
  }
}

// The next tensors (at most `most`, empty ones left out) into a launch's set; returns the chunks.
template <class Set, class Extra>
int fill(Set& s, int most, const GradTensor* t, int64_t n, int64_t& next, int& k, Extra extra) {
  int64_t chunks = 0;
  k = 0;
  for (; next < n && k < most; ++next) {
    if (t[next].n == 0) continue;
    s.g[k] = t[next].g;
    s.n[k] = t[next].n;
    s.bf16[k] = static_cast<uint8_t>(t[next].bf16);
    s.first[k] = static_cast<int32_t>(chunks);
    extra(k, t[next]);
    chunks += (t[next].n + kChunk - 1) / kChunk;
    ++k;
  }
  s.first[k] = static_cast<int32_t>(chunks);
  return static_cast<int>(chunks);
}
static_assert(kMaxGradElements / kChunk + kNormSet < 0x7fffffff, "chunks are numbered in 31 bits");

int blocks_for(int chunks) { return chunks < kNormBlocks ? chunks : kNormBlocks; }

}  // namespace

hipError_t launch_grad_norm(const GradTensor* t, int64_t n, double* part, float* norm,
                            hipStream_t stream) {
  int64_t next = 0, parts = 0, bytes = 0;
  for (int64_t i = 0; i < n; ++i) bytes += t[i].n * (t[i].bf16 ? 2 : 4);
  const auto kernel = bytes > kStreamBytes ? norm_part_kernel<true> : norm_part_kernel<false>;
  while (next < n) {
    NormSet s;
    int count;
    const int chunks = fill(s, kNormSet, t, n, next, count, [](int, const GradTensor&) {});
    if (chunks == 0) continue;
    const int blocks = blocks_for(chunks);
    hipLaunchKernelGGL(kernel, dim3(blocks), dim3(256), 0, stream, s, count, chunks,
                       part + parts);
    parts += blocks;
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(norm_finish_kernel, dim3(1), dim3(256), 0, stream, part, parts, norm);
  return hipGetLastError();
}

hipError_t launch_clip_grads(const GradTensor* t, int64_t n, const float* norm, float max_norm,
                             hipStream_t stream) {
  int64_t next = 0;
  bool same = true;
  for (int64_t i = 0; i < n; ++i) same = same && (t[i].out == t[i].g || t[i].n == 0);
  while (next < n) {
    ClipSet s;
    int count;
    const int chunks =
        fill(s, kClipSet, t, n, next, count,
             [&](int k, const GradTensor& g) { s.out[k] = g.out; });
    if (chunks == 0) continue;
    hipLaunchKernelGGL(clip_kernel, dim3(blocks_for(chunks)), dim3(256), 0, stream, s, count, chunks,
                       same ? 1 : 0, norm, max_norm);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace dbl
