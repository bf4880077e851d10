// Microscaled rows (4-bit e2m1 or 8-bit e4m3 values in blocks of 32 that share a power of two, the block
// format of the OCP Microscaling specification): quantisation, the values back, and the
// root-mean-square norm with the residual's addition that quantises its result.
//
// All of it is bound by memory. A lane holds eight consecutive values of a row (one 16-byte load of
// bf16), four lanes a block: the block's largest magnitude is two exchanges among neighbours, its
// scale's byte is that magnitude's binary32 exponent field less the code's largest exponent (kept from
// below by 0), and multiplying by the scale's inverse, a power of two, is exact, so a value is rounded
// once, by the conversion instruction (to nearest, ties to even).
//
// Rows of 8 n values are read and written 16 bytes at a time. Others are a value at a time, at 1.5 to 2.4 TB/s where
// those reach 4.3 to 5.3 (norm of 8192 rows with a residual, 8 bits, bf16 51 us at d = 4096 and 148 at 4097, 17 at
// 1000 and 37 at 1001, fp32 82 and 234; 30,000 rows of bf16 to 8 bits and back 142 and 341).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.hpp"

namespace dbl {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// Eight values of a row from column j on (0 past column d). VEC: d % 8 == 0, so that eight values are
// all there or none, and 16-byte aligned.
template <class T, bool VEC>
__device__ __forceinline__ void load8(const T* row, int j, int d, float (&x)[8]) {
  if constexpr (VEC) {
    if (j < d) {
      if constexpr (sizeof(T) == 2) {
        const bf16x8 v = *reinterpret_cast<const bf16x8*>(row + j);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = static_cast<float>(v[i]);
      } else {
        const f32x4 a = *reinterpret_cast<const f32x4*>(row + j);
        const f32x4 b = *reinterpret_cast<const f32x4*>(row + j + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[i] = a[i];
          x[4 + i] = b[i];
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = 0.0f;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = j + i < d ? static_cast<float>(row[j + i]) : 0.0f;
  }
}

template <class T, bool VEC>
__device__ __forceinline__ void store8(T* row, int j, int d, const float (&x)[8]) {
  if constexpr (VEC) {
    if (j >= d) return;
    if constexpr (sizeof(T) == 2) {
      bf16x8 v;
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = static_cast<__bf16>(x[i]);
      *reinterpret_cast<bf16x8*>(row + j) = v;
    } else {
      *reinterpret_cast<f32x4*>(row + j) = f32x4{x[0], x[1], x[2], x[3]};
      *reinterpret_cast<f32x4*>(row + j + 4) = f32x4{x[4], x[5], x[6], x[7]};
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (j + i < d) row[j + i] = static_cast<T>(x[i]);
  }
}

// Quantises the eight values of a lane, four lanes (4 n .. 4 n + 3) a block: codes to `codes` at value
// offset j of the row, the scale's byte to scales[j / 32]. Every lane of the four calls it. A block that
// holds an infinity or NaN gets the scale NaN (255) and codes 0: all its values are NaN.
template <int BITS>
__device__ __forceinline__ void quantize8(const float (&x)[8], uint8_t* codes, uint8_t* scales, int j) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
  top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 1)));
  top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 2)));
  const int e = static_cast<int>(top >> 23);  // biased exponent, 0 for subnormals
  const bool bad = e == 255;
  const int byte = bad ? 255 : max(e - (BITS == 4 ? 2 : 8), 0);
  const float inv = __uint_as_float(static_cast<uint32_t>(254 - (bad ? 127 : byte)) << 23);
  if constexpr (BITS == 4) {
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0] * inv, x[1] * inv, 1.0f, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2] * inv, x[3] * inv, 1.0f, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4] * inv, x[5] * inv, 1.0f, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6] * inv, x[7] * inv, 1.0f, 3);
    *reinterpret_cast<uint32_t*>(codes + j / 2) = bad ? 0u : c;
  } else {
    float y[8];  // the conversion makes NaN of what rounds past 448
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = __builtin_amdgcn_fmed3f(x[i] * inv, -448.0f, 448.0f);
    int lo = 0, hi = 0;
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], lo, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], hi, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], hi, true);
    *reinterpret_cast<u32x2*>(codes + j) =
        bad ? u32x2{0u, 0u} : u32x2{static_cast<uint32_t>(lo), static_cast<uint32_t>(hi)};
  }
  if ((j & 31) == 0) scales[j >> 5] = static_cast<uint8_t>(byte);
}

// The eight values at offset j of a coded row.
template <int BITS>
__device__ __forceinline__ void values8(const uint8_t* codes, const uint8_t* scales, int j, float (&x)[8]) {
  const uint32_t byte = scales[j >> 5];
  // 2^(byte - 127): 2^-127 is subnormal, 255 is NaN.
  const float s = __uint_as_float(byte == 0 ? 0x00400000u : byte == 255 ? 0x7fc00000u : byte << 23);
  if constexpr (BITS == 4) {
    const uint32_t c = *reinterpret_cast<const uint32_t*>(codes + j / 2);
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 0);
    const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 1);
    const f32x2 e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 2);
    const f32x2 f = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 3);
    x[0] = a[0], x[1] = a[1], x[2] = b[0], x[3] = b[1], x[4] = e[0], x[5] = e[1], x[6] = f[0], x[7] = f[1];
  } else {
    const u32x2 c = *reinterpret_cast<const u32x2*>(codes + j);
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(c[0]), false);
    const f32x2 b = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(c[0]), true);
    const f32x2 e = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(c[1]), false);
    const f32x2 f = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(c[1]), true);
    x[0] = a[0], x[1] = a[1], x[2] = b[0], x[3] = b[1], x[4] = e[0], x[5] = e[1], x[6] = f[0], x[7] = f[1];
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] *= s;
}

// A workgroup takes 256 kUnroll consecutive groups of eight values of the padded rows, taken as one
// sequence: its first group's row by a 64-bit division once, the others' by a 32-bit one.
constexpr int kUnroll = 4;
struct Place {
  int64_t row;
  int j;
};
__device__ __forceinline__ Place place_of(int64_t row0, uint32_t rest0, uint32_t k, uint32_t per_row) {
  const uint32_t g = rest0 + k;
  const uint32_t r = g / per_row;
  return {row0 + r, static_cast<int>(8 * (g - r * per_row))};
}

template <class T, int BITS, bool VEC>
__global__ __launch_bounds__(256) void quantize_kernel(const T* __restrict__ x, uint8_t* __restrict__ codes,
                                                       uint8_t* __restrict__ scales, int64_t M, int d,
                                                       int dp) {
  const uint32_t per_row = dp / 8;
  const int64_t g0 = static_cast<int64_t>(blockIdx.x) * (256 * kUnroll);
  const int64_t row0 = g0 / per_row;
  const uint32_t rest0 = static_cast<uint32_t>(g0 - row0 * per_row);
  float v[kUnroll][8];
  Place at[kUnroll];
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    at[u] = place_of(row0, rest0, threadIdx.x + 256 * u, per_row);
    if (at[u].row < M) load8<T, VEC>(x + at[u].row * d, at[u].j, d, v[u]);
  }
#pragma unroll
  for (int u = 0; u < kUnroll; ++u)
    if (at[u].row < M)  // the same for the four lanes of a block: a row is a multiple of 128 values
      quantize8<BITS>(v[u], codes + at[u].row * (dp / 8 * BITS), scales + at[u].row * (dp / 32), at[u].j);
}

template <class T, int BITS, bool VEC>
__global__ __launch_bounds__(256) void dequantize_kernel(T* __restrict__ x, const uint8_t* __restrict__ codes,
                                                         const uint8_t* __restrict__ scales, int64_t M, int d,
                                                         int dp) {
  const uint32_t per_row = dp / 8;
  const int64_t g0 = static_cast<int64_t>(blockIdx.x) * (256 * kUnroll);
  const int64_t row0 = g0 / per_row;
  const uint32_t rest0 = static_cast<uint32_t>(g0 - row0 * per_row);
  float v[kUnroll][8];
  Place at[kUnroll];
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    at[u] = place_of(row0, rest0, threadIdx.x + 256 * u, per_row);
    if (at[u].row < M)
      values8<BITS>(codes + at[u].row * (dp / 8 * BITS), scales + at[u].row * (dp / 32), at[u].j, v[u]);
  }
#pragma unroll
  for (int u = 0; u < kUnroll; ++u)
    if (at[u].row < M) store8<T, VEC>(x + at[u].row * d, at[u].j, d, v[u]);
}

// Rounded to T and back.
template <class T>
__device__ __forceinline__ float as(float x) {
  return static_cast<float>(static_cast<T>(x));
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

// binary64 to binary32 so that a further rounding to fewer bits gives what rounding the binary64 number
// would: towards zero, and odd where bits are lost. (Infinite only where x is.)
__device__ __forceinline__ float round_odd(double x) {
  const float f = static_cast<float>(x);
  const double b = static_cast<double>(f);
  const uint32_t u = __float_as_uint(f);
  return __uint_as_float(b == x ? u : ((fabs(b) > fabs(x) ? u - 1 : u) | 1u));
}

// Norm with the residual's addition. TPR threads take a row (256 / TPR rows to a workgroup), ITEMS
// groups of eight values each, which stay in registers between the sum of squares and the result, so that
// every input is read once. The sum, the root and the products are in binary64 and y is rounded once, to
// its code, so that a value near a border between two codes falls on its own side of it (16,384 rows of 4,096
// with a residual 92 us, 5.1 TB/s read and written; 85 in binary32, of whose codes a few in a billion were the
// neighbours). ITEMS = 0: rows of any length, read a second time (h from `sum`, which the
// same thread has written, if there is one).
template <class T, int BITS, bool VEC, int TPR, int ITEMS>
__global__ __launch_bounds__(256) void norm_kernel(const T* x, const T* residual, const T* __restrict__ weight,
                                                   float eps, T* sum, T* y, uint8_t* __restrict__ codes,
                                                   uint8_t* __restrict__ scales, int64_t M, int d, int dp) {
  constexpr int ROWS = 256 / TPR;
  __shared__ double part[4];
  const int64_t row = static_cast<int64_t>(blockIdx.x) * ROWS + threadIdx.x / TPR;
  const int t = threadIdx.x % TPR;
  if (TPR == 64 && row >= M) return;  // whole wavefronts; TPR == 256: a workgroup per row
  const T* const xr = x + row * d;
  const T* const rr = residual ? residual + row * d : nullptr;
  T* const sr = sum ? sum + row * d : nullptr;
  constexpr int kHeld = ITEMS ? ITEMS : 1;
  float h[kHeld][8];
  double ss = 0.0;
  auto take = [&](int j, float (&v)[8]) {
    load8<T, VEC>(xr, j, d, v);
    if (rr) {
      float r[8];
      load8<T, VEC>(rr, j, d, r);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = as<T>(v[i] + r[i]);
      if (sr) store8<T, VEC>(sr, j, d, v);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) ss = fma(static_cast<double>(v[i]), static_cast<double>(v[i]), ss);
  };
  if constexpr (ITEMS > 0) {
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      const int j = 8 * (t + TPR * k);
      if (j < dp) take(j, h[k]);
    }
  } else {
    for (int j = 8 * t; j < dp; j += 8 * TPR) take(j, h[0]);
  }
  ss = wave_sum(ss);
  if constexpr (TPR == 256) {
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = ss;
    __syncthreads();
    ss = (part[0] + part[1]) + (part[2] + part[3]);
  }
  const double scale = 1.0 / sqrt(ss / static_cast<double>(d) + static_cast<double>(eps));
  auto give = [&](int j, float (&v)[8]) {
    float w[8];
    load8<T, VEC>(weight, j, d, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const double p = static_cast<double>(v[i]) * scale * static_cast<double>(w[i]);
      v[i] = j < d ? round_odd(p) : 0.0f;  // padding is 0 also where the row's scale is infinite or NaN
      w[i] = sizeof(T) == 4 ? static_cast<float>(p) : v[i];
    }
    if (y) store8<T, VEC>(y + row * d, j, d, w);
    quantize8<BITS>(v, codes + row * (dp / 8 * BITS), scales + row * (dp / 32), j);
  };
  if constexpr (ITEMS > 0) {
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      const int j = 8 * (t + TPR * k);
      if (j < dp) give(j, h[k]);
    }
  } else {
    for (int j = 8 * t; j < dp; j += 8 * TPR) {
      if (sr) {
        load8<T, VEC>(sr, j, d, h[0]);
      } else {
        load8<T, VEC>(xr, j, d, h[0]);
        if (rr) {
          float r[8];
          load8<T, VEC>(rr, j, d, r);
#pragma unroll
          for (int i = 0; i < 8; ++i) h[0][i] = as<T>(h[0][i] + r[i]);
        }
      }
      give(j, h[0]);
    }
  }
}

template <class T, int BITS, bool VEC>
hipError_t launch_norm_as(const MxNormArgs& a, hipStream_t stream) {
  const int dp = static_cast<int>(mx_row(a.q.d));
  auto go = [&](auto kernel, int rows) {
    const int64_t blocks = (a.q.M + rows - 1) / rows;
    if (blocks > kMaxThreads / 256) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, stream,
                       static_cast<const T*>(a.q.x), static_cast<const T*>(a.residual),
                       static_cast<const T*>(a.weight), a.eps, static_cast<T*>(a.sum),
                       static_cast<T*>(a.y), static_cast<uint8_t*>(a.q.codes), a.q.scales, a.q.M, a.q.d,
                       dp);
    return hipGetLastError();
  };
  if (dp <= 512) return go(norm_kernel<T, BITS, VEC, 64, 1>, 4);
  if (dp <= 2048) return go(norm_kernel<T, BITS, VEC, 256, 1>, 1);
  if (dp <= 4096) return go(norm_kernel<T, BITS, VEC, 256, 2>, 1);
  if (dp <= 8192) return go(norm_kernel<T, BITS, VEC, 256, 4>, 1);
  return go(norm_kernel<T, BITS, VEC, 256, 0>, 1);
}

template <class T, int BITS, bool VEC>
hipError_t launch_quant_as(const MxQuantArgs& a, bool back, hipStream_t stream) {
  const int64_t dp = mx_row(a.d), per = 256 * kUnroll;
  const int64_t blocks = (a.M * (dp / 8) + per - 1) / per;
  if (blocks > kMaxThreads / 256) return hipErrorInvalidConfiguration;
  const dim3 grid(static_cast<unsigned>(blocks));
  if (back)
    hipLaunchKernelGGL((dequantize_kernel<T, BITS, VEC>), grid, dim3(256), 0, stream,
                       static_cast<T*>(const_cast<void*>(a.x)), static_cast<const uint8_t*>(a.codes),
                       a.scales, a.M, a.d, static_cast<int>(dp));
  else
    hipLaunchKernelGGL((quantize_kernel<T, BITS, VEC>), grid, dim3(256), 0, stream,
                       static_cast<const T*>(a.x), static_cast<uint8_t*>(a.codes), a.scales, a.M, a.d,
                       static_cast<int>(dp));
  return hipGetLastError();
}

// f(type tag, bits, whether 8 divides d).
template <class F>
hipError_t by_form(const MxQuantArgs& a, F f) {
  auto bits = [&](auto t) {
    auto vec = [&](auto b) {
      return a.d % 8 == 0 ? f(t, b, std::true_type{}) : f(t, b, std::false_type{});
    };
    return a.bits == 4 ? vec(std::integral_constant<int, 4>{}) : vec(std::integral_constant<int, 8>{});
  };
  return a.bf16 ? bits(__bf16{}) : bits(float{});
}

}  // namespace

hipError_t launch_mx_quantize(const MxQuantArgs& a, hipStream_t stream) {
  return by_form(a, [&](auto t, auto b, auto v) {
    return launch_quant_as<decltype(t), decltype(b)::value, decltype(v)::value>(a, false, stream);
  });
}

hipError_t launch_mx_dequantize(const MxQuantArgs& a, hipStream_t stream) {
  return by_form(a, [&](auto t, auto b, auto v) {
    return launch_quant_as<decltype(t), decltype(b)::value, decltype(v)::value>(a, true, stream);
  });
}

hipError_t launch_mx_norm(const MxNormArgs& a, hipStream_t stream) {
  return by_form(a.q, [&](auto t, auto b, auto v) {
    return launch_norm_as<decltype(t), decltype(b)::value, decltype(v)::value>(a, stream);
  });
}

}  // namespace dbl
