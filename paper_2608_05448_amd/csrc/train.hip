// Training: the negative log-likelihood of given tokens under the LM head and its gradient, and the
// backward pass of the branch expander.
//
// Head. A row's loss is nll = lse - logit[token]; its gradient with respect to the logits is
// u = p - [v = token] times the loss's gradient g, and dh = (g u) w, dw = (g u)^T h. The logits are
// never kept: the forward pass reduces them in the head GEMM's epilogue, the backward pass forms them
// again, a piece of the vocabulary at a time, as u in bf16 (fp32 for fp32 inputs), which the two
// products then read.
// Rows whose token is outside [0, V) do not count: the rows that do are gathered first, so that the
// others cost nothing and whatever they hold (NaN, infinities) reaches no result.
//
// Products. Both operands of the products meet along a dimension that at least one of them does not
// hold contiguously ([K, n] row-major). Such an operand is copied to LDS as it lies and its MFMA
// fragments are read with the transposing LDS reads (ds_read_b64_tr_b16). The output's contiguous
// dimension lies on the MFMA rows, so that a lane holds four consecutive outputs.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "kernels.hpp"

namespace dbl {
namespace {

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;

// ---------------------------------------------------------------------------------------
// Rows that count.

__device__ __forceinline__ bool counts(int32_t x, int64_t V) { return x >= 0 && x < V; }

__device__ __forceinline__ int wave_sum_int(int v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

// Up to this many positions every workgroup of the gather counts the positions before its own itself
// (at most 16 KB from L2); beyond, one workgroup counts them all first.
constexpr int64_t kCountInline = 4096;

__global__ __launch_bounds__(1024) void count_positions_kernel(const int32_t* __restrict__ x, int64_t P,
                                                               int R, int64_t V,
                                                               int32_t* __restrict__ inv,
                                                               int32_t* __restrict__ count) {
  __shared__ int part[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int before = 0;
  for (int64_t p0 = 0; p0 < P; p0 += 1024) {
    const int64_t p = p0 + threadIdx.x;
    const bool c = p < P && counts(x[p], V);
    const uint64_t mask = __ballot(c);
    if (lane == 0) part[wave] = __popcll(mask);
    __syncthreads();
    int at = before, all = 0;
    for (int i = 0; i < 16; ++i) {
      at += i < wave ? part[i] : 0;
      all += part[i];
    }
    at += __popcll(mask & ((uint64_t(1) << lane) - 1));
    if (p < P) inv[p] = c ? at : -1;
    before += all;
    __syncthreads();
  }
  if (threadIdx.x == 0) *count = before * R;
}

// One workgroup per row: its position's place among those that count, its states copied there (and, for
// dw, times their scale), and what the head's kernels need of it.
template <class T>
__global__ __launch_bounds__(256) void gather_rows_kernel(const NllArgs a, int counted) {
  __shared__ int part[4];
  const int64_t p = blockIdx.x;
  const int R = static_cast<int>(a.R), d = a.d, r = blockIdx.y;
  const int32_t token = a.x[p];
  const bool mine = counts(token, a.V);
  int at;
  if (counted) {
    at = a.inv[p];
  } else {
    int c = 0;
    for (int64_t i = threadIdx.x; i < p; i += 256) c += counts(a.x[i], a.V) ? 1 : 0;
    c = wave_sum_int(c);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = c;
    __syncthreads();
    at = part[0] + part[1] + part[2] + part[3];
    if (threadIdx.x == 0 && r == 0) {
      a.inv[p] = mine ? at : -1;
      if (p == a.P - 1) *a.count = (at + (mine ? 1 : 0)) * R;
    }
  }
  if (!mine) return;
  const int64_t from = p * R + r, to = static_cast<int64_t>(at) * R + r;
  TrainRow row{0.0f, 0.0f, 0.0f, token};
  if (a.g) {
    const float lse = a.lse[from], g = a.g[from], nll = a.nll[from];
    const float q = nll < 0.0f ? 0.0f : -expm1f(-nll);  // NaN stays, also in qc (fmaxf would drop it)
    if (sizeof(T) == 2) {
      const float qc = q < 0x1p-24f ? 0x1p-24f : q;
      row.shift = (lse + logf(qc)) * kLog2e;
      row.at_token = -q / qc;
      row.scale = g * qc;
    } else {
      row.shift = lse;
      row.at_token = -q;
      row.scale = g;
    }
  }
  if (threadIdx.x == 0) a.rows[to] = row;
  const T* src = static_cast<const T*>(a.h) + from * d;
  T* dst = static_cast<T*>(a.hc) + to * d;
  T* dss = a.hs ? static_cast<T*>(a.hs) + to * d : nullptr;
  if (sizeof(T) == 2) {  // d % 8 == 0
#pragma unroll 2
    for (int j = 8 * threadIdx.x; j < d; j += 2048) {
      const bf16x8 v = *reinterpret_cast<const bf16x8*>(src + j);
      *reinterpret_cast<bf16x8*>(dst + j) = v;
      if (dss) {
        bf16x8 y;
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = static_cast<__bf16>(static_cast<float>(v[i]) * row.scale);
        *reinterpret_cast<bf16x8*>(dss + j) = y;
      }
    }
  } else {
    for (int j = threadIdx.x; j < d; j += 256) {
      const T v = src[j];
      dst[j] = v;
      if (dss) dss[j] = static_cast<T>(static_cast<float>(v) * row.scale);
    }
  }
}

hipError_t gather_rows(const NllArgs& a, hipStream_t stream) {
  const int counted = a.P > kCountInline;
  if (counted)
    hipLaunchKernelGGL(count_positions_kernel, dim3(1), dim3(1024), 0, stream, a.x, a.P,
                       static_cast<int>(a.R), a.V, a.inv, a.count);
  const dim3 grid(static_cast<unsigned>(a.P), static_cast<unsigned>(a.R));
  if (a.bf16)
    hipLaunchKernelGGL(gather_rows_kernel<__bf16>, grid, dim3(256), 0, stream, a, counted);
  else
    hipLaunchKernelGGL(gather_rows_kernel<float>, grid, dim3(256), 0, stream, a, counted);
  return hipGetLastError();
}

// lse and nll of every row from the tile log-masses; 0 for the rows that do not count. One wave a row,
// 32 masses a lane at a time (V up to 262,144 in one pass): all loads in flight, then their maximum and
// their sum of exponentials, joined to the running ones. A tile with a NaN or a logit of plus infinity has a
// mass of NaN (exp(inf - inf)), and so have the row's lse and nll.
__global__ __launch_bounds__(256) void nll_finish_kernel(const NllArgs a, int nT) {
  constexpr int kRegs = 32;
  const int64_t m = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (m >= a.P * a.R) return;
  const int at = a.inv[m / a.R];
  float lse = 0.0f, nll = 0.0f;
  if (at >= 0) {
    const int64_t i = static_cast<int64_t>(at) * a.R + m % a.R;
    const float* row = a.lmass + i * nT;
    float mx = -INFINITY, s = 0.0f;
    for (int t0 = 0; t0 < nT; t0 += 64 * kRegs) {
      float v[kRegs], top = mx;
#pragma unroll
      for (int k = 0; k < kRegs; ++k) {
        const int t = t0 + lane + 64 * k;
        v[k] = t < nT ? row[t] : -INFINITY;
      }
#pragma unroll
      for (int k = 0; k < kRegs; ++k) top = fmaxf(top, v[k]);
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
      // Masses of minus infinity only add 0. So that a NaN, which the maximum passes over, is added all the
      // same where it leaves none, the exponentials are taken there as well.
      const float base = top > -INFINITY ? top : 0.0f;
      if (top > -INFINITY) s *= expf(mx - top);
      float add = 0.0f;
#pragma unroll
      for (int k = 0; k < kRegs; ++k) add += expf(v[k] - base);
      s += add;
      mx = top;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
    lse = mx + logf(s);
    nll = lse - a.tgt[i];
  }
  if (lane == 0) {
    a.lse[m] = lse;
    a.nll[m] = nll;
  }
}

// ---------------------------------------------------------------------------------------
// Sum over the splits of four columns of a row's parts, eight loads in flight.
__device__ __forceinline__ f32x4 sum_parts(const float* part, int64_t stride, int splits) {
  f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
  int s = 0;
  for (; s + 8 <= splits; s += 8) {
    f32x4 u[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) u[i] = *reinterpret_cast<const f32x4u*>(part + (s + i) * stride);
#pragma unroll
    for (int i = 0; i < 8; ++i) v += u[i];
  }
  for (; s < splits; ++s) v += *reinterpret_cast<const f32x4u*>(part + s * stride);
  return v;
}
__device__ __forceinline__ void store4(__bf16* o, f32x4 v) {
  *reinterpret_cast<bf16x4*>(o) = bf16x4{static_cast<__bf16>(v[0]), static_cast<__bf16>(v[1]),
                                         static_cast<__bf16>(v[2]), static_cast<__bf16>(v[3])};
}

// A weight gradient from its parts, n values each.
template <class T>
__global__ __launch_bounds__(256) void weight_finish_kernel(const float* __restrict__ part, int64_t n, int splits,
                                                            T* __restrict__ out) {
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 1024 + 4 * threadIdx.x;
  if (i + 4 <= n) {
    const f32x4 v = sum_parts(part + i, n, splits);
    if constexpr (sizeof(T) == 2)
      store4(out + i, v);
    else
      *reinterpret_cast<f32x4*>(out + i) = v;
  } else {
    for (int64_t j = i; j < n; ++j) {
      float v = 0.0f;
      for (int s = 0; s < splits; ++s) v += part[s * n + j];
      out[j] = static_cast<T>(v);
    }
  }
}

// ---------------------------------------------------------------------------------------
// bf16 products out[b, a] = sum_k B(k, b) A[k, a] with A [K, lda] row-major.

struct Prod {
  const __bf16* A;       // [K, lda], columns na
  const __bf16* B;       // TRB: [K, ldb], columns nb; else [nb, ldb], contiguous along K
  int64_t lda, ldb, na, nb, K;
  const int32_t* count;  // if set: K (TRB) or nb
  float* part;           // [splits, nb_max, na] fp32 sums, or null
  int64_t part_stride;   // elements between splits
  int accumulate;        // add to what part holds
  __bf16* out;           // [nb, na] bf16 (one split)
  int splits;
  int n_btiles;
};

__device__ __forceinline__ uint32_t lds_addr(const char* p) {
  return static_cast<uint32_t>(
      reinterpret_cast<uintptr_t>((const __attribute__((address_space(3))) char*)(p)));
}

// One global_load_lds_dwordx4 (lane i copies 16 bytes from sbase + voff to LDS byte m0 + 16 i), issued
// through inline asm so that the compiler does not drain every outstanding copy before each LDS read;
// completion is tracked with wait_vmcnt. The wait states cover a VALU write of the scalar base.
// NT: non-temporal, for an operand that the launch reads once.
template <bool NT = false>
__device__ __forceinline__ void lds_dma16(const char* sbase, uint32_t voff, uint32_t m0v) {
  if constexpr (NT)
    asm volatile("s_nop 4\n\tglobal_load_lds_dwordx4 %0, %1 nt" ::"v"(voff), "s"(sbase), "{m0}"(m0v)
                 : "memory");
  else
    asm volatile("s_nop 4\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(voff), "s"(sbase), "{m0}"(m0v)
                 : "memory");
}

template <int N>
__device__ __forceinline__ void wait_vmcnt() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

__device__ __forceinline__ int xcd_remap(int id, int n) {
  const int q = n >> 3, rem = n & 7;
  const int x = id & 7, s = id >> 3;
  return x < rem ? x * (q + 1) + s : rem * (q + 1) + (x - rem) * q + s;
}

// Four bf16 from each of the 16 lanes of a group, transposed: with lane i's address at row i / 4,
// columns 4 (i % 4) .. + 3 of a 4 x 16 block, lane i receives column i, rows 0 .. 3.
__device__ __forceinline__ s16x4 lds_read_tr(const char* p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (__attribute__((address_space(3))) s16x4*)(uintptr_t)(lds_addr(p)));
}

__device__ __forceinline__ bf16x8 join(s16x4 lo, s16x4 hi) {
  typedef short s16x8 __attribute__((ext_vector_type(8)));
  const s16x8 v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
  return __builtin_bit_cast(bf16x8, v);
}

// The first n (of 8) values of a fragment, the others 0.
__device__ __forceinline__ bf16x8 keep_first(bf16x8 v, int n) {
  u32x4 u = __builtin_bit_cast(u32x4, v);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    u[i] = n >= 2 * i + 2 ? u[i] : n == 2 * i + 1 ? (u[i] & 0xffffu) : 0u;
  return __builtin_bit_cast(bf16x8, u);
}

// LDS layout of a transposed operand: row k of a stage holds C columns; 16-byte chunk c of row k lies
// at chunk c ^ tr_swz(k), so that the four rows that a transposing read takes 64 bytes of each lie in
// different banks.
template <int C>
__device__ __forceinline__ int tr_swz(int k) {
  static_assert(C == 64 || C % 128 == 0, "columns per LDS row");
  return C == 64 ? 4 * ((k >> 1) & 1) : 4 * (k & 3);
}
// LDS layout of an operand held along K: 128-byte rows, chunk c of row r at chunk c ^ ((r / 2) % 8).
__device__ __forceinline__ int row_swz(int r) { return (r >> 1) & 7; }

// Stores a wave's block of outputs, 32 rows x 32 NRA columns at a time through LDS so that a store
// instruction writes whole row segments (the register layout would write 8 or 16 bytes of 32 rows): lane
// l holds row l % 32 and, in registers 4 g .. 4 g + 3 of block i, columns 32 i + 8 g + 4 (l / 32) + {0 .. 3}.
// xp: 32 rows of 32 NRA values of LDS that no other wave touches. Chunks of a row are permuted by the row.
enum ProdOut : int { kOutPart = 0, kOutKeep = 1, kOutStream = 2 };  // fp32 sums; bf16; bf16 past the caches
template <int NRA, int NCB, int OUT>
__device__ __forceinline__ void store_block(f32x16 (&acc)[NRA][NCB], const Prod& p, int64_t nb,
                                            int64_t b0, int64_t a0, int split, int lane, char* xp) {
  constexpr bool PART = OUT == kOutPart;
  constexpr int COLS = 32 * NRA, ROWB = COLS * (PART ? 4 : 2), CH = ROWB / 16;  // 16-byte chunks a row
  constexpr int RPI = 64 / CH;                                                // rows per instruction
  static_assert(CH >= 4 && CH <= 64 && (CH & (CH - 1)) == 0, "whole rows per instruction");
  const int lr = lane & 31, half = lane >> 5;
  constexpr int MASK = CH < 16 ? CH - 1 : 15;
#pragma unroll
  for (int j = 0; j < NCB; ++j) {
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < NRA; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x16& v = acc[i][j];
        if constexpr (PART)
          *reinterpret_cast<f32x4*>(xp + lr * ROWB + ((8 * i + 2 * g + half) ^ (lr & MASK)) * 16) =
              f32x4{v[4 * g], v[4 * g + 1], v[4 * g + 2], v[4 * g + 3]};
        else
          *reinterpret_cast<bf16x4*>(xp + lr * ROWB + ((4 * i + g) ^ (lr & MASK)) * 16 + half * 8) =
              bf16x4{static_cast<__bf16>(v[4 * g]), static_cast<__bf16>(v[4 * g + 1]),
                     static_cast<__bf16>(v[4 * g + 2]), static_cast<__bf16>(v[4 * g + 3])};
      }
    // Wave-private LDS region: the writes above precede these reads in the wave's LDS queue.
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
    for (int r0 = 0; r0 < 32; r0 += RPI) {
      const int r = r0 + lane / CH, c = lane % CH;
      const int64_t b = b0 + 32 * j + r, a = a0 + c * (PART ? 4 : 8);
      const char* at = xp + r * ROWB + (c ^ (r & MASK)) * 16;
      if (b < nb && a < p.na) {  // na % 8 == 0
        if constexpr (PART) {
          f32x4 v = *reinterpret_cast<const f32x4*>(at);
          f32x4* o = reinterpret_cast<f32x4*>(p.part + split * p.part_stride + b * p.na + a);
          if (p.accumulate) v += *o;
          *o = v;
        } else {
          const u32x4 v = *reinterpret_cast<const u32x4*>(at);
          u32x4* o = reinterpret_cast<u32x4*>(p.out + b * p.na + a);
          if constexpr (OUT == kOutStream)
            __builtin_nontemporal_store(v, o);
          else
            *o = v;
        }
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  }
}

// Tile order: groups of kGroupB b tiles; a group sweeps every a tile before the next group starts, its b
// tiles consecutive for one a tile, so that the 32 workgroups of an XCD share 8 a and 4 b tiles. The
// splits of the sum come one after the other.
constexpr int kGroupB = 4;
__device__ __forceinline__ void prod_tile(int L, int n_atiles, int n_btiles, int* at, int* bt, int* split) {
  const int n = n_atiles * n_btiles;
  *split = L / n;
  L -= *split * n;
  const int full = n_btiles / kGroupB * kGroupB * n_atiles;
  const int g = L < full ? kGroupB : n_btiles % kGroupB;
  const int base = L < full ? L / (kGroupB * n_atiles) * kGroupB : n_btiles - g;
  const int rem = L < full ? L % (kGroupB * n_atiles) : L - full;
  // In scalar registers: the copies' base addresses are made of these.
  *split = __builtin_amdgcn_readfirstlane(*split);
  *at = __builtin_amdgcn_readfirstlane(rem / g);
  *bt = __builtin_amdgcn_readfirstlane(base + rem % g);
}

// Ring kernel: BA x BB output tile, WA x WB waves, BK-deep stages copied global -> LDS into an S-slot
// ring S - 1 stages ahead, one barrier per stage.
template <int BA_, int BB_, int WA_, int WB_, int S_, int BK_ = 64, bool NT_ = false>
struct RingCfg {
  static constexpr int BA = BA_, BB = BB_, WA = WA_, WB = WB_, S = S_, BK = BK_;
  static constexpr bool NT = NT_;
  static constexpr int NW = WA * WB, kThreads = 64 * NW;
  static constexpr int NRA = BA / WA / 32, NCB = BB / WB / 32;
  static constexpr int TILEA = BA * BK * 2, TILEB = BB * BK * 2, STAGE = TILEA + TILEB;
  static constexpr int AI = TILEA / 1024 / NW, BI = TILEB / 1024 / NW;  // copies per wave and stage
  static constexpr int PER = AI + BI;
  static constexpr int kLds = S * STAGE;
  static constexpr int kWgPerCu = 160 * 1024 / kLds;
  static constexpr int kWaves = kWgPerCu * NW / 4;
  static constexpr int kWavesPerEu = kWaves < 1 ? 1 : kWaves > 4 ? 4 : kWaves;
  static_assert(TILEA % (1024 * NW) == 0 && TILEB % (1024 * NW) == 0, "whole copies");
  static_assert(NRA >= 1 && NCB >= 1 && BA % (32 * WA) == 0 && BB % (32 * WB) == 0, "tiling");
  static_assert((S - 1) * PER <= 63 && kLds <= 160 * 1024, "ring");
};

template <class C, bool TRB, int OUT>
__global__ __launch_bounds__(C::kThreads, C::kWavesPerEu) void prod_ring_kernel(const Prod p) {
  constexpr int BA = C::BA, BB = C::BB, NRA = C::NRA, NCB = C::NCB, BK = C::BK;
  static_assert(TRB || BK == 64, "an operand held along K has 128-byte LDS rows");
  __shared__ __attribute__((aligned(1024))) char smem[C::kLds];
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wa = wave / C::WB, wb = wave % C::WB;

  int64_t K = p.K, nb = p.nb;
  if (p.count) {
    if (TRB) K = *p.count;
    else nb = *p.count;
  }
  int at, bt, split;
  prod_tile(xcd_remap(blockIdx.x, gridDim.x), static_cast<int>((p.na + BA - 1) / BA), p.n_btiles, &at,
            &bt, &split);
  const int64_t a0 = static_cast<int64_t>(at) * BA, b0 = static_cast<int64_t>(bt) * BB;
  if (b0 >= nb) return;
  // Stages are dealt to the splits in turn, so that all of them read one front that moves through the
  // operands (60 rows, d = 2560, K = 151,936: 136 us; with a range of its own for each split 144).
  const int64_t stages = (K + BK - 1) / BK;
  const int nk = static_cast<int>(stages > split ? (stages - split + p.splits - 1) / p.splits : 0);
  const int64_t kb = static_cast<int64_t>(split) * BK, step = static_cast<int64_t>(p.splits) * BK;

  // Copies. Transposed operand: an instruction covers 512 / columns rows of the stage.
  constexpr int APR = BA / 8, BPR = TRB ? BB / 8 : 8;  // 16-byte chunks per LDS row
  uint32_t ca[C::AI], cb[C::BI];                       // column (or row) part of the offset, bytes
  int ra[C::AI], rb[C::BI];                            // row of the stage (transposed operands)
#pragma unroll
  for (int i = 0; i < C::AI; ++i) {
    const int c = (wave * C::AI + i) * 64 + lane;
    ra[i] = c / APR;
    const int64_t col = a0 + 8 * ((c % APR) ^ tr_swz<BA>(ra[i]));
    ca[i] = static_cast<uint32_t>(2 * (col < p.na ? col : p.na - 8));
  }
#pragma unroll
  for (int i = 0; i < C::BI; ++i) {
    const int c = (wave * C::BI + i) * 64 + lane;
    if (TRB) {
      rb[i] = c / BPR;
      const int64_t col = b0 + 8 * ((c % BPR) ^ tr_swz<TRB ? BB : 64>(rb[i]));
      cb[i] = static_cast<uint32_t>(2 * (col < p.ldb ? col : p.ldb - 8));
    } else {
      const int r = c / 8;
      rb[i] = 8 * ((c % 8) ^ row_swz(r));  // first k of the chunk
      const int64_t gr = r < nb - b0 ? r : nb - b0 - 1;
      cb[i] = static_cast<uint32_t>(2 * gr * p.ldb);
    }
  }
  const char* const baseA = reinterpret_cast<const char*>(p.A);
  const char* const baseB =
      reinterpret_cast<const char*>(p.B) + (TRB ? 0 : static_cast<int64_t>(2) * b0 * p.ldb);
  const uint32_t lds0 = lds_addr(smem);
  const uint32_t lda2 = static_cast<uint32_t>(2 * p.lda), ldb2 = static_cast<uint32_t>(2 * p.ldb);
  // Stage s: rows (or chunks) past the end of the range repeat its last one; what they hold counts
  // as 0 (see tail below).
  auto copy = [&](int s, int slot) {
    const int64_t k0 = kb + step * static_cast<int64_t>(s);
    const int left = static_cast<int>(K - k0 < BK ? K - k0 : BK);  // >= 1
    const uint32_t to = lds0 + slot * C::STAGE;
    const char* sa = baseA + k0 * lda2;
    const char* sb = TRB ? baseB + k0 * ldb2 : baseB + 2 * k0;
#pragma unroll
    for (int i = 0; i < C::AI; ++i)
      lds_dma16<C::NT>(sa, ca[i] + static_cast<uint32_t>(ra[i] < left ? ra[i] : left - 1) * lda2,
                to + (wave * C::AI + i) * 1024);
#pragma unroll
    for (int i = 0; i < C::BI; ++i) {
      const uint32_t off =
          TRB ? cb[i] + static_cast<uint32_t>(rb[i] < left ? rb[i] : left - 1) * ldb2
              : cb[i] + 2 * static_cast<uint32_t>(rb[i] < left ? rb[i] : 0);
      lds_dma16(sb, off, to + C::TILEA + (wave * C::BI + i) * 1024);
    }
  };

  f32x16 acc[NRA][NCB];
#pragma unroll
  for (int i = 0; i < NRA; ++i)
#pragma unroll
    for (int j = 0; j < NCB; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;

  // Fragments of a 16-deep k step: lane l holds column l % 32 of a 32-column block, k values
  // 8 (l / 32) .. + 7. Transposing read j (of two) takes rows 8 (l / 32) + 4 j + (l % 16) / 4.
  const int i16 = lane & 15, g16 = (lane >> 4) & 1, half = lane >> 5;
  auto frag_tr = [&](const char* tile, int row_bytes, int cols64, int block, int ks) {
    // chunk of the block's 64 bytes: 4 block + 2 g16 + (i16 % 4) / 2, permuted by its row
    const int k = 16 * ks + 8 * half + (i16 >> 2);
    const int swz = cols64 ? 4 * ((k >> 1) & 1) : 4 * (k & 3);
    const int chunk = (4 * block + 2 * g16 + ((i16 & 3) >> 1)) ^ swz;
    const char* at0 = tile + k * row_bytes + chunk * 16 + (i16 & 1) * 8;
    return join(lds_read_tr(at0), lds_read_tr(at0 + 4 * row_bytes));
  };
  auto stage = [&](int slot, int left) {
    const char* sa = smem + slot * C::STAGE;
    const char* sb = sa + C::TILEA;
    const bool tail = left < BK;
#pragma unroll
    for (int ks = 0; ks < BK / 16; ++ks) {
      bf16x8 af[NRA], bf[NCB];
#pragma unroll
      for (int i = 0; i < NRA; ++i) af[i] = frag_tr(sa, BA * 2, BA == 64, wa * NRA + i, ks);
#pragma unroll
      for (int j = 0; j < NCB; ++j) {
        if constexpr (TRB) {
          bf[j] = frag_tr(sb, BB * 2, BB == 64, wb * NCB + j, ks);
        } else {
          const int r = (wb * NCB + j) * 32 + (lane & 31);
          bf[j] = *reinterpret_cast<const bf16x8*>(sb + r * 128 + ((2 * ks + half) ^ row_swz(r)) * 16);
        }
      }
      if (tail) {  // both operands: what a copy past the end repeats may hold infinities
        const int n = left - 16 * ks - 8 * half;
#pragma unroll
        for (int i = 0; i < NRA; ++i) af[i] = keep_first(af[i], n);
#pragma unroll
        for (int j = 0; j < NCB; ++j) bf[j] = keep_first(bf[j], n);
      }
#pragma unroll
      for (int i = 0; i < NRA; ++i)
#pragma unroll
        for (int j = 0; j < NCB; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(af[i], bf[j], acc[i][j], 0, 0, 0);
    }
  };

#pragma unroll
  for (int j = 0; j < C::S - 1; ++j)
    if (j < nk) copy(j, j);
  int slot = 0;
  for (int kt = 0; kt < nk; ++kt) {
    // Stages kt + 1 .. kt + S - 2 may still be in flight; near the end all have to be in.
    if (kt + C::S - 1 <= nk)
      wait_vmcnt<(C::S - 2) * C::PER>();
    else
      wait_vmcnt<0>();
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    // Every wave has read stage kt - 1: its slot takes stage kt + S - 1.
    if (kt + C::S - 1 < nk) copy(kt + C::S - 1, slot == 0 ? C::S - 1 : slot - 1);
    const int64_t left = K - kb - step * static_cast<int64_t>(kt);
    stage(slot, left < BK ? static_cast<int>(left) : BK);
    slot = slot + 1 == C::S ? 0 : slot + 1;
  }

  // The ring is free once every wave has left its last stage (every copy has landed).
  __syncthreads();
  constexpr int XP = 32 * 32 * NRA * (OUT == kOutPart ? 4 : 2);
  static_assert(C::NW * XP <= C::kLds, "LDS for the stores");
  store_block<NRA, NCB, OUT>(acc, p, nb, b0 + wb * NCB * 32, a0 + wa * NRA * 32, split, lane,
                              smem + wave * XP);
}

// Ping-pong kernel: 256 x 256 output tile, 64-deep stages, 8 waves of 128 a x 64 b in two groups of four
// that take turns between workgroup barriers: one group issues MFMAs (16 a turn, 32 of a stage's 64 k)
// while the other reads its next fragments from LDS and issues global -> LDS copies (4 a wave and turn).
// The dispatcher places waves w and w + 4 on the same SIMD, so that each SIMD's matrix pipe is fed by
// one wave or the other. LDS: three slots of A stages and two of B stages (160 KB). Copies: even turn 2 s
// the B rows of stage s + 1, odd turn 2 s + 1 the A rows of stage s + 2.
constexpr int kPpTile = 32768;  // bytes of an operand's stage
__device__ __forceinline__ void pp_barrier() {
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);
}

template <bool TRB, int OUT>
__global__ __launch_bounds__(512, 1) void prod_pp_kernel(const Prod p) {
  constexpr int NRA = 4, NCB = 2, TILE = kPpTile, BOFF = 3 * TILE;
  __shared__ __attribute__((aligned(1024))) char smem[5 * TILE];
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int grp = wave >> 2;  // group 0 computes first in every pair of turns
  const int wa = wave & 1;    // half of the 256 a
  const int wb = wave >> 1;   // quarter of the 256 b

  int64_t K = p.K, nb = p.nb;
  if (p.count) {
    if (TRB) K = *p.count;
    else nb = *p.count;
  }
  int at, bt, split;
  prod_tile(xcd_remap(blockIdx.x, gridDim.x), static_cast<int>((p.na + 255) / 256), p.n_btiles, &at,
            &bt, &split);
  const int64_t a0 = static_cast<int64_t>(at) * 256, b0 = static_cast<int64_t>(bt) * 256;
  if (b0 >= nb) return;
  const int64_t per = ((K + p.splits - 1) / p.splits + 63) / 64 * 64;
  const int64_t kb = split * per < K ? split * per : K;
  const int64_t ke = kb + per < K ? kb + per : K;
  const int nk = static_cast<int>((ke - kb + 63) / 64);

  // Copy i of a wave: rows 2 (4 wave + i) + lane / 32 of a transposed operand's stage (512 bytes each),
  // rows 8 (4 wave + i) + lane / 8 of an operand held along K (128 bytes each). The lane's place in the
  // LDS row fetches the chunk that is permuted there. Columns past the operand's end repeat its last
  // chunk (they reach outputs past the end only).
  const uint32_t lda2 = static_cast<uint32_t>(2 * p.lda), ldb2 = static_cast<uint32_t>(2 * p.ldb);
  uint32_t offA[4], offB[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = 2 * (4 * wave + i) + (lane >> 5);
    const int c = 8 * ((lane & 31) ^ tr_swz<256>(r));
    const int64_t ca = a0 + c < p.na ? a0 + c : p.na - 8;
    offA[i] = static_cast<uint32_t>(2 * ca) + r * lda2;
    if (TRB) {
      const int64_t cb = b0 + c < p.ldb ? b0 + c : p.ldb - 8;
      offB[i] = static_cast<uint32_t>(2 * cb) + r * ldb2;
    } else {
      const int rb = 8 * (4 * wave + i) + (lane >> 3);
      const int64_t gr = rb < nb - b0 ? rb : nb - b0 - 1;
      offB[i] = static_cast<uint32_t>(2 * gr * p.ldb) + 16 * ((lane & 7) ^ row_swz(rb));
    }
  }
  const char* const baseA = reinterpret_cast<const char*>(p.A) + kb * lda2;
  const char* const baseB = reinterpret_cast<const char*>(p.B) +
                            (TRB ? kb * ldb2 : static_cast<int64_t>(2) * (b0 * p.ldb + kb));
  const uint32_t lds0 = lds_addr(smem) + wave * 4096;
  // The last stage of a range may hold fewer than 64 k: rows (or chunks) past them repeat the last row
  // (the first chunk) and count as 0 in the fragments.
  const int last = static_cast<int>(ke - kb - 64 * static_cast<int64_t>(nk - 1));
  auto copy_A = [&](int s, int slot) {
    const char* base = baseA + static_cast<int64_t>(s) * 64 * lda2;
    const bool tail = s == nk - 1 && last < 64;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t off = offA[i];
      if (tail) {
        const int r = 2 * (4 * wave + i) + (lane >> 5);
        off -= r < last ? 0u : static_cast<uint32_t>(r - last + 1) * lda2;
      }
      lds_dma16(base, off, lds0 + slot * TILE + i * 1024);
    }
  };
  auto copy_B = [&](int s, int slot) {
    const char* base = baseB + (TRB ? static_cast<int64_t>(s) * 64 * ldb2 : static_cast<int64_t>(s) * 128);
    const bool tail = s == nk - 1 && last < 64;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t off = offB[i];
      if (tail) {
        if (TRB) {
          const int r = 2 * (4 * wave + i) + (lane >> 5);
          off -= r < last ? 0u : static_cast<uint32_t>(r - last + 1) * ldb2;
        } else {
          const int c = (lane & 7) ^ row_swz(8 * (4 * wave + i) + (lane >> 3));
          off -= 8 * c < last ? 0u : 16u * c;
        }
      }
      lds_dma16(base, off, lds0 + BOFF + slot * TILE + i * 1024);
    }
  };

  f32x16 acc[NRA][NCB];
#pragma unroll
  for (int i = 0; i < NRA; ++i)
#pragma unroll
    for (int j = 0; j < NCB; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;

  // Fragments. Transposing read: lane l takes rows 8 (l / 32) + (l % 16) / 4 (and 4 further) of a
  // 16-deep k step, 8 bytes at column 16 ((l / 16) % 2) + 4 (l % 4) of a 32-column block; its row's
  // permutation moves the block's low two bits only.
  const int i16 = lane & 15, half = lane >> 5;
  const int tr0 = (8 * half + (i16 >> 2)) * 512 + ((lane >> 4) & 1) * 32 + (i16 & 3) * 8;
  int fa[NRA], fb[NCB];
#pragma unroll
  for (int i = 0; i < NRA; ++i) fa[i] = tr0 + 64 * ((4 * wa + i) ^ (i16 >> 2));
#pragma unroll
  for (int j = 0; j < NCB; ++j)
    fb[j] = BOFF + (TRB ? tr0 + 64 * ((2 * wb + j) ^ (i16 >> 2))
                        : (64 * wb + 32 * j + (lane & 31)) * 128);
  const int bx = 16 * (half ^ row_swz(lane & 31));
  bf16x8 af[2][NRA], bf[2][NCB];
  auto load_frags = [&](int aslot, int bslot, int kk, int ks) {  // k step kk of a stage, to set ks
    const char* sa = smem + aslot * TILE;
    const char* sb = smem + bslot * TILE;
#pragma unroll
    for (int i = 0; i < NRA; ++i) {
      const char* q = sa + fa[i] + kk * 8192;
      af[ks][i] = join(lds_read_tr(q), lds_read_tr(q + 2048));
    }
#pragma unroll
    for (int j = 0; j < NCB; ++j) {
      if constexpr (TRB) {
        const char* q = sb + fb[j] + kk * 8192;
        bf[ks][j] = join(lds_read_tr(q), lds_read_tr(q + 2048));
      } else {
        bf[ks][j] = *reinterpret_cast<const bf16x8*>(sb + fb[j] + ((32 * kk) ^ bx));
      }
    }
  };
  // Both operands: what a copy past the end repeats may hold infinities.
  auto mask = [&](int kk0, int left) {
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      const int n = left - 16 * (kk0 + ks) - 8 * half;
#pragma unroll
      for (int i = 0; i < NRA; ++i) af[ks][i] = keep_first(af[ks][i], n);
#pragma unroll
      for (int j = 0; j < NCB; ++j) bf[ks][j] = keep_first(bf[ks][j], n);
    }
  };
  auto mfmas = [&](int ks) {
#pragma unroll
    for (int i = 0; i < NRA; ++i)
#pragma unroll
      for (int j = 0; j < NCB; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(af[ks][i], bf[ks][j], acc[i][j], 0, 0, 0);
  };

  // Turns 2 s and 2 s + 1 take a stage's halves. A turn: its memory half (fragments, and copies into slots
  // that stage s - 1 has left), a barrier, its compute half, a barrier. Group 1 runs one barrier behind
  // group 0, so that each half of one group meets the other half of the other. The first fragments of an
  // odd turn are read in the even turn's compute half, into registers that its first MFMAs have left: with
  // all 24 transposing reads in one memory half that half was the longer one. At odd turns every wave
  // waits for its own copies of stage s + 1 (all but the 4 of stage s + 2 just issued) before the barrier
  // that opens the first memory half that reads stage s + 1.
  auto turn = [&](auto odd_c, int s, int a3, int b2) {  // a3 = s % 3, b2 = s % 2
    constexpr bool odd = decltype(odd_c)::value;
    if constexpr (!odd) load_frags(a3, b2, 0, 0);
    load_frags(a3, b2, odd ? 3 : 1, 1);
    if constexpr (!odd) {
      if (s >= 1 && s + 1 < nk) copy_B(s + 1, b2 ^ 1);
    } else {
      if (s + 2 < nk) copy_A(s + 2, a3 == 0 ? 2 : a3 - 1);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (s == nk - 1 && last < 64) mask(odd ? 2 : 0, last);
    if (odd && grp == 1) {
      if (s + 2 < nk) wait_vmcnt<4>(); else wait_vmcnt<0>();
    }
    pp_barrier();
    __builtin_amdgcn_s_setprio(1);  // the computing wave issues before its neighbour's copies and reads
    mfmas(0);
    if constexpr (!odd) {
      __builtin_amdgcn_sched_barrier(0);
      load_frags(a3, b2, 2, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
    mfmas(1);
    __builtin_amdgcn_s_setprio(0);
    if (odd && grp == 0) {
      if (s + 2 < nk) wait_vmcnt<4>(); else wait_vmcnt<0>();
    }
    if (!(grp == 1 && odd && s == nk - 1)) pp_barrier();
  };
  if (nk > 0) {
    copy_A(0, 0);
    copy_B(0, 0);
    if (nk > 1) {
      copy_A(1, 1);
      copy_B(1, 1);
      wait_vmcnt<8>();
    } else {
      wait_vmcnt<0>();
    }
    pp_barrier();
    if (grp == 1) pp_barrier();
    int a3 = 0;
    for (int s = 0; s < nk; ++s) {
      turn(std::false_type{}, s, a3, s & 1);
      turn(std::true_type{}, s, a3, s & 1);
      a3 = a3 == 2 ? 0 : a3 + 1;
    }
  }

  // No memory half reads the slots any more (group 0 passed the barrier closing the last one; group 1
  // reads none in its last compute half) and every copy has landed, so each wave stages its stores in its
  // own 16 KB of them.
  store_block<NRA, NCB, OUT>(acc, p, nb, b0 + 64 * wb, a0 + 128 * wa, split, lane, smem + wave * 16384);
}

// Few rows: the other operand streams past once, non-temporally. 60 rows, d = 2560, K = 151,936:
// 128-column tiles, two workgroups to a CU, 165 us (160 non-temporal); these 136 (144 before the splits
// took their stages in turn).
using RingFew = RingCfg<256, 64, 4, 2, 4, 64, true>;
using RingFew128 = RingCfg<256, 128, 4, 2, 3, 64, true>;
// Narrow outputs, two workgroups to a CU.
using RingNarrow = RingCfg<128, 128, 2, 2, 2>;
using RingNarrow64 = RingCfg<128, 64, 2, 2, 3>;
// Short sums: loads, stores and a few MFMAs a tile, which four workgroups to a CU hide from one another
// (us, outputs of 32768 x 4096 and 151936 x 4096, 256 and 200 terms: two workgroups of 64-deep stages 117
// and -, three with a third 32-deep slot 110 and 522, these 99 and 477; 256 x 128 tiles 101 and 498).
using RingShort = RingCfg<128, 128, 2, 2, 2, 32>;

template <class C, bool TRB, int OUT>
hipError_t launch_ring(Prod p, hipStream_t stream) {
  const int64_t na = (p.na + C::BA - 1) / C::BA, nb = (p.nb + C::BB - 1) / C::BB;
  const int64_t n = na * nb * p.splits;
  if (n > kMaxThreads / C::kThreads) return hipErrorInvalidConfiguration;
  p.n_btiles = static_cast<int>(nb);
  hipLaunchKernelGGL((prod_ring_kernel<C, TRB, OUT>), dim3(static_cast<unsigned>(n)),
                     dim3(C::kThreads), 0, stream, p);
  return hipGetLastError();
}

// Sums of 65 to 256 terms with both operands across the sum and a large output (the weight gradients of a
// few blocks): the output is much larger than what it is made of, so the kernel is a stream of stores with
// a few MFMAs between them. A workgroup of eight waves owns 512 columns of A, whose fragments for all K
// (64 KT at most) stay in registers, 64 columns a wave, and walks a range of B's columns 64 at a time: a
// [K, 64] tile per step, copied global -> LDS two steps ahead, one barrier a step. A's panel is read once
// per range and B once per panel. prod_kind says where it is the faster form.
// The stores are buffer stores, dropped by the hardware past the output's end, so that every step issues
// the same number of them and the wait for a tile can leave the stores since its copy in flight: memory
// operations of a wave complete in order.
constexpr int kStreamTile = 64, kStreamPanel = 512;
template <int KT, int OUT>
__global__ __launch_bounds__(512, 2) void prod_stream_kernel(const Prod p, int per_range) {
  constexpr int STAGE = KT * 8192, S = 3;         // bytes of a B tile: 64 KT rows of 128
  constexpr int PER = STAGE / 1024 / 8;           // copies per wave and step
  constexpr int NST = 8;                          // stores per wave and step
  constexpr int RING = S * STAGE;
  constexpr int AT = 2;                           // 64-row tiles of A's panel that pass through LDS at a time
  constexpr int LDS = RING + 8 * 4096 > AT * 65536 ? RING + 8 * 4096 : AT * 65536;
  static_assert(LDS <= 160 * 1024 && KT % AT == 0 && PER + 2 * NST <= 63, "LDS, vmcnt");
  __shared__ __attribute__((aligned(1024))) char smem[LDS];
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t K = p.count ? *p.count : p.K;
  // Panels of one range of B are consecutive, so that they share B's tiles in an XCD's L2.
  const int n_panels = static_cast<int>((p.na + kStreamPanel - 1) / kStreamPanel);
  const int L = xcd_remap(blockIdx.x, gridDim.x);
  const int panel = __builtin_amdgcn_readfirstlane(L % n_panels);
  const int range = __builtin_amdgcn_readfirstlane(L / n_panels);
  const int64_t a0 = static_cast<int64_t>(panel) * kStreamPanel;
  const int64_t tiles = (p.nb + kStreamTile - 1) / kStreamTile;
  const int64_t t0 = static_cast<int64_t>(range) * per_range;
  const int nt = static_cast<int>(tiles - t0 < per_range ? tiles - t0 : per_range);
  if (nt <= 0) return;
  const uint32_t lds0 = lds_addr(smem);
  const int i16 = lane & 15, half = lane >> 5;

  // A's fragments: 128 rows of the panel at a time through LDS (1 KB rows, one copy instruction each,
  // chunk c of row k at c ^ tr_swz(k)); rows past K repeat the last one, and count as 0 (in both operands:
  // what is repeated may hold infinities).
  bf16x8 af[4 * KT][2];
#pragma unroll
  for (int kt = 0; kt < KT; kt += AT) {
    if (64 * kt < K) {
#pragma unroll
      for (int i = 0; i < 8 * AT; ++i) {
        const int r = 8 * AT * wave + i;
        const int64_t k = 64 * kt + r < K ? 64 * kt + r : K - 1;
        const int64_t c = a0 + 8 * (lane ^ tr_swz<512>(r));
        lds_dma16(reinterpret_cast<const char*>(p.A) + 2 * k * p.lda,
                  static_cast<uint32_t>(2 * (c < p.na ? c : p.na - 8)), lds0 + r * 1024);
      }
      wait_vmcnt<0>();
      __syncthreads();
    }
#pragma unroll
    for (int ks = 0; ks < 4 * AT; ++ks)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        af[4 * kt + ks][i] = bf16x8{};
        if (64 * kt + 16 * ks < K) {
          const int k = 16 * ks + 8 * half + (i16 >> 2);
          const int chunk = (4 * (2 * wave + i) + 2 * ((lane >> 4) & 1) + ((i16 & 3) >> 1)) ^ tr_swz<512>(k);
          const char* q = smem + k * 1024 + chunk * 16 + (i16 & 1) * 8;
          af[4 * kt + ks][i] = keep_first(join(lds_read_tr(q), lds_read_tr(q + 4096)),
                                          static_cast<int>(K - 64 * kt) - 16 * ks - 8 * half);
        }
      }
    __syncthreads();
  }

  // B tiles: row k of 64 columns at 128 k, chunk c at c ^ tr_swz(k); a copy instruction covers 8 rows.
  uint32_t off[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int r = (wave * PER + i) * 8 + (lane >> 3);
    const int64_t k = r < K ? r : K - 1;
    off[i] = static_cast<uint32_t>(2 * k * p.ldb + 16 * ((lane & 7) ^ tr_swz<64>(r)));
  }
  auto copy = [&](int t) {
    if (t >= nt || K == 0) return;
    const int64_t at = t0 + t;
    const char* base = reinterpret_cast<const char*>(p.B) + 2 * kStreamTile * at;
    // The last tile may reach past B's columns: its chunks there are moved back onto the row's last one.
    const int64_t left = p.ldb - kStreamTile * at;  // >= 8
    const uint32_t to = lds0 + (t % S) * STAGE;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      uint32_t o = off[i];
      if (left < kStreamTile) {
        const int c = (lane & 7) ^ tr_swz<64>((wave * PER + i) * 8 + (lane >> 3));
        if (8 * c >= left) o -= 16u * static_cast<uint32_t>(c - (left / 8 - 1));
      }
      lds_dma16(base, o, to + (wave * PER + i) * 1024);
    }
  };
  copy(0);
  copy(1);
  char* const xp = smem + RING + wave * 4096;
  const int64_t aw = a0 + 64 * wave;
  for (int t = 0; t < nt; ++t) {
    // Issued since step t's copies, two steps ago: two steps' stores and, but for the last step, one step's
    // copies.
    if (t + 1 < nt) {
      if (t == 0) wait_vmcnt<PER>();
      else if (t == 1) wait_vmcnt<PER + NST>();
      else wait_vmcnt<PER + 2 * NST>();
    } else {
      if (t == 0) wait_vmcnt<0>();
      else if (t == 1) wait_vmcnt<NST>();
      else wait_vmcnt<2 * NST>();
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    copy(t + 2);  // into the slot of step t - 1, which every wave has read
    const char* sb = smem + (t % S) * STAGE;
    f32x16 acc[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
#pragma unroll
    for (int ks = 0; ks < 4 * KT; ++ks) {
      if (16 * ks < K) {
        bf16x8 bf[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int k = 16 * ks + 8 * half + (i16 >> 2);
          const int chunk = (4 * j + 2 * ((lane >> 4) & 1) + ((i16 & 3) >> 1)) ^ tr_swz<64>(k);
          const char* q = sb + k * 128 + chunk * 16 + (i16 & 1) * 8;
          bf[j] = join(lds_read_tr(q), lds_read_tr(q + 512));
        }
        if (16 * ks + 16 > K) {
#pragma unroll
          for (int j = 0; j < 2; ++j) bf[j] = keep_first(bf[j], static_cast<int>(K) - 16 * ks - 8 * half);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(af[ks][i], bf[j], acc[i][j], 0, 0, 0);
      }
    }
    // 32 rows x 64 columns at a time through LDS (chunk c of row r at c ^ (r % 8)): a store writes eight
    // 128-byte row segments.
    const int64_t b0 = kStreamTile * (t0 + t);
    const int64_t rows = p.nb - b0 < kStreamTile ? p.nb - b0 : kStreamTile;
    const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(p.out + b0 * p.na, 0,
                                                        static_cast<int>(2 * rows * p.na), 0x00027000);
    const int lr = lane & 31;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const f32x16& v = acc[i][j];
          *reinterpret_cast<bf16x4*>(xp + lr * 128 + ((4 * i + g) ^ (lr & 7)) * 16 + half * 8) =
              bf16x4{static_cast<__bf16>(v[4 * g]), static_cast<__bf16>(v[4 * g + 1]),
                     static_cast<__bf16>(v[4 * g + 2]), static_cast<__bf16>(v[4 * g + 3])};
        }
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
      for (int r0 = 0; r0 < 32; r0 += 8) {
        const int r = r0 + (lane >> 3), c = lane & 7;
        const u32x4 v = *reinterpret_cast<const u32x4*>(xp + r * 128 + (c ^ (r & 7)) * 16);
        const int64_t a = aw + 8 * c;
        const uint32_t o = a < p.na ? static_cast<uint32_t>(2 * ((32 * j + r) * p.na + a)) : 0x80000000u;
        __builtin_amdgcn_raw_buffer_store_b128(v, rsrc, o, 0, OUT == kOutStream ? 2 : 0);
      }
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
  }
}

template <int KT, int OUT>
hipError_t launch_stream(const Prod& p, hipStream_t stream) {
  const int64_t panels = (p.na + kStreamPanel - 1) / kStreamPanel;
  const int64_t tiles = (p.nb + kStreamTile - 1) / kStreamTile;
  const int64_t ranges = panels < 256 ? 256 / panels : 1;  // one workgroup to a CU
  const int64_t per = (tiles + ranges - 1) / ranges;
  const int64_t n = panels * ((tiles + per - 1) / per);
  if (n > kMaxThreads / 512 || per > 0x7fffffff) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL((prod_stream_kernel<KT, OUT>), dim3(static_cast<unsigned>(n)), dim3(512), 0, stream, p,
                     static_cast<int>(per));
  return hipGetLastError();
}

template <bool TRB, int OUT>
hipError_t launch_prod_out(Prod p, hipStream_t stream) {
  const ProdKind kind = prod_kind(TRB, p.na, p.nb, p.K);
  if (kind == kProdPp) {
    const int64_t na = (p.na + 255) / 256, nb = (p.nb + 255) / 256, n = na * nb * p.splits;
    if (n > kMaxThreads / 512) return hipErrorInvalidConfiguration;
    p.n_btiles = static_cast<int>(nb);
    hipLaunchKernelGGL((prod_pp_kernel<TRB, OUT>), dim3(static_cast<unsigned>(n)), dim3(512), 0, stream,
                       p);
    return hipGetLastError();
  }
  if constexpr (TRB) {
    if constexpr (OUT != kOutPart)
      if (kind == kProdStream)
        return p.K <= 128 ? launch_stream<2, OUT>(p, stream) : launch_stream<4, OUT>(p, stream);
    return launch_ring<RingShort, TRB, OUT>(p, stream);
  } else {
    if (kind == kProdFew)
      return p.nb > 64 ? launch_ring<RingFew128, TRB, OUT>(p, stream)
                       : launch_ring<RingFew, TRB, OUT>(p, stream);
    return p.nb > 64 ? launch_ring<RingNarrow, TRB, OUT>(p, stream)
                     : launch_ring<RingNarrow64, TRB, OUT>(p, stream);
  }
}

// fp32 sums of a product with one operand across the sum.
hipError_t launch_prod_part(const Prod& p, hipStream_t stream) {
  return launch_prod_out<false, kOutPart>(p, stream);
}

// A product of two operands across the sum in parts, and their sum.
template <class T, class A, class F>
hipError_t launch_weight_parts(A p, T* out, hipStream_t stream, F launch) {
  p.part_stride = p.na * p.nb;
  const hipError_t e = launch(p, stream);
  if (e != hipSuccess) return e;
  const int64_t blocks = (p.part_stride + 1023) / 1024;  // of at most 512 tiles
  hipLaunchKernelGGL(weight_finish_kernel<T>, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, stream, p.part,
                     p.part_stride, p.splits, out);
  return hipGetLastError();
}

// The bf16 product of two operands across the sum. An output that would fill the 256 MB Infinity Cache is
// written past it (151936 x 2560 outputs of 60 terms 174 ->
// 141 us); a smaller one stays there for its next reader (50257 x 1000 outputs 34 us, 43 non-temporally).
hipError_t launch_prod(const Prod& p, hipStream_t stream) {
  if (p.splits > 1) return launch_weight_parts<__bf16>(p, p.out, stream, launch_prod_out<true, kOutPart>);
  return 2 * p.na * p.nb >= (int64_t(256) << 20) ? launch_prod_out<true, kOutStream>(p, stream)
                                                : launch_prod_out<true, kOutKeep>(p, stream);
}

// ---------------------------------------------------------------------------------------
// fp32 GEMM: out(a, b) = sum_k A(k, a) B(k, b) on v_mfma_f32_32x32x2_f32 (fp32 products and sums). Four
// waves, 32-deep stages staged through registers. An operand is either [K, n] (TR) or [n, K] row-major;
// any size and 4-byte alignment. ROWS = 64: 128 x 64 tile, waves of 64 a x 32 b, three workgroups
// to a CU. ROWS = 32, for up to 32 rows: 128 x 32 tile, waves of 32 a x 32 b. Measured: 128 x 128 tiles take
// 11 us for 8 rows at d = 64, V = 256, 4 of them MFMAs on rows that are not there, these 5.6.
// Tile log-masses are of 32 ids in both, so that a row's sums do not depend on the kernel.

struct F32Args {
  const float* A;
  const float* B;
  int64_t lda, ldb, na, nb, K;
  const int32_t* count_b;  // if set: nb
  const int32_t* count_k;  // if set: K
  // products
  float* part;             // [splits, nb_max, na]
  int64_t part_stride;
  int accumulate;
  float* out;              // [nb, na]
  int splits;
  int n_btiles;
  // head
  const TrainRow* rows;
  float* lmass;
  float* tgt;
  float* grad;
  int64_t ldg, vbase;
  int nT;
};

enum F32Epi : int { kF32Part = 0, kF32Out = 1, kF32Nll = 2, kF32Grad = 3 };

// 32 x N values of an operand in LDS as rows of k, N / 32 groups of four a thread: eight lanes read 128
// contiguous bytes (of a row of K with TR, else along K; with 64 bytes a thread the vector cache's lines
// were touched four times). Column i of row k lies at i ^ perm(k): the halves of a wave read neighbouring
// k from other banks, and the eight lanes of an operand along K write theirs to other banks. The loads are
// buffer loads, which give 0 past the array's end, so that none of them has a condition (with one, the two
// paths' loads met in the same registers and each stage waited for its loads before its MFMAs: 120 us for
// 512 x 500 against 20,000 ids): TR past the last row (values past a row's end belong to the next one, and
// to outputs that do not exist), else with the rows past the last one repeating it and the values past K
// set to 0 as they are stored.
template <bool TR, int N>
struct F32Stage {
  static constexpr int G = N / 32, LD = N < 64 ? 64 : N;
  static __device__ __forceinline__ int perm(int k) { return 8 * ((k >> 2) & 7) ^ 32 * (k & 1); }
  static __device__ __forceinline__ int at(int k, int i) { return k * LD + (i ^ perm(k)); }
  f32x4 r[G];
  uint32_t off[G];  // of a group in the tile, bytes
  __device__ __forceinline__ void init(int64_t ld, int64_t i0, int64_t n) {
    const int t8 = threadIdx.x >> 3, c4 = 4 * (threadIdx.x & 7);
#pragma unroll
    for (int j = 0; j < G; ++j) {
      if constexpr (TR) {
        off[j] = static_cast<uint32_t>(4 * (t8 * ld + c4 + 32 * j));
      } else {
        const int row = t8 + 32 * j;
        off[j] = static_cast<uint32_t>(4 * ((row < n - i0 ? row : n - i0 - 1) * ld + c4));
      }
    }
  }
  // rows: of the array (K for TR, n else).
  __device__ __forceinline__ void load(const float* X, int64_t ld, int64_t i0, int64_t k0, int64_t rows) {
    const int64_t from = TR ? k0 * ld + i0 : i0 * ld + k0;
    const int64_t left = 4 * (rows * ld - from);
    const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<float*>(X + from), 0,
        static_cast<int>(left < 0xffffffffll ? static_cast<uint32_t>(left) : 0xffffffffu), 0x00027000);
#pragma unroll
    for (int j = 0; j < G; ++j)
      r[j] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, off[j], 0, 0));
  }
  // left: k of the stage that are there.
  __device__ __forceinline__ void store(float* S, int64_t left) {
    const int t8 = threadIdx.x >> 3, c4 = 4 * (threadIdx.x & 7);
    if constexpr (TR) {
#pragma unroll
      for (int j = 0; j < G; ++j) *reinterpret_cast<f32x4*>(S + at(t8, c4 + 32 * j)) = r[j];
    } else {
      if (left < 32) {
#pragma unroll
        for (int j = 0; j < G; ++j)
#pragma unroll
          for (int q = 0; q < 4; ++q) r[j][q] = c4 + q < left ? r[j][q] : 0.0f;
      }
#pragma unroll
      for (int j = 0; j < G; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) S[at(c4 + q, t8 + 32 * j)] = r[j][q];
    }
  }
};

template <bool TRA, bool TRB, int EPI, int ROWS>
__global__ __launch_bounds__(256) void gemm_f32_kernel(const F32Args p) {
  constexpr int BK = 32, NRA = ROWS / 32, IDS = 32 * NRA;  // a of a wave
  static_assert(ROWS == 32 || ROWS == 64, "wave layouts");
  using SA = F32Stage<TRA, 128>;
  using SB = F32Stage<TRB, ROWS>;
  __shared__ __attribute__((aligned(16))) float As[2][BK * SA::LD], Bs[2][BK * SB::LD];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int half = lane >> 5;
  const int wa = ROWS == 64 ? (wave & 1) * 64 : wave * 32, wb = ROWS == 64 ? (wave >> 1) * 32 : 0;
  const int64_t K = p.count_k ? *p.count_k : p.K;
  const int64_t nb = p.count_b ? *p.count_b : p.nb;
  const int n_atiles = static_cast<int>((p.na + 127) / 128);
  const int bt = blockIdx.x % p.n_btiles, rest = blockIdx.x / p.n_btiles;
  // In scalar registers: the loads' resources are made of these.
  const int at = __builtin_amdgcn_readfirstlane(rest % n_atiles);
  const int split = __builtin_amdgcn_readfirstlane(rest / n_atiles);
  const int64_t a0 = static_cast<int64_t>(at) * 128;
  const int64_t b0 = static_cast<int64_t>(__builtin_amdgcn_readfirstlane(bt)) * ROWS;
  if (b0 >= nb) return;
  const int64_t per = ((K + p.splits - 1) / p.splits + BK - 1) / BK * BK;
  const int64_t kb = split * per < K ? split * per : K;
  const int64_t ke = kb + per < K ? kb + per : K;

  f32x16 acc[NRA];
#pragma unroll
  for (int i = 0; i < NRA; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[i][r] = 0.0f;

  if (kb < ke) {
    SA ra;
    SB rb;
    ra.init(p.lda, a0, p.na);
    rb.init(p.ldb, b0, nb);
    auto load = [&](int64_t k0) {
      ra.load(p.A, p.lda, a0, k0, TRA ? K : p.na);
      rb.load(p.B, p.ldb, b0, k0, TRB ? K : nb);
    };
    auto store = [&](int buf, int64_t k0) {
      ra.store(As[buf], ke - k0);
      rb.store(Bs[buf], ke - k0);
    };
    load(kb);
    store(0, kb);
    __syncthreads();
    int buf = 0;
    for (int64_t k0 = kb; k0 < ke; k0 += BK, buf ^= 1) {
      const bool more = k0 + BK < ke;
      if (more) load(k0 + BK);
      const float* sa = As[buf] + half * SA::LD;
      const float* sb = Bs[buf] + half * SB::LD;
#pragma unroll
      for (int kk = 0; kk < BK; kk += 2) {  // k = kk + half, kk even
        const int x = SA::perm(kk) ^ (32 * half);
        const float b = sb[kk * SB::LD + ((wb + (lane & 31)) ^ x)];
#pragma unroll
        for (int i = 0; i < NRA; ++i)
          acc[i] = __builtin_amdgcn_mfma_f32_32x32x2f32(
              sa[kk * SA::LD + ((wa + 32 * i + (lane & 31)) ^ x)], b, acc[i], 0, 0, 0);
      }
      if (more) store(buf ^ 1, k0 + BK);
      __syncthreads();
    }
  }

  // Lane l holds b = l % 32 of its wave's and, in registers 4 g .. 4 g + 3 of block i, a = 32 i + 8 g +
  // 4 (l / 32) + {0 .. 3}.
  const int64_t b = b0 + wb + (lane & 31), aw = a0 + wa;
  if constexpr (EPI == kF32Part || EPI == kF32Out) {
    if (b >= nb) return;
    float* const row = EPI == kF32Part ? p.part + split * p.part_stride + b * p.na : p.out + b * p.na;
    const bool add = EPI == kF32Part && p.accumulate;
#pragma unroll
    for (int i = 0; i < NRA; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int64_t a = aw + 32 * i + 8 * g + 4 * half;
        f32x4 v = {acc[i][4 * g], acc[i][4 * g + 1], acc[i][4 * g + 2], acc[i][4 * g + 3]};
        if (a + 4 <= p.na) {
          f32x4u* o = reinterpret_cast<f32x4u*>(row + a);
          if (add) v += *o;
          *o = v;
        } else {
#pragma unroll
          for (int q = 0; q < 4; ++q)
            if (a + q < p.na) row[a + q] = v[q] + (add ? row[a + q] : 0.0f);
        }
      }
  } else {
    // a: ids, b: rows (the lane layout of the bf16 head's epilogues).
    if (aw >= p.na) return;
    const int lim = static_cast<int>(p.na - aw < IDS ? p.na - aw : IDS) - 4 * half;
    if constexpr (EPI == kF32Nll) {
      const int64_t o = b < nb ? p.rows[b].token - aw - 4 * half : -1;
#pragma unroll
      for (int i = 0; i < NRA; ++i) {
        if (aw + 32 * i >= p.na) break;
        float x[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r] = 32 * i + 8 * (r >> 2) + (r & 3) < lim ? acc[i][r] : -INFINITY;
        if (o >= 32 * i && o < 32 * i + 32 && o < lim && !(o & 4)) {
          float t = 0.0f;
#pragma unroll
          for (int r = 0; r < 16; ++r) t = o == 32 * i + 8 * (r >> 2) + (r & 3) ? x[r] : t;
          p.tgt[b] = t;
        }
        float mx = -INFINITY;
#pragma unroll
        for (int r = 0; r < 16; ++r) mx = fmaxf(mx, x[r]);
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const float top = mx > -INFINITY ? mx : 0.0f;  // logits of minus infinity only: mass 0
        float s = 0.0f;
#pragma unroll
        for (int r = 0; r < 16; ++r) s += __expf(x[r] - top);
        s += __shfl_xor(s, 32);
        if (b < nb && half == 0) p.lmass[b * p.nT + aw / 32 + i] = mx + logf(s);
      }
    } else {
      if (b >= nb) return;
      const TrainRow row = p.rows[b];
      const int64_t o = row.token - p.vbase - aw - 4 * half;
#pragma unroll
      for (int i = 0; i < NRA; ++i)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          f32x4 y;
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const int at0 = 32 * i + 8 * g + q;
            float u = expf(acc[i][4 * g + q] - row.shift);
            u = o == at0 ? row.at_token : u;
            y[q] = at0 < lim ? u : 0.0f;
          }
          *reinterpret_cast<f32x4*>(p.grad + b * p.ldg + aw + 32 * i + 8 * g + 4 * half) = y;
        }
    }
  }
}

template <bool TRA, bool TRB, int EPI, int ROWS>
hipError_t launch_f32_rows(F32Args p, hipStream_t stream) {
  const int64_t na = (p.na + 127) / 128, nb = (p.nb + ROWS - 1) / ROWS;
  const int64_t n = na * nb * p.splits;
  if (n > kMaxThreads / 256) return hipErrorInvalidConfiguration;
  p.n_btiles = static_cast<int>(nb);
  hipLaunchKernelGGL((gemm_f32_kernel<TRA, TRB, EPI, ROWS>), dim3(static_cast<unsigned>(n)), dim3(256), 0,
                     stream, p);
  return hipGetLastError();
}

template <bool TRA, bool TRB, int EPI>
hipError_t launch_f32(const F32Args& p, hipStream_t stream) {
  if constexpr (!TRB)  // the products over the rows have the vocabulary there, many ids
    if (p.nb <= kF32FewRows) return launch_f32_rows<TRA, TRB, EPI, 32>(p, stream);
  return launch_f32_rows<TRA, TRB, EPI, 64>(p, stream);
}

// dh of every row: the sum of its parts times its scale, 0 for the rows that do not count. A wave takes
// 256 columns of a row.
template <class T>
__global__ __launch_bounds__(64) void dh_finish_kernel(const NllArgs a, int64_t part_stride) {
  const int64_t m = blockIdx.x;
  const int at = a.inv[m / a.R];
  const int64_t i = static_cast<int64_t>(at) * a.R + m % a.R;
  T* out = static_cast<T*>(a.dh) + m * a.d;
  const int j = blockIdx.y * 256 + 4 * threadIdx.x;
  if (j >= a.d) return;
  const float scale = at >= 0 ? a.rows[i].scale : 0.0f;
  if (j + 4 <= a.d) {
    f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
    if (at >= 0) v = sum_parts(a.part + i * a.d + j, part_stride, a.splits) * scale;
    if constexpr (sizeof(T) == 2)
      store4(out + j, v);
    else
      *reinterpret_cast<f32x4u*>(out + j) = v;
  } else {  // fp32 with d % 4 != 0
    for (int c = j; c < a.d; ++c) {
      float v = 0.0f;
      if (at >= 0)
        for (int s = 0; s < a.splits; ++s) v += a.part[s * part_stride + i * a.d + c];
      out[c] = static_cast<T>(at >= 0 ? v * scale : 0.0f);
    }
  }
}

// The expander's trunk gradient (the product's parts and the residual path's R branch gradients, in fp32,
// rounded once) and bias gradient, in one launch: the first n_dh workgroups take blocks of 256 columns of
// trunk rows, one a wave at a time, the others 64 features each.
__global__ __launch_bounds__(256) void expand_finish_kernel(const ExpandBackwardArgs a, int64_t n_dh) {
  const int d = a.d, R = static_cast<int>(a.R);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (blockIdx.x < n_dh) {
    const int blocks = (d + 255) / 256;
    for (int64_t at = static_cast<int64_t>(blockIdx.x) * 4 + wave; at < a.P * blocks; at += n_dh * 4) {
      const int64_t p = at / blocks;
      const int j = static_cast<int>(at % blocks) * 256 + 4 * lane;
      if (j >= d) continue;
      const __bf16* g = static_cast<const __bf16*>(a.dout) + p * R * d + j;
      f32x4 v = sum_parts(a.part + p * d + j, a.P * d, a.splits);
#pragma unroll 8
      for (int z = 0; z < R; ++z) {
        const bf16x4 u = *reinterpret_cast<const bf16x4*>(g + static_cast<int64_t>(z) * d);
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] += static_cast<float>(u[q]);
      }
      store4(static_cast<__bf16*>(a.dh) + p * d + j, v);
    }
    return;
  }
  // dc: the sum over the trunk rows of every branch feature's gradient, 32 rows side by side.
  __shared__ float part[4][65];
  const int64_t n = a.R * d, j0 = (blockIdx.x - n_dh) * 64;
  const int c = threadIdx.x & 7, r = threadIdx.x >> 3;
  const int64_t j = j0 + 8 * c;
  float s[8] = {};
  if (j < n) {
    const __bf16* dout = static_cast<const __bf16*>(a.dout) + j;
#pragma unroll 8
    for (int64_t p = r; p < a.P; p += 32) {
      const bf16x8 v = *reinterpret_cast<const bf16x8*>(dout + p * n);
#pragma unroll
      for (int i = 0; i < 8; ++i) s[i] += static_cast<float>(v[i]);
    }
  }
  // The eight rows of a wave first, then the four waves.
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int o = 8; o < 64; o <<= 1) s[i] += __shfl_xor(s[i], o);
  if (lane < 8) {
#pragma unroll
    for (int i = 0; i < 8; ++i) part[wave][8 * c + i] = s[i];
  }
  __syncthreads();
  if (threadIdx.x < 64 && j0 + threadIdx.x < n)
    static_cast<__bf16*>(a.dc)[j0 + threadIdx.x] =
        static_cast<__bf16>((part[0][threadIdx.x] + part[1][threadIdx.x]) +
                            (part[2][threadIdx.x] + part[3][threadIdx.x]));
}

// Ids v0 .. v0 + n - 1 of the backward pass: their part of the logits' gradient, added to the sums of dh, and
// their rows of dw. Without rows (M = 0) only dw is written: products over no terms.
hipError_t nll_piece_bf16(const NllArgs& a, int64_t v0, int64_t n, hipStream_t stream) {
  const int64_t M = a.P * a.R;
  const __bf16* w = static_cast<const __bf16*>(a.w) + v0 * a.d;
  if (M > 0) {
    HeadTrainArgs h{};
    h.M = M;
    h.V = n;
    h.d = a.d;
    h.h = a.hc;
    h.w = w;
    h.count = a.count;
    h.rows = a.rows;
    h.grad = a.grad;
    h.ldg = a.piece;
    h.vbase = v0;
    hipError_t e = launch_head_train(h, true, stream);
    if (e != hipSuccess) return e;
    Prod p{};
    p.A = w;
    p.lda = p.na = a.d;
    p.B = static_cast<const __bf16*>(a.grad);
    p.ldb = a.piece;
    p.nb = M;
    p.K = n;
    p.count = a.count;
    p.part = a.part;
    p.part_stride = M * a.d;
    p.accumulate = v0 > 0;
    p.splits = a.splits;
    e = launch_prod_part(p, stream);
    if (e != hipSuccess) return e;
  }
  if (!a.dw) return hipSuccess;
  Prod q{};
  q.A = static_cast<const __bf16*>(a.hs);
  q.lda = q.na = a.d;
  q.B = static_cast<const __bf16*>(a.grad);
  q.ldb = a.piece;
  q.nb = n;
  q.K = M;
  q.count = M > 0 ? a.count : nullptr;
  q.part = a.dw_part;
  q.out = static_cast<__bf16*>(a.dw) + v0 * a.d;
  q.splits = a.dw_splits;
  return launch_prod(q, stream);
}

hipError_t nll_piece_f32(const NllArgs& a, int64_t v0, int64_t n, hipStream_t stream) {
  const int64_t M = a.P * a.R;
  const float* w = static_cast<const float*>(a.w) + v0 * a.d;
  if (M > 0) {
    F32Args p{};
    p.A = w;
    p.B = static_cast<const float*>(a.hc);
    p.lda = p.ldb = p.K = a.d;
    p.na = n;
    p.nb = M;
    p.count_b = a.count;
    p.splits = 1;
    p.rows = a.rows;
    p.grad = static_cast<float*>(a.grad);
    p.ldg = a.piece;
    p.vbase = v0;
    hipError_t e = launch_f32<false, false, kF32Grad>(p, stream);
    if (e != hipSuccess) return e;
    F32Args q{};
    q.A = w;
    q.lda = q.na = a.d;
    q.B = static_cast<const float*>(a.grad);
    q.ldb = a.piece;
    q.nb = M;
    q.K = n;
    q.count_b = a.count;
    q.part = a.part;
    q.part_stride = M * a.d;
    q.accumulate = v0 > 0;
    q.splits = a.splits;
    e = launch_f32<true, false, kF32Part>(q, stream);
    if (e != hipSuccess) return e;
  }
  if (!a.dw) return hipSuccess;
  F32Args r{};
  r.A = static_cast<const float*>(a.hs);
  r.lda = r.na = a.d;
  r.B = static_cast<const float*>(a.grad);
  r.ldb = a.piece;
  r.nb = n;
  r.K = M;
  r.count_k = M > 0 ? a.count : nullptr;
  r.part = a.dw_part;
  r.out = static_cast<float*>(a.dw) + v0 * a.d;
  r.splits = a.dw_splits;
  if (r.splits > 1) return launch_weight_parts<float>(r, r.out, stream, launch_f32<true, true, kF32Part>);
  return launch_f32<true, true, kF32Out>(r, stream);
}

}  // namespace

hipError_t launch_nll(const NllArgs& a, hipStream_t stream) {
  const int64_t M = a.P * a.R;
  const int nT = static_cast<int>(nll_tiles(a.bf16, a.V));
  hipError_t e = gather_rows(a, stream);
  if (e != hipSuccess) return e;
  if (a.bf16) {
    HeadTrainArgs h{};
    h.M = M;
    h.V = a.V;
    h.d = a.d;
    h.h = a.hc;
    h.w = a.w;
    h.count = a.count;
    h.rows = a.rows;
    h.lmass = a.lmass;
    h.tgt = a.tgt;
    e = launch_head_train(h, false, stream);
  } else {
    F32Args p{};
    p.A = static_cast<const float*>(a.w);
    p.B = static_cast<const float*>(a.hc);
    p.lda = p.ldb = p.K = a.d;
    p.na = a.V;
    p.nb = M;
    p.count_b = a.count;
    p.splits = 1;
    p.rows = a.rows;
    p.lmass = a.lmass;
    p.tgt = a.tgt;
    p.nT = nT;
    e = launch_f32<false, false, kF32Nll>(p, stream);
  }
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(nll_finish_kernel, dim3(static_cast<unsigned>((M + 3) / 4)), dim3(256), 0, stream,
                     a, nT);
  return hipGetLastError();
}

hipError_t launch_nll_backward(const NllArgs& a, hipStream_t stream) {
  const int64_t M = a.P * a.R;
  if (M > 0) {
    const hipError_t e = gather_rows(a, stream);
    if (e != hipSuccess) return e;
  }
  for (int64_t v0 = 0; v0 < a.V; v0 += a.piece) {
    const int64_t n = a.V - v0 < a.piece ? a.V - v0 : a.piece;
    const hipError_t e = a.bf16 ? nll_piece_bf16(a, v0, n, stream) : nll_piece_f32(a, v0, n, stream);
    if (e != hipSuccess) return e;
  }
  if (M == 0) return hipSuccess;
  const dim3 grid(static_cast<unsigned>(M), static_cast<unsigned>((a.d + 255) / 256));
  if (a.bf16)
    hipLaunchKernelGGL(dh_finish_kernel<__bf16>, grid, dim3(64), 0, stream, a, M * a.d);
  else
    hipLaunchKernelGGL(dh_finish_kernel<float>, grid, dim3(64), 0, stream, a, M * a.d);
  return hipGetLastError();
}

hipError_t launch_expand_backward(const ExpandBackwardArgs& a, hipStream_t stream) {
  const int64_t n = a.R * a.d;
  hipError_t e = hipSuccess;
  if (a.dh) {
    Prod p{};
    p.A = static_cast<const __bf16*>(a.W);
    p.lda = p.na = a.d;
    p.B = static_cast<const __bf16*>(a.dout);
    p.ldb = n;
    p.nb = a.P;
    p.K = n;
    p.part = a.part;
    p.part_stride = a.P * a.d;
    p.splits = a.splits;
    e = launch_prod_part(p, stream);
    if (e != hipSuccess) return e;
  }
  if (a.dW) {
    Prod q{};
    q.A = static_cast<const __bf16*>(a.h);
    q.lda = q.na = a.d;
    q.B = static_cast<const __bf16*>(a.dout);
    q.ldb = n;
    q.nb = n;
    q.K = a.P;
    q.part = a.dW_part;
    q.out = static_cast<__bf16*>(a.dW);
    q.splits = a.dW_splits;
    e = launch_prod(q, stream);
    if (e != hipSuccess) return e;
  }
  int64_t n_dh = a.dh ? (a.P * ((a.d + 255) / 256) + 3) / 4 : 0;
  n_dh = n_dh < 1 << 20 ? n_dh : 1 << 20;
  const int64_t blocks = n_dh + (a.dc ? (n + 63) / 64 : 0);  // at most 2^20 + 2^17
  if (blocks == 0) return hipSuccess;
  hipLaunchKernelGGL(expand_finish_kernel, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, stream, a,
                     n_dh);
  return hipGetLastError();
}

}  // namespace dbl
