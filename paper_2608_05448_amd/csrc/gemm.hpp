// What the matrix-product kernels share: the tile order, the direct copies global -> LDS, and the head's
// epilogue. Internal; everything is local to the translation unit that includes it.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.hpp"

namespace dbl {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));

constexpr int kVTile = 128;
constexpr float kLog2e = 1.4426950408889634f;

// Argmax of a row across vocabulary tiles: every tile contributes the 64-bit key
// (order-preserving bits of its maximum logit, ~id) through an atomic maximum, so the winner is
// the largest logit and, among equal logits, the lowest id. -0 is folded into +0.
__device__ __forceinline__ uint64_t argmax_key(float x, int64_t v) {
  uint32_t u = __float_as_uint(x + 0.0f);
  u = (u & 0x80000000u) ? ~u : (u | 0x80000000u);
  return (static_cast<uint64_t>(u) << 32) | (0xFFFFFFFFu - static_cast<uint32_t>(v));
}

// Epilogue of the register-staged kernel: the same results as tile_logsoftmax_store, with
// the stores routed through a 16 KB LDS scratch per wave (xp). In the register layout a
// 16-byte store instruction covers 32 rows, 32 bytes each; every row of tls is V * 4 bytes from
// the next, so each such instruction needs tens of address translations, which the vector L1
// serialises. Here the wave writes its 32 rows x 128 ids to LDS as 512-byte rows (16-byte chunk
// c of row r at chunk c ^ (r % 16): conflict-free both ways) and reads them back so that each
// store instruction writes two whole 512-byte row segments. One block of 32 rows at a time:
// its 64 logits per lane are copied out of the accumulators once; in the vocabulary's last,
// partial tile the ids past V are set to -inf first, so every tile takes the same arithmetic.
// MASKED: also the whole tiles of a partial 32-row block take the non-temporal stores (with few
// branch rows that is every tile; in the 256-row kernel the second form cost 1% of the call).
template <int NRB, int NCB, bool ARG, bool MASKED = false>
__device__ __forceinline__ void tile_logsoftmax_store_lds(f32x16 (&acc)[NRB][NCB], float* tls,
                                                          float* lmass, uint64_t* amax,
                                                          int64_t M, int64_t V, int nT,
                                                          int64_t v0w, int64_t m0w, int lane,
                                                          char* xp) {
  const int half = lane >> 5;
  const int lr = lane & 31;
  const int t = static_cast<int>(v0w / kVTile);
  const int vlim = static_cast<int>(V - v0w < kVTile ? V - v0w : kVTile);  // ids in this tile
  const bool full = vlim == kVTile;
  constexpr int NX = NRB * 16;
#pragma unroll
  for (int cb = 0; cb < NCB; ++cb) {
    __builtin_amdgcn_sched_barrier(0);
    const int64_t m = m0w + cb * 32 + lr;
    float x[NX];  // x[16 rb + r]: id 32 rb + 8 (r / 4) + 4 half + r % 4 of the tile
#pragma unroll
    for (int rb = 0; rb < NRB; ++rb)
#pragma unroll
      for (int r = 0; r < 16; ++r) x[16 * rb + r] = acc[rb][cb][r];
    // Id offset of x[16 rb + r] in the tile: 32 rb + 8 (r / 4) + (r % 4) + 4 half; the
    // compile-time part is compared against limits shifted by 4 half, so no per-value offset
    // is held in a register.
    if (!full) {
      const int lim = vlim - 4 * half;
#pragma unroll
      for (int rb = 0; rb < NRB; ++rb)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (rb * 32 + 8 * (r >> 2) + (r & 3) >= lim) x[16 * rb + r] = -INFINITY;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int i = 0; i < NX; ++i) mx = fmaxf(mx, x[i]);
    int vi = 0;  // offset in the tile of this lane's first maximum (ARG only)
    if constexpr (ARG) {
      vi = 1 << 30;
#pragma unroll
      for (int rb = NRB - 1; rb >= 0; --rb)
#pragma unroll
        for (int r = 15; r >= 0; --r)
          vi = x[16 * rb + r] == mx ? rb * 32 + 8 * (r >> 2) + (r & 3) : vi;
      vi = vi == (1 << 30) ? 0 : vi + 4 * half;
      const float omx = __shfl_xor(mx, 32);
      const int ovi = __shfl_xor(vi, 32);
      if (omx > mx || (omx == mx && ovi < vi)) {
        mx = omx;
        vi = ovi;
      }
    } else {
      mx = fmaxf(mx, __shfl_xor(mx, 32));
    }
    const float nb = -mx * kLog2e;
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < NX; ++i) s += __builtin_amdgcn_exp2f(fmaf(x[i], kLog2e, nb));
    s += __shfl_xor(s, 32);
    const float lm = mx + __logf(s);
    if (m < M && half == 0) {
      lmass[m * nT + t] = lm;
      if constexpr (ARG)
        atomicMax(reinterpret_cast<unsigned long long*>(amax + m),
                  static_cast<unsigned long long>(argmax_key(mx, v0w + vi)));
    }
    float* const base = tls + (m0w + cb * 32) * V + v0w;  // wave-uniform
#pragma unroll
    for (int rb = 0; rb < NRB; ++rb)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        float4 o;
        o.x = x[16 * rb + 4 * g + 0] - lm;
        o.y = x[16 * rb + 4 * g + 1] - lm;
        o.z = x[16 * rb + 4 * g + 2] - lm;
        o.w = x[16 * rb + 4 * g + 3] - lm;
        const int chunk = (rb * 8 + 2 * g + half) ^ (lr & 15);
        *reinterpret_cast<float4*>(xp + lr * 512 + chunk * 16) = o;
      }
    // Wave-private LDS region: the writes above precede these reads in the wave's LDS queue.
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    float4 o[16];  // o[jj]: ids 4 lr .. 4 lr + 3 of block row 2 jj + half
#pragma unroll
    for (int jj = 0; jj < 16; ++jj) {
      const int rr = 2 * jj + half;
      o[jj] = *reinterpret_cast<const float4*>(xp + rr * 512 + ((lr ^ (rr & 15)) * 16));
    }
    // 16-byte stores at any alignment of the row (global vector stores need 4-byte alignment only).
    // Whole blocks are written non-temporally: the 256 KB a workgroup writes per tile would otherwise
    // evict the operand slabs its XCD's other tiles are still reading from L2 (1% faster; where the
    // weight is streamed once, at 64 rows and d = 2560, 168 -> 157 us).
    const int64_t rows = M - (m0w + cb * 32);  // of this block, 32 or more if it is whole
    if (full && rows >= 32) {
      const uint32_t lo = static_cast<uint32_t>(half * V + 4 * lr);  // 32-bit lane offsets
      const uint32_t step = static_cast<uint32_t>(2 * V);
#pragma unroll
      for (int jj = 0; jj < 16; ++jj)
        __builtin_nontemporal_store(f32x4u{o[jj].x, o[jj].y, o[jj].z, o[jj].w},
                                    reinterpret_cast<f32x4u*>(base + (lo + jj * step)));
    } else if (MASKED && full) {
      const uint32_t lo = static_cast<uint32_t>(half * V + 4 * lr);
      const uint32_t step = static_cast<uint32_t>(2 * V);
#pragma unroll
      for (int jj = 0; jj < 16; ++jj)
        if (2 * jj + half < rows)
          __builtin_nontemporal_store(f32x4u{o[jj].x, o[jj].y, o[jj].z, o[jj].w},
                                      reinterpret_cast<f32x4u*>(base + (lo + jj * step)));
    } else {
#pragma unroll
      for (int jj = 0; jj < 16; ++jj) {
        const int rr = 2 * jj + half;
        if (m0w + cb * 32 + rr < M) {
          float* q = base + rr * V + 4 * lr;
          if (4 * lr + 3 < vlim) {
            *reinterpret_cast<f32x4u*>(q) = f32x4u{o[jj].x, o[jj].y, o[jj].z, o[jj].w};
          } else {
            if (4 * lr + 0 < vlim) q[0] = o[jj].x;
            if (4 * lr + 1 < vlim) q[1] = o[jj].y;
            if (4 * lr + 2 < vlim) q[2] = o[jj].z;
            if (4 * lr + 3 < vlim) q[3] = o[jj].w;
          }
        }
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  }
}

// Maps the hardware workgroup id to a logical tile id so that consecutive logical ids land on
// the same XCD: workgroups are dispatched round-robin over the 8 XCDs, each with its own L2.
__device__ __forceinline__ int xcd_remap(int id, int n) {
  const int q = n >> 3, rem = n & 7;
  const int x = id & 7, s = id >> 3;
  return x < rem ? x * (q + 1) + s : rem * (q + 1) + (x - rem) * q + s;
}

// Logical tile id -> (vocabulary tile, branch-row tile). Branch-row tiles are taken in groups
// of up to g; a group sweeps every vocabulary tile before the next group starts, and within a
// vocabulary tile the group's branch-row tiles are consecutive. With groups of 4, the ~32
// workgroups resident on one XCD cover about 8 vocabulary x 4 branch-row tiles: each slab of w
// is read by up to 4 of them and each slab of h by about 8, from that XCD's L2. Measured: groups
// of 4 are 1% faster than 8 at 8 branch-row tiles (the Qwen3-8B head) and 1.7% at 32 (B = 256,
// K = 8, R = 4), 3% faster than no grouping; with 128 branch-row tiles (a 128-block chunk at
// K = R = 16, where each group re-streams all of w from HBM) groups of 8 are 1.7% faster than 4
// and groups of 16 or 32 slower.
constexpr int kGroupM = 4;
constexpr int kGroupMLarge = 8;      // from kGroupLargeFrom branch-row tiles up
constexpr int kGroupLargeFrom = 64;
__device__ __forceinline__ void tile_of(int L, int n_vtiles, int n_mtiles, int* vt, int* mt) {
  const int gm = n_mtiles >= kGroupLargeFrom ? kGroupMLarge : kGroupM;
  const int n_groups = (n_mtiles + gm - 1) / gm;
  const int per_full = n_vtiles * gm;
  if (L < (n_groups - 1) * per_full) {
    const int g = L / per_full, rem = L % per_full;
    *vt = rem / gm;
    *mt = g * gm + rem % gm;
  } else {
    const int rem = L - (n_groups - 1) * per_full;
    const int gl = n_mtiles - (n_groups - 1) * gm;
    *vt = rem / gl;
    *mt = (n_groups - 1) * gm + rem % gl;
  }
}

template <int CPR>
__device__ __forceinline__ int dma_swz(int r) {
  return CPR == 4 ? ((r >> 2) & 3) : ((r >> 1) & 7);
}

// One global_load_lds_dwordx4: lane i copies 16 bytes from sbase + voff (its own offset) to
// LDS byte M0 + 16 i. Issued through inline asm so that the compiler does not model the LDS write: its
// conservative wait-count insertion would otherwise drain every outstanding stage before each
// LDS read. Completion is tracked explicitly with wait_vmcnt.
__device__ __forceinline__ void lds_dma16(const char* sbase, uint32_t voff, uint32_t m0v) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(voff), "s"(sbase), "{m0}"(m0v)
               : "memory");
}

// The same with the five wait states that a vector memory instruction needs after a VALU write of
// its scalar base (v_readlane of a spilled base, v_readfirstlane): the compiler places them for its
// own instructions, not in front of inline asm. For kernels with more bases than stay in scalar
// registers.
template <bool NT>
__device__ __forceinline__ void lds_dma16_wait(const char* sbase, uint32_t voff, uint32_t m0v) {
  if constexpr (NT)
    asm volatile("s_nop 4\n\tglobal_load_lds_dwordx4 %0, %1 nt" ::"v"(voff), "s"(sbase), "{m0}"(m0v)
                 : "memory");
  else
    asm volatile("s_nop 4\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(voff), "s"(sbase), "{m0}"(m0v)
                 : "memory");
}

// LDS byte address of a __shared__ location (the value M0 expects).
__device__ __forceinline__ uint32_t lds_addr(const char* p) {
  return static_cast<uint32_t>(
      reinterpret_cast<uintptr_t>((const __attribute__((address_space(3))) char*)(p)));
}

template <int N>
__device__ __forceinline__ void wait_vmcnt() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

}  // namespace
}  // namespace dbl
