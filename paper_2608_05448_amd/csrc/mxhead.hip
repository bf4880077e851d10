// Products of microscaled rows: logit[m, v] = sum_j h[m, j] w[v, j] with w in 4 bits (e2m1) and h in 4 or
// 8 (e4m3), every 32 values of a row under one power of two, on the scaled matrix instruction
// v_mfma_scale_f32_32x32x64_f8f6f4, which takes the codes and the scales as they are. The logits are
// stored, or go through the head's epilogue (tile log-mass, tile-normalised log-probabilities, LSE).
//
// As in the bf16 head the vocabulary lies along the MFMA rows and the states along its columns. Lane l of a
// 64-deep step gives row l % 32: of a 4-bit operand the 16 bytes of the 32 values from 32 (l / 32) on; of
// an 8-bit one 16 bytes from value 16 (l / 32) on and 16 from 32 + 16 (l / 32) on. In both cases its scale
// is that of the 32 values from 32 (l / 32) on (checked lane by lane against sums of random codes).
//
// What bounds it: for few states the weight's stream (17 at d = 2560 against 151,936 ids 58 us, 3.7 TB/s; one state
// 57; at d = 4096 one takes 80, 69 in 4 bits), for many
// the matrix pipes (registers alone reach 6.5-7.4 PFLOP/s in 4 bits on random codes, 4.4 with an 8-bit h, at the clock
// that the power leaves) and then the stores (2048 at d = 4096, head's form: 809-841 us; 626 in a copy without
// the stores beside 841 with them; 1.25 GB of results leave in bursts, as all workgroups end at about the same time).
// The same states in 8 bits take two instructions a product: 1626 us.
//
// The precision of the instruction, measured by planting one small product beside a large one: with both
// operands in 4 bits, and from one group of eight consecutive values to the next, a sum is as in
// binary32 (a product 2^-23 of the other still counts). Within a group of eight whose h has 8 bits,
// products are cut at 13 bits below the largest's exponent. 4-bit products need 9 of those bits, so nothing is lost there; an 8-bit code has
// exponents -9 to 8. Where the result is binary32, an 8-bit h is therefore taken in two instructions, the
// codes of magnitude 2 and more and the others (one bit of the code tells them apart): in each the products are
// multiples of 2^-3 or of 2^-10 with exponents up to 10 or 2, within the 13 bits, and nothing is
// cut. With logits rounded to bf16 one instruction does: it cuts each product at 2^-13 of the power of two of its
// group's largest, 2^-4 of the rounding of a sum of that size. A sum that is small by cancellation loses more than its
// own rounding; the caller who needs it takes fp32 logits (272 rows at d = 4096: 302 us where bf16 takes 193).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>
#include <utility>

#include "gemm.hpp"
#include "kernels.hpp"

namespace dbl {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4u __attribute__((ext_vector_type(4), aligned(4)));

// One global_load_lds_dword: lane i copies 4 bytes to LDS byte M0 + 4 i (see lds_dma16_wait).
__device__ __forceinline__ void lds_dma4_wait(const uint8_t* sbase, uint32_t voff, uint32_t m0v) {
  asm volatile("s_nop 4\n\tglobal_load_lds_dword %0, %1" ::"v"(voff), "s"(sbase), "{m0}"(m0v) : "memory");
}

// A wave-uniform address in scalar registers, whatever the compiler has kept it in.
template <class T>
__device__ __forceinline__ const T* uniform(const T* p) {
  const uint64_t u = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<int>(static_cast<uint32_t>(u)));
  const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<int>(static_cast<uint32_t>(u >> 32)));
  return reinterpret_cast<const T*>(static_cast<uint64_t>(hi) << 32 | lo);
}

// For the kernel's lambdas: one that is left a call keeps the accumulators in memory.
#define MX_INLINE __attribute__((always_inline))

// f(0), ..., f(N - 1), each with a constant.
template <class F, int... I>
__device__ __forceinline__ void constant_for_each(F&& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void constant_for(F&& f) {
  constant_for_each(static_cast<F&&>(f), std::make_integer_sequence<int, N>{});
}

enum MxEpi : int { kMxLogits32 = 0, kMxLogits16 = 1, kMxHead = 2, kMxHeadArgmax = 3 };

// WV x WM waves, each with a vocabulary tile of 128 ids and 32 NCB states. A stage is 64 KS values of every row,
// copied global -> LDS ahead into a ring of S. The scales come in groups of 512 values (G4; 16 bytes of a row at
// a time: a copy of 64 rows touches 64 cache lines, however little it takes from each) or, where 512 does not
// divide the padded row, 128 (KS = 2), into a ring of their own.
template <int HB_, int WV_, int WM_, int NCB_, int KS_, int S_, bool G4_>
struct MxCfg {
  static constexpr int HB = HB_, WV = WV_, WM = WM_, NCB = NCB_, KS = KS_, S = S_;
  static constexpr bool G4 = G4_;
  static constexpr int NW = WV * WM, kThreads = 64 * NW;
  static constexpr int NRB = 4, TM = 32 * NCB, BV = 128 * WV, BM = TM * WM;
  static constexpr int ROWA = 32 * KS, ROWB = 8 * HB * KS;    // bytes of a row and stage
  static constexpr int CPA = ROWA / 16, CPB = ROWB / 16;      // its 16-byte chunks
  static constexpr int SB = (BM + 63) / 64 * 64;              // rows of h's scales, in whole copies
  static constexpr int GB = G4 ? 16 : 4;                      // bytes of a row's scales in a group
  static constexpr int SPG = GB / (2 * KS);                   // stages of a group
  static constexpr int OFFB = BV * ROWA, STAGE = OFFB + BM * ROWB;
  static constexpr int NG = SPG == 1 ? S : 2;                 // groups in LDS
  static constexpr int GROUP = GB * (BV + SB), OFFS = S * STAGE;
  static constexpr int AI = BV * ROWA / 1024, AW = AI / NW;   // copies of a stage, and of a wave: w rows,
  static constexpr int BI = BM * ROWB / 1024, BW = (BI + NW - 1) / NW;  // h rows (some of them twice),
  static constexpr int SI = (BV + SB) / 64, SW = (SI + NW - 1) / NW;    // scales (some of them twice)
  static constexpr int PER = AW + BW;
  static constexpr int kRing = OFFS + NG * GROUP, kStore = 16384 * NW;  // the epilogue's share of the same memory
  static constexpr int kLds = kRing > kStore ? kRing : kStore;
  static constexpr int kWgPerCu = 160 * 1024 / kLds;
  static constexpr int kWavesPerEu = kWgPerCu * NW < 8 || NCB > 2 ? 1 : 2;
  static_assert(AI % NW == 0 && BI >= 1, "whole copies");
  static_assert(KS == 2 || (KS == 4 && G4), "whole groups of stages");
  static_assert(SPG == 1 || S <= SPG, "the ring's stages are of two groups at most");
  static_assert(S >= 2 && (S - 1) * PER <= 63, "ring depth and vmcnt range");
  static_assert(kLds <= 160 * 1024, "LDS per CU");
};

// Place of 16-byte chunk c of row r in a row of CP chunks in LDS, so that 16 lanes reading a chunk each of
// consecutive rows meet all 64 banks.
template <int CP>
__device__ __forceinline__ int chunk_swz(int r) {
  if constexpr (CP == 16) return r & 15;
  else return dma_swz<CP>(r);
}

// Logits of a wave's 128 ids x 32 NCB states through LDS (16 KB of this wave, 8 for bf16), so that a store
// instruction writes whole segments of a row, as in tile_logsoftmax_store_lds.
template <int NCB, bool BF16>
__device__ __forceinline__ void logits_store(f32x16 (&acc)[4][NCB], void* logits, int64_t M, int64_t V,
                                             int64_t v0w, int64_t m0w, int lane, char* xp) {
  const int half = lane >> 5, lr = lane & 31;
  const int vlim = static_cast<int>(V - v0w < kVTile ? V - v0w : kVTile);
#pragma unroll
  for (int cb = 0; cb < NCB; ++cb) {
    const int64_t rows = M - (m0w + cb * 32);
    if (rows <= 0) return;
#pragma unroll
    for (int rb = 0; rb < 4; ++rb)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x16& a = acc[rb][cb];
        if constexpr (BF16) {
          typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
          const bf16x4 o = {static_cast<__bf16>(a[4 * g]), static_cast<__bf16>(a[4 * g + 1]),
                            static_cast<__bf16>(a[4 * g + 2]), static_cast<__bf16>(a[4 * g + 3])};
          // Row lr of 256 bytes: 16-byte chunk c at c ^ (lr % 16).
          const int chunk = (rb * 4 + g) ^ (lr & 15);
          *reinterpret_cast<bf16x4*>(xp + lr * 256 + chunk * 16 + 8 * half) = o;
        } else {
          const int chunk = (rb * 8 + 2 * g + half) ^ (lr & 15);
          *reinterpret_cast<float4*>(xp + lr * 512 + chunk * 16) =
              make_float4(a[4 * g], a[4 * g + 1], a[4 * g + 2], a[4 * g + 3]);
        }
      }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    if constexpr (BF16) {
      __bf16* const base = static_cast<__bf16*>(logits) + (m0w + cb * 32) * V + v0w;
      const int c = lane & 15;
#pragma unroll
      for (int jj = 0; jj < 8; ++jj) {
        const int rr = 4 * jj + (lane >> 4);
        const uint4 o = *reinterpret_cast<const uint4*>(xp + rr * 256 + ((c ^ (rr & 15)) * 16));
        if (rr >= rows) continue;
        __bf16* q = base + rr * V + 8 * c;
        // Rows 4-byte aligned. Odd V: a value at a time, which costs (1024 states at d = 2048 146 us at V = 50,257,
        // 94 at 50,256; 272 states 56 and 40; 17 states 16 and 17).
        if (V % 2 == 0 && 8 * c + 7 < vlim) {
          __builtin_nontemporal_store(u32x4u{o.x, o.y, o.z, o.w}, reinterpret_cast<u32x4u*>(q));
        } else {
          const uint32_t w[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (8 * c + e < vlim)
              reinterpret_cast<uint16_t*>(q)[e] = static_cast<uint16_t>(w[e / 2] >> (16 * (e & 1)));
        }
      }
    } else {
      float* const base = static_cast<float*>(logits) + (m0w + cb * 32) * V + v0w;
#pragma unroll
      for (int jj = 0; jj < 16; ++jj) {
        const int rr = 2 * jj + half;
        const float4 o = *reinterpret_cast<const float4*>(xp + rr * 512 + ((lr ^ (rr & 15)) * 16));
        if (rr >= rows) continue;
        float* q = base + rr * V + 4 * lr;
        if (4 * lr + 3 < vlim) {
          __builtin_nontemporal_store(f32x4u{o.x, o.y, o.z, o.w}, reinterpret_cast<f32x4u*>(q));
        } else {
          if (4 * lr + 0 < vlim) q[0] = o.x;
          if (4 * lr + 1 < vlim) q[1] = o.y;
          if (4 * lr + 2 < vlim) q[2] = o.z;
        }
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  }
}

// 0xff in the bytes of 8-bit codes of magnitude 2 and more (0x40 .. 0x7f without the sign).
__device__ __forceinline__ uint32_t large_codes(uint32_t x) {
  const uint32_t one = (x >> 6) & 0x01010101u;
  return (one << 8) - one;
}

template <class C, int EPI>
__global__ __launch_bounds__(C::kThreads, C::kWavesPerEu) void mx_product_kernel(
    const uint8_t* __restrict__ h, const uint8_t* __restrict__ hs, const uint8_t* __restrict__ w,
    const uint8_t* __restrict__ ws, void* __restrict__ logits, float* __restrict__ tls,
    float* __restrict__ lmass, uint64_t* __restrict__ amax, int64_t M, int64_t V, int dp, int n_mtiles) {
  constexpr int NRB = C::NRB, NCB = C::NCB, HB = C::HB;
  // The weight's copies are non-temporal where no other workgroup reads them at about the same time.
  constexpr bool kStream = C::NCB * C::WM <= 2;
  constexpr bool kSplit = HB == 8 && EPI != kMxLogits16;
  __shared__ __attribute__((aligned(1024))) char smem[C::kLds];
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave % C::WM, wv = wave / C::WM;
  int vt, mt;
  tile_of(xcd_remap(blockIdx.x, gridDim.x), gridDim.x / n_mtiles, n_mtiles, &vt, &mt);
  const int64_t v0 = static_cast<int64_t>(vt) * C::BV;
  const int64_t m0 = static_cast<int64_t>(mt) * C::BM;
  const int64_t nv = V - v0, nm = M - m0;  // rows there are from here on; past them the last one repeats

  // Copies. The 16-byte chunks of a row lie in another order by row.
  const int64_t pa = dp / 2, pb = dp / 8 * HB, ps = dp / 32;  // bytes of a row
  const char* const srcA = uniform(reinterpret_cast<const char*>(w) + v0 * pa);
  const char* const srcB = uniform(reinterpret_cast<const char*>(h) + m0 * pb);
  const uint8_t* const srcS[2] = {uniform(ws + v0 * ps), uniform(hs + m0 * ps)};
  constexpr int CPA = C::CPA, CPB = C::CPB, RPA = 64 / CPA, RPB = 64 / CPB;  // chunks of a row, rows of a copy
  uint32_t offA[C::AW], offB[C::BW], offS[C::SW];
#pragma unroll
  for (int i = 0; i < C::AW; ++i) {
    const int r = (wave * C::AW + i) * RPA + lane / CPA;
    offA[i] = static_cast<uint32_t>((r < nv ? r : nv - 1) * pa + ((lane % CPA) ^ chunk_swz<CPA>(r)) * 16);
  }
#pragma unroll
  for (int i = 0; i < C::BW; ++i) {
    const int r = (wave + i * C::NW) % C::BI * RPB + lane / CPB;
    offB[i] = static_cast<uint32_t>((r < nm ? r : nm - 1) * pb + ((lane % CPB) ^ chunk_swz<CPB>(r)) * 16);
  }
#pragma unroll
  for (int i = 0; i < C::SW; ++i) {
    const int g = (wave + i * C::NW) % C::SI;  // 64 rows: of w, then of h
    const int64_t r = 64 * (g < C::BV / 64 ? g : g - C::BV / 64) + lane;
    const int64_t n = g < C::BV / 64 ? nv : nm;
    offS[i] = static_cast<uint32_t>((r < n ? r : n - 1) * ps);
  }
  const uint32_t lds0 = lds_addr(smem);
  // Copy i of the kCopies that a wave makes for a stage, of stage s to ring slot `slot`: the scales, if a group
  // begins with it, so that waiting for all but later stages' data waits for these, too; w; h. The stages of a copy
  // come in order, and its offset moves on from one to the next.
  constexpr int kCopies = C::SW + C::AW + C::BW;
  auto copy = [&](auto i_, int s, int slot, auto group) MX_INLINE {
    constexpr int i = decltype(i_)::value;
    const uint32_t to = lds0 + slot * C::STAGE;
    if constexpr (i < C::SW) {
      if (group) {
        const int at = (wave + i * C::NW) % C::SI;
        const uint8_t* const from = uniform(at < C::BV / 64 ? srcS[0] : srcS[1]);
        const uint32_t into = lds0 + C::OFFS + s / C::SPG % C::NG * C::GROUP + at * 64 * C::GB;
        if constexpr (C::G4)
          lds_dma16_wait<false>(reinterpret_cast<const char*>(from), offS[i], into);
        else
          lds_dma4_wait(from, offS[i], into);
        offS[i] += C::GB;
      }
    } else if constexpr (i < C::SW + C::AW) {
      constexpr int a = i - C::SW;
      lds_dma16_wait<kStream>(srcA, offA[a], to + (wave * C::AW + a) * 1024);
      offA[a] += C::ROWA;
    } else {
      constexpr int b = i - C::SW - C::AW;
      lds_dma16_wait<false>(srcB, offB[b], to + C::OFFB + (wave + b * C::NW) % C::BI * 1024);
      offB[b] += C::ROWB;
    }
  };

  f32x16 acc[NRB][NCB];
#pragma unroll
  for (int rb = 0; rb < NRB; ++rb)
#pragma unroll
    for (int cb = 0; cb < NCB; ++cb)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[rb][cb][r] = 0.0f;

  const int lr = lane & 31, half = lane >> 5;
  const int ta = chunk_swz<CPA>(lr), tb = chunk_swz<CPB>(lr);  // the same for every block of 32 rows
  const int a_base = (wv * kVTile + lr) * C::ROWA;
  const int b_base = C::OFFB + (wm * C::TM + lr) * C::ROWB;
  const int sa_base = (wv * kVTile + lr) * C::GB;
  const int sb_base = (C::BV + wm * C::TM + lr) * C::GB;
  const int nk = dp / (64 * C::KS);
  // Fragments of two 64-deep steps, the one that is computed and the next one's, by its parity.
  i32x8 af[2][NRB], bf[2][NCB];
  // Read i of the kReads of a step's fragments, in the order in which the products need them.
  constexpr int kReads = NRB + NCB;
  auto read = [&](auto i_, const char* base, auto ks_) MX_INLINE {
    constexpr int i = decltype(i_)::value, ks = decltype(ks_)::value, p = ks & 1;
    if constexpr (i >= 1 && i <= NRB) {
      constexpr int rb = i - 1;
      const i32x4 x = *reinterpret_cast<const i32x4*>(base + a_base + rb * 32 * C::ROWA + (((2 * ks + half) ^ ta) * 16));
      af[p][rb] = __builtin_shufflevector(x, i32x4{}, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
      constexpr int cb = i == 0 ? 0 : i - NRB;
      const char* row = base + b_base + cb * 32 * C::ROWB;
      if constexpr (HB == 4) {
        const i32x4 x = *reinterpret_cast<const i32x4*>(row + (((2 * ks + half) ^ tb) * 16));
        bf[p][cb] = __builtin_shufflevector(x, i32x4{}, 0, 1, 2, 3, 4, 5, 6, 7);
      } else {
        const i32x4 x = *reinterpret_cast<const i32x4*>(row + (((4 * ks + half) ^ tb) * 16));
        const i32x4 y = *reinterpret_cast<const i32x4*>(row + (((4 * ks + 2 + half) ^ tb) * 16));
        bf[p][cb] = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
      }
    }
  };
  // A stage's scales: words of two steps each, of which bytes 0 and 2 are this lane's after the shift.
  constexpr int SWD = C::KS / 2;
  struct Scales {
    int a[SWD][NRB], b[SWD][NCB];
  };
  Scales sc, next;
  auto load_scales = [&](int s, Scales& to) MX_INLINE {
    const char* base = smem + C::OFFS + s / C::SPG % C::NG * C::GROUP + s % C::SPG * (2 * C::KS);
#pragma unroll
    for (int rb = 0; rb < NRB; ++rb)
#pragma unroll
      for (int i = 0; i < SWD; ++i)
        to.a[i][rb] = *reinterpret_cast<const int*>(base + sa_base + rb * 32 * C::GB + 4 * i);
#pragma unroll
    for (int cb = 0; cb < NCB; ++cb)
#pragma unroll
      for (int i = 0; i < SWD; ++i)
        to.b[i][cb] = *reinterpret_cast<const int*>(base + sb_base + cb * 32 * C::GB + 4 * i);
  };
  auto take_scales = [&](const Scales& from) MX_INLINE {
#pragma unroll
    for (int i = 0; i < SWD; ++i) {
#pragma unroll
      for (int rb = 0; rb < NRB; ++rb) sc.a[i][rb] = from.a[i][rb] >> (8 * half);
#pragma unroll
      for (int cb = 0; cb < NCB; ++cb) sc.b[i][cb] = from.b[i][cb] >> (8 * half);
    }
  };
  // A step, and other(n) after its product n. A product takes the matrix pipe for 32 cycles (64 with an 8-bit h), and
  // the wave issues in order: what it does besides (LDS reads, copies) goes a little at a time between products, since
  // a burst of it leaves the pipe empty, with one wave to a SIMD (2048 rows at d = 4096 against 151,936 ids: 985 us with
  // it in bursts of four products, 841 so).
  constexpr int kProducts = NRB * NCB;
  auto step = [&](auto ks_, auto other) MX_INLINE {
    constexpr int ks = decltype(ks_)::value, p = ks & 1, fmt = HB == 4 ? 4 : 0, i = ks / 2, op = 2 * (ks & 1);
    i32x8 large, small;
    constant_for<kProducts>([&](auto n_) MX_INLINE {
      constexpr int n = decltype(n_)::value, cb = n / NRB, rb = n % NRB;
      if constexpr (kSplit) {
        if constexpr (rb == 0) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const uint32_t m = large_codes(static_cast<uint32_t>(bf[p][cb][e]));
            large[e] = bf[p][cb][e] & static_cast<int>(m);
            small[e] = bf[p][cb][e] & static_cast<int>(~m);
          }
        }
        acc[rb][cb] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
            af[p][rb], small, acc[rb][cb], 4, fmt, op, sc.a[i][rb], op, sc.b[i][cb]);
        acc[rb][cb] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
            af[p][rb], large, acc[rb][cb], 4, fmt, op, sc.a[i][rb], op, sc.b[i][cb]);
      } else {
        acc[rb][cb] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
            af[p][rb], bf[p][cb], acc[rb][cb], 4, fmt, op, sc.a[i][rb], op, sc.b[i][cb]);
      }
      __builtin_amdgcn_sched_barrier(0);
      other(n_);
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  // f(i) for those of `count` things that come after product n, if they are spread over the first `over` products.
  auto spread = [&](auto n_, auto count_, auto over_, auto f) MX_INLINE {
    constexpr int n = decltype(n_)::value, count = decltype(count_)::value, over = decltype(over_)::value;
    constant_for<count>([&](auto i_) MX_INLINE {
      if constexpr (decltype(i_)::value * over / count == n) f(i_);
    });
  };
  // The next step's fragments: all under way before the last products, which cover their latency.
  constexpr std::integral_constant<int, kReads> reads{};
  constexpr std::integral_constant<int, (kProducts * 3 + 3) / 4> early{};
  // The copies of a stage go into kCopySteps steps: the last one of stage s - S, whose slot they take, and the
  // first ones of the stage after that, as long as a step is left before they are waited for.
  constexpr int kCopySteps = C::S > 2 ? C::KS : C::KS - 1;
  auto copies = [&](auto n_, auto step_, int s, int slot, auto group) MX_INLINE {
    constexpr int from = (decltype(step_)::value * kCopies + kCopySteps - 1) / kCopySteps;
    constexpr int to = ((decltype(step_)::value + 1) * kCopies + kCopySteps - 1) / kCopySteps;
    if constexpr (decltype(step_)::value < kCopySteps && to > from)
      spread(n_, std::integral_constant<int, to - from>{}, std::integral_constant<int, kProducts>{},
             [&](auto i_) MX_INLINE { copy(std::integral_constant<int, from + decltype(i_)::value>{}, s, slot, group); });
  };

  // Prologue: the ring in flight, of the last stage in it what the last step of the one before the first would start.
  constexpr int kFirst = (kCopies + kCopySteps - 1) / kCopySteps;  // copies of a stage in its first step
#pragma unroll
  for (int j = 0; j < C::S; ++j)
    if (j < nk)
      constant_for<kCopies>([&](auto i_) MX_INLINE {
        if (j + 1 < C::S || decltype(i_)::value < kFirst) copy(i_, j, j, j % C::SPG == 0);
      });
  if (nk >= C::S)
    wait_vmcnt<(C::S - 2) * C::PER + (kFirst > C::SW ? kFirst - C::SW : 0)>();
  else
    wait_vmcnt<0>();
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  constant_for<kReads>([&](auto i_) MX_INLINE { read(i_, smem, std::integral_constant<int, 0>{}); });
  load_scales(0, next);
  // A wave reads its fragments a step before it needs them. So before the last step of a stage every wave has all of
  // it in registers, and the barrier that lies there (each wave has waited for its own copies of the next
  // stage) both opens the next stage and frees this one's slot, for the copies of stage kt + S.
  // late: the rest of the copies of stage kt + S - 1; more: a stage follows; begin: stage kt + S is there; now, then:
  // whether a group of scales begins with those two. Constants in the main part of the loop: around a branch the
  // compiler moves the products away from what is to run beside them.
  int slot = 0;
  auto stage = [&](int kt, auto late, auto more, auto begin, auto now, auto then) MX_INLINE {
    const char* const base = smem + slot * C::STAGE;
    take_scales(next);
    const int before = slot == 0 ? C::S - 1 : slot - 1;
    constant_for<C::KS - 1>([&](auto ks_) MX_INLINE {
      constexpr int ks = decltype(ks_)::value;
      step(ks_, [&](auto n_) MX_INLINE {
        spread(n_, reads, early, [&](auto i_) MX_INLINE { read(i_, base, std::integral_constant<int, ks + 1>{}); });
        if (late) copies(n_, std::integral_constant<int, ks + 1>{}, kt + C::S - 1, before, now);
      });
    });
    const int after = slot + 1 == C::S ? 0 : slot + 1;
    if (more) {
      // Stages kt + 2 .. kt + S - 1 may still be in flight; near the end all have to be in.
      if (begin || C::S == 2)
        wait_vmcnt<(C::S - 2) * C::PER>();
      else
        wait_vmcnt<0>();
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
    }
    step(std::integral_constant<int, C::KS - 1>{}, [&](auto n_) MX_INLINE {
      if (more) {
        spread(n_, reads, early,
               [&](auto i_) MX_INLINE { read(i_, smem + after * C::STAGE, std::integral_constant<int, 0>{}); });
        if constexpr (decltype(n_)::value == 0) load_scales(kt + 1, next);
      }
      if (begin) copies(n_, std::integral_constant<int, 0>{}, kt + C::S, slot, then);
    });
    slot = after;
  };
  const std::true_type yes{};
  const std::false_type no{};
  int kt = 0;
  for (; kt + C::S + C::SPG - 1 < nk; kt += C::SPG)
    constant_for<C::SPG>([&](auto g_) MX_INLINE {
      constexpr int g = decltype(g_)::value;
      stage(kt + g, yes, yes, yes, std::integral_constant<bool, (g + C::S - 1) % C::SPG == 0>{},
            std::integral_constant<bool, (g + C::S) % C::SPG == 0>{});
    });
  for (; kt + C::S < nk; ++kt) stage(kt, yes, yes, yes, (kt + C::S - 1) % C::SPG == 0, (kt + C::S) % C::SPG == 0);
  if (kt + 1 < nk && kt + C::S - 1 < nk) stage(kt, yes, yes, no, (kt + C::S - 1) % C::SPG == 0, no), ++kt;
  for (; kt + 1 < nk; ++kt) stage(kt, no, yes, no, no, no);
  stage(kt, no, no, no, no, no);
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();  // the ring is free: nothing reads it, every copy has landed
  asm volatile("" ::: "memory");

  const int64_t v0w = v0 + wv * kVTile, m0w = m0 + wm * C::TM;
  if (v0w >= V || m0w >= M) return;
  char* const xp = smem + wave * 16384;
  if constexpr (EPI == kMxHead || EPI == kMxHeadArgmax)
    tile_logsoftmax_store_lds<NRB, NCB, EPI == kMxHeadArgmax, true>(
        acc, tls, lmass, amax, M, V, static_cast<int>((V + kVTile - 1) / kVTile), v0w, m0w, lane, xp);
  else
    logits_store<NCB, EPI == kMxLogits16>(acc, logits, M, V, v0w, m0w, lane, xp);
}

template <class C, int EPI>
hipError_t launch_as(const MxProductArgs& a, hipStream_t stream) {
  const int64_t dm = (a.M + C::BM - 1) / C::BM;
  const int64_t nwg = ((a.V + C::BV - 1) / C::BV) * dm;
  if (nwg > kMaxThreads / C::kThreads || nwg > 0x7fffffff) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL((mx_product_kernel<C, EPI>), dim3(static_cast<unsigned>(nwg)), dim3(C::kThreads), 0,
                     stream, static_cast<const uint8_t*>(a.h), a.hs, static_cast<const uint8_t*>(a.w), a.ws,
                     a.logits, a.tls, a.lmass, a.amax_keys, a.M, a.V, a.dp, static_cast<int>(dm));
  return hipGetLastError();
}

// Tiles, us by (ids x states, values of a stage, waves a CU) at V = 151,936: 17 states of 8 bits at d = 2560 60 with
// 256 x 64, 256 deep, 61 with 256 x 32, 256 deep, 73 with 256 x 32, 128 deep, 94 with 512 x 32. 272 states of 8 bits
// at d = 4096, bf16 logits: 193 with 256 x 128, 128 deep, two workgroups to a CU, 220 with one of three stages, 214
// with 256 x 192, 256 with 256 x 256. 2048 states of 4 bits at d = 4096, the head's form: 841 with 256 x 256,
// 256 deep (128 x 128 a wave), 862 with 128 deep, 857 with eight waves of 128 x 64, 1004 with 256 x 128, two
// workgroups to a CU. Of an 8-bit h a product takes twice as long, and the second workgroup, which hides the
// first one's stores, is worth more than the larger tile.
// The rule for 4 bits (below) has its 0.84 from d = 4096. Both sides there and at smaller d, larger tile and smaller (us,
// V = 151,936, states x d, bf16 logits): 2048 x 4096 643, 855; 512 x 4096 182, 236; 2048 x 2048 383, 463; 2048 x 1024
// 232, 240; 512 x 1024 65, 68; 2048 x 512 171, 161; 512 x 512 48, 47; the head's form 2048 x 4096 781, 956; x 2048 521,
// 566; x 1024 355, 341; x 512 294, 269. So up to d = 1024 the stores count and the smaller tile, not taken there, is as
// good or up to 10% better, and where one round of either does, better by more (272 states at d = 1024 against 20,000
// ids 12.6 where the larger takes 18.2). Rows that 512 does not divide have the smaller tile only, with a scale
// copy for every 128 values (d = 896 and 1024, 8 bits: 272 states 65 and 58, 2048 states 328 and 304).
template <int HB, int EPI>
hipError_t launch_bits(const MxProductArgs& a, hipStream_t stream) {
  if (a.dp % 512 != 0) {
    if (a.M <= 64) return launch_as<MxCfg<HB, 2, 2, 1, 2, 3, false>, EPI>(a, stream);
    return launch_as<MxCfg<HB, 2, 2, 2, 2, 3, false>, EPI>(a, stream);
  }
  if (a.M <= 64) return launch_as<MxCfg<HB, 2, 2, 1, 4, 2, true>, EPI>(a, stream);
  if constexpr (HB == 4) {
    // In rounds of the GPU, one workgroup to a CU or two: a round of the larger tiles takes 0.84 of one of the others
    // at d = 4096.
    const int64_t vt = (a.V + 255) / 256;
    const int64_t large = (vt * ((a.M + 255) / 256) + 255) / 256, small = (vt * ((a.M + 127) / 128) + 511) / 512;
    if (a.M > 128 && 84 * large <= 100 * small) return launch_as<MxCfg<HB, 2, 2, 4, 4, 2, true>, EPI>(a, stream);
  }
  return launch_as<MxCfg<HB, 2, 2, 2, 2, 2, true>, EPI>(a, stream);
}

template <int EPI>
hipError_t launch_epi(const MxProductArgs& a, hipStream_t stream) {
  return a.bits == 4 ? launch_bits<4, EPI>(a, stream) : launch_bits<8, EPI>(a, stream);
}

}  // namespace

hipError_t launch_mx_product(const MxProductArgs& a, hipStream_t stream) {
  if (a.logits) return a.bf16 ? launch_epi<kMxLogits16>(a, stream) : launch_epi<kMxLogits32>(a, stream);
  if (a.argmax)
    if (const hipError_t e = launch_argmax_clear(a.amax_keys, a.M, stream); e != hipSuccess) return e;
  const hipError_t e = a.argmax ? launch_epi<kMxHeadArgmax>(a, stream) : launch_epi<kMxHead>(a, stream);
  if (e != hipSuccess) return e;
  return launch_lse(a.lmass, a.lse, a.argmax ? a.amax_keys : nullptr, a.argmax, a.M,
                    static_cast<int>((a.V + kVTile - 1) / kVTile), stream);
}

}  // namespace dbl
