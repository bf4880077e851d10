// One token per row of logits by temperature, top-k, top-p and min-p, from a given random word.
//
// The distribution is the target transform's (target.hip): s = fl32(logit / T), integer weights
// w = floor(detexp32(fl32(s - max)) 2^40), top-k with its ties, then top-p by decreasing s and
// increasing id; and then min-p. The token is the inverse CDF of the word over the kept weights in id
// order. Everything that decides is an integer, so the token depends neither on how a row is
// split nor on the other rows.
//
// What bounds it is reading the logits and, where masses are needed, the exponentials. A row lies in segments of
// kDrawSeg ids, and about 2048 workgroups share the segments of all rows, so that few rows still use the whole
// GPU. Workgroups of a row meet at the ends of launches only: an agent-wide fence per workgroup, for
// a counter that lets the last one go on, writes back and empties an L2 each time (1024 rows of 50,257 ids
// took 2,080 us that way, 82 now). The launches after the first read the logits from the caches:
//   top     maximum of each part of a row, and of each 128 ids
//   bins    without filters the sum of each segment's weights; under top-p alone (or with min-p), masses in
//           bins of max - s; under a top-k past the number of 128s, counts
//   find    (only where there are filters) a workgroup per row finds the cut's bound, as follows
//   cut     (only where there are filters) lists the ids that the cut goes through, and sums by segment what is
//           surely kept. Top-k: the k-th largest of the maxima of 128 ids is a bound from below for the k-th
//           largest id, so that what reaches it holds all that is kept and nothing else is looked at: about k ids for
//           small k and large logits at random ids, more the nearer k is to the number of groups (k = 1000 of 1187:
//           2200, from 1150 on past the list) or the more large logits share groups (ids in the order of their
//           frequency: 2300 at k = 50, 4600 at 100). Otherwise: the bin that the cut falls into is listed, what is
//           above it summed
//   finish  a workgroup per row: sorts the list, finds the exact cut and draws. Rows whose list is
//           longer than kListMost, or with a top-k past kListMost / 2 and top-p at once, are selected by
//           radix over their order-preserving keys here, about ten reads of the row by that one workgroup
// Long lists are not rare: a bf16 number in the tail of a nucleus may have more than kListMost ids (V = 151,936, of
// rows like Zipf's law 11% at a temperature of 0.7 and 17% at 1 under top_p = 0.95), and k and the order of the ids
// make them as above. Such a row costs 0.5 to 0.6 ms where others take 31 us alone, and 272 rows with some of
// them 1.0 ms (bf16 nucleus; fp32 167 us) to 1.15 (top-k 100 to 1187 of ids in order; 101 us for 50 of spread ids).
// 272 rows of 151,936 ids under parameters of their own 133 us (top 38, bins 28, find 9, cut 31, finish 29; reading them
// once takes 24.5), one under a nucleus 31. A weight costs 33 vector operations, which bounds bins and cut.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "contract.hpp"
#include "kernels.hpp"
#include "wave.hpp"

namespace dbl {
namespace {

constexpr int kT = 512;        // threads of a workgroup
constexpr int kW = kT / 64;
// Bins of max - s, 144 to a unit. What is in the last one, from 28.4 on, weighs 0 (weights end at 40 ln 2 = 27.73).
constexpr int kBins = kDrawBins;
constexpr float kPerBin = 144.0f;
__device__ __forceinline__ int bin_of(float distance) {
  return static_cast<int>(fminf(distance * kPerBin, static_cast<float>(kBins - 1)));  // NaN: the last one
}
constexpr int kListMost = kDrawList;
constexpr int kRun = kBins / kT;  // bins of a thread where they are summed up
static_assert(kRun % 4 == 0, "16-byte loads of a thread's counts");
constexpr int kMostSegments = ((1 << 24) + 6) / kDrawSeg + 1;  // of a row
constexpr int kGroups = kDrawSeg / 128;  // maxima of a segment
constexpr int kKeyed = 64;               // segments up to which the maxima of a row are looked at for top-k

// kList: the list takes all that may be kept. kSums: the list takes bin cut_bin (by != 0), the bins before it are
// summed by segment. by: 0, nothing is cut inside that bin; 1, by rank: `need` is the last one's, from 1 within
// the bin; 2, by mass: an id is kept while less than `need` is kept before it in the bin.
enum RowMode : uint32_t { kNothing = 0, kList = 1, kSums = 2, kRadix = 3 };
using RowState = DrawState;
using Layout = DrawLayout;
constexpr int kListFew = kT;  // up to here keys are sorted by counting (see sort_lds)

__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return __uint_as_float((k & 0x80000000u) ? (k & 0x7fffffffu) : ~k);
}

// A row of logits in 16-byte words from the aligned address at or below its start: word i holds ids
// i VEC - shift + e.
template <class T>
struct Row {
  static constexpr int VEC = 16 / sizeof(T);
  const T* base;
  const T* end;  // of the tensor
  int64_t V;
  int shift;
  __device__ Row(const DrawArgs& a, int64_t row) : V(a.V) {
    const T* p = static_cast<const T*>(a.logits) + row * a.V;
    shift = static_cast<int>(reinterpret_cast<uintptr_t>(p) % 16 / sizeof(T));
    base = p - shift;
    end = static_cast<const T*>(a.logits) + a.N * a.V;
  }
  static __device__ __forceinline__ void unpack(const uint4 q, float (&x)[VEC]) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      if constexpr (sizeof(T) == 4)
        x[e] = __uint_as_float(w[e]);
      else
        x[e] = __uint_as_float((e & 1) ? (w[e / 2] & 0xffff0000u) : (w[e / 2] << 16));
    }
  }
  // The values of word i, -inf outside the row.
  __device__ __forceinline__ void load(int64_t i, float (&x)[VEC]) const {
    const int64_t v0 = i * VEC - shift;
    const T* p = base + i * VEC;
    if (v0 < V && p + VEC <= end) {
      unpack(*reinterpret_cast<const uint4*>(p), x);
      if (v0 < 0 || v0 + VEC > V) {
#pragma unroll
        for (int e = 0; e < VEC; ++e)
          if (v0 + e < 0 || v0 + e >= V) x[e] = -INFINITY;
      }
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        x[e] = v0 + e >= 0 && v0 + e < V ? static_cast<float>(p[e]) : -INFINITY;
    }
  }
};

struct Params {
  float T, top_p;
  int64_t k;        // 0: off
  uint64_t min_w;   // smallest weight that is kept (0: off)
  float min_p;
  bool ok;
  __device__ Params(const DrawArgs& a, int64_t row) {
    T = a.temperatures ? a.temperatures[row] : a.temperature;
    top_p = a.top_ps ? a.top_ps[row] : a.top_p;
    min_p = a.min_ps ? a.min_ps[row] : a.min_p;
    k = a.top_ks ? a.top_ks[row] : a.top_k;
    ok = T >= 0.0f && T < INFINITY && top_p > 0.0f && top_p <= 1.0f && min_p >= 0.0f && min_p <= 1.0f && k >= 0;
    if (k >= a.V) k = 0;
    // w >= min_p 2^40, which is exact in binary64, for whole numbers w.
    min_w = ok ? static_cast<uint64_t>(ceil(static_cast<double>(min_p) * 0x1p40)) : 0;
  }
  __device__ bool filtered() const { return k > 0 || top_p < 1.0f || min_w > 0; }
  // Whether the k-th largest of the maxima of 128 ids bounds the k-th largest id.
  __device__ bool keyed(int64_t V, int G) const { return k > 0 && k <= V / 128 && G <= kKeyed; }
  __device__ bool counts(int64_t V, int G) const { return k > 0 && !keyed(V, G); }
  __device__ bool masses() const { return k == 0 && top_p < 1.0f; }
};

struct Shared {
  uint64_t red[kW + 1];
  uint64_t out[4];
  uint32_t flag;
};

// Inclusive scan over a wave's 64 lanes by an operation with identity 0, on data-parallel primitives (a few cycles
// a step where a shuffle through LDS takes its latency): within rows of 16 lanes, then across them. Lane 63 has
// the whole.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint64_t dpp_u64(uint64_t v) {
  const int lo = __builtin_amdgcn_update_dpp(0, static_cast<int>(static_cast<uint32_t>(v)), CTRL, ROWS, 0xf, true);
  const int hi = __builtin_amdgcn_update_dpp(0, static_cast<int>(static_cast<uint32_t>(v >> 32)), CTRL, ROWS, 0xf, true);
  return static_cast<uint64_t>(static_cast<uint32_t>(hi)) << 32 | static_cast<uint32_t>(lo);
}
template <class Op>
__device__ __forceinline__ uint64_t wave_scan(uint64_t v, Op op) {
  v = op(v, dpp_u64<0x111, 0xf>(v));  // from the lane 1, 2, 4, 8 before in the row
  v = op(v, dpp_u64<0x112, 0xf>(v));
  v = op(v, dpp_u64<0x114, 0xf>(v));
  v = op(v, dpp_u64<0x118, 0xf>(v));
  v = op(v, dpp_u64<0x142, 0xa>(v));  // from lane 15 of the row before, to rows 1 and 3
  v = op(v, dpp_u64<0x143, 0xc>(v));  // from lane 31, to rows 2 and 3
  return v;
}
struct Add {
  __device__ __forceinline__ uint64_t operator()(uint64_t x, uint64_t y) const { return x + y; }
};
struct Max {
  __device__ __forceinline__ uint64_t operator()(uint64_t x, uint64_t y) const { return x > y ? x : y; }
};
template <class Op>
__device__ __forceinline__ uint64_t wave_all(uint64_t v, Op op) {
  return lane_u64(wave_scan(v, op), 63);
}
template <class Op>
__device__ __forceinline__ uint64_t block_reduce(uint64_t v, Shared& sh, Op op) {
  v = wave_scan(v, op);
  __syncthreads();
  if (lane_id() == 63) sh.red[threadIdx.x >> 6] = v;
  __syncthreads();
  uint64_t r = sh.red[0];
#pragma unroll
  for (int w = 1; w < kW; ++w) r = op(r, sh.red[w]);
  return r;
}
__device__ __forceinline__ uint64_t block_sum(uint64_t v, Shared& sh) { return block_reduce(v, sh, Add{}); }
__device__ __forceinline__ uint64_t block_max(uint64_t v, Shared& sh) { return block_reduce(v, sh, Max{}); }
__device__ __forceinline__ uint64_t block_min(uint64_t v, Shared& sh) { return ~block_max(~v, sh); }
// Sum over the threads up to and including this one; *all: of the workgroup.
__device__ __forceinline__ uint64_t block_scan(uint64_t v, Shared& sh, uint64_t* all) {
  uint64_t s = wave_scan(v, Add{});
  __syncthreads();
  if (lane_id() == 63) sh.red[threadIdx.x >> 6] = s;
  __syncthreads();
  uint64_t t = 0;
#pragma unroll
  for (int w = 0; w < kW; ++w) {
    if (w < static_cast<int>(threadIdx.x >> 6)) s += sh.red[w];
    t += sh.red[w];
  }
  *all = t;
  return s;
}

// The distribution of a row: weight of a logit, its key, and what is kept.
struct Dist {
  float m;
  Quotient q;
  bool fast;
  __device__ Dist(float T, float m_) : m(m_), q(T), fast(q.short_form && fabsf(m_) <= 0x1p100f) {}
  // fl32(x / T).
  __device__ __forceinline__ float s(float x) const {
    const float a = fabsf(x);
    float r = q.quick(x);
    if (!(q.short_form && a <= 0x1p100f && (a >= 0x1p-100f || a == 0.0f)))
      r = a == INFINITY ? x : __fdiv_rn(x, q.T);
    return r;
  }
  __device__ __forceinline__ uint64_t weight(float sv) const { return quant_detexp32(__fsub_rn(sv, m)); }
  // fl32(s - max) of logit x <= max, FAST where `fast`: the short division's result for every x that
  // matters. Tiny quotients may be off in their last place, which a difference from the maximum, or the
  // exponential of one, does not show; huge ones and minus infinity may come out as NaN, which weighs 0
  // and lies in the last bin, as they do.
  template <bool FAST>
  __device__ __forceinline__ float below(float x) const {
    return __fsub_rn(FAST ? q.quick(x) : s(x), m);
  }
  // The weight of fl32(s - max) as a binary32 number (24 bits hold it exactly, as they hold the
  // exponential): n is rounded by an addition whose low bits then are n + 40, to be added to p's exponent.
  __device__ __forceinline__ float weight_f(float c) const {
#pragma clang fp contract(off)
    c = fmaxf(c, -100.0f);
    constexpr float kMagic = 0x1.8p23f + 40.0f;
    const float t = __fadd_rn(__fmul_rn(c, 0x1.715476p+0f), kMagic);
    const float n = __fsub_rn(t, kMagic);
    const float r = __fsub_rn(__fsub_rn(c, __fmul_rn(n, 0x1.62e4p-1f)), __fmul_rn(n, 0x1.7f7d1cp-20f));
    float p = static_cast<float>(1.0 / 5040.0);
    p = __fadd_rn(__fmul_rn(p, r), static_cast<float>(1.0 / 720.0));
    p = __fadd_rn(__fmul_rn(p, r), static_cast<float>(1.0 / 120.0));
    p = __fadd_rn(__fmul_rn(p, r), static_cast<float>(1.0 / 24.0));
    p = __fadd_rn(__fmul_rn(p, r), static_cast<float>(1.0 / 6.0));
    p = __fadd_rn(__fmul_rn(p, r), 0.5f);
    p = __fadd_rn(__fmul_rn(p, r), 1.0f);
    p = __fadd_rn(__fmul_rn(p, r), 1.0f);
    return floorf(__uint_as_float((__float_as_uint(t) << 23) + __float_as_uint(p)));
  }
};
struct Keep {
  uint32_t kth = 0;      // keys at or above
  uint32_t cut = 0;      // keys above, and those equal with ids up to last
  uint32_t last = 0xffffffffu;
  uint64_t min_w = 0;
  __device__ __forceinline__ uint64_t weight(const Dist& d, float sv, uint32_t id) const {
    const uint32_t k = order_key(sv);
    const uint64_t w = d.weight(sv);
    return k >= kth && (k > cut || (k == cut && id <= last)) && w >= min_w ? w : 0;
  }
};

__device__ __forceinline__ void give(const DrawArgs& a, int64_t row, int64_t id, uint64_t w, uint64_t total) {
  a.token[row] = static_cast<int32_t>(id);
  const double W = static_cast<double>(w), S = static_cast<double>(total);
  a.logprob[row] = static_cast<float>(2 * w > total ? log1p(-static_cast<double>(total - w) / S) : log(W / S));
}
__device__ __forceinline__ void give_none(const DrawArgs& a, int64_t row) {
  a.token[row] = -1;
  a.logprob[row] = NAN;
}

// Draws from the sums of a row's segments, seg[0 .. G) in LDS: the segment that holds the threshold, and in it the id.
// Every thread of the workgroup calls it.
template <class T>
__device__ void draw_from_segments(const DrawArgs& a, int64_t row, uint32_t word, const uint64_t* seg, int G,
                                   const Dist& d, const Keep& keep, Shared& sh) {
  uint64_t mine = 0, total;
  const int per = (G + kT - 1) / kT, g0 = min(G, static_cast<int>(threadIdx.x) * per), g1 = min(G, g0 + per);
  for (int g = g0; g < g1; ++g) mine += seg[g];
  const uint64_t incl = block_scan(mine, sh, &total);
  if (total == 0) {  // unreachable: the maximum weighs 2^40 and is kept
    if (threadIdx.x == 0) give_none(a, row);
    return;
  }
  const uint64_t at = icdf_threshold(word, total);
  if (incl - mine <= at && at < incl) {
    uint64_t c = incl - mine;
    for (int g = g0; g < g1; ++g) {
      if (at < c + seg[g]) {
        sh.out[0] = static_cast<uint64_t>(g);
        sh.out[1] = c;
        break;
      }
      c += seg[g];
    }
  }
  __syncthreads();
  const int64_t g = static_cast<int64_t>(sh.out[0]);
  const uint64_t before = sh.out[1];
  constexpr int VEC = Row<T>::VEC, PER = kDrawSeg / VEC / kT;
  const Row<T> r(a, row);
  const int64_t i0 = g * (kDrawSeg / VEC) + static_cast<int64_t>(threadIdx.x) * PER;
  uint64_t w[PER * VEC], sum = 0, all;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    float x[VEC];
    r.load(i0 + i, x);
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      w[i * VEC + e] = keep.weight(d, d.s(x[e]), static_cast<uint32_t>((i0 + i) * VEC - r.shift + e));
      sum += w[i * VEC + e];
    }
  }
  const uint64_t in = block_scan(sum, sh, &all) + before;
  if (in - sum <= at && at < in) {
    uint64_t c = in - sum;
#pragma unroll
    for (int i = 0; i < PER * VEC; ++i) {
      if (c <= at && at < c + w[i]) give(a, row, i0 * VEC - r.shift + i, w[i], total);
      c += w[i];
    }
  }
}

// Ascending sort of n <= kListMost different keys in LDS. Up to kListFew by counting the smaller ones (every
// thread reads the same words, without barriers), more by a bitonic network, which needs a barrier a
// stage and ~0 up to a power of two behind the keys.
__device__ void sort_lds(uint64_t* v, int n) {
  if (n <= kListFew) {
    const uint64_t x = v[min(static_cast<int>(threadIdx.x), n - 1)];
    int at = 0;
#pragma unroll 8
    for (int j = 0; j < n; ++j) at += v[j] < x ? 1 : 0;
    __syncthreads();
    if (static_cast<int>(threadIdx.x) < n) v[at] = x;
    __syncthreads();
    return;
  }
  int size = 64;
  while (size < n) size *= 2;
  for (int i = n + threadIdx.x; i < size; i += kT) v[i] = ~0ull;
  __syncthreads();
  for (int k = 2; k <= size; k *= 2)
    for (int j = k / 2; j > 0; j /= 2) {
      for (int t = threadIdx.x; t < size / 2; t += kT) {
        const int i = 2 * t - (t & (j - 1)), o = i + j;
        const uint64_t x = v[i], y = v[o];
        if ((x > y) == ((i & k) == 0)) {
          v[i] = y;
          v[o] = x;
        }
      }
      __syncthreads();
    }
}

// ---------------------------------------------------------------------------------------
// What a workgroup of the first three launches works on: segments g0 .. g1 - 1, part `part` of its row's P.
struct Part {
  int64_t row;
  int part, g0, g1;
  Layout L;
  char* ws;
  __device__ Part(const DrawArgs& a, int G, int P) : L(G) {
    row = blockIdx.x / P;
    part = blockIdx.x % P;
    g0 = static_cast<int>(static_cast<int64_t>(G) * part / P);
    g1 = static_cast<int>(static_cast<int64_t>(G) * (part + 1) / P);
    ws = a.ws + row * L.total;
  }
};

// f(id of the first value, values) of every 16-byte word of a segment that this thread has.
template <class T>
struct Segment {
  static constexpr int VEC = Row<T>::VEC, PER = kDrawSeg / VEC / kT;
  float x[PER][VEC];
  int64_t first;
  __device__ __forceinline__ Segment(const Row<T>& r, int g) {
    const int64_t at = static_cast<int64_t>(g) * kDrawSeg;
    first = at + threadIdx.x * VEC - r.shift;
    if (at >= r.shift && at + kDrawSeg - r.shift <= r.V) {  // inside the row, for the whole workgroup
      const uint4* p = reinterpret_cast<const uint4*>(r.base + at) + threadIdx.x;
      uint4 q[PER];
#pragma unroll
      for (int u = 0; u < PER; ++u) q[u] = p[kT * u];
#pragma unroll
      for (int u = 0; u < PER; ++u) Row<T>::unpack(q[u], x[u]);
    } else {
#pragma unroll
      for (int u = 0; u < PER; ++u) r.load(at / VEC + threadIdx.x + kT * u, x[u]);
    }
  }
  __device__ __forceinline__ int64_t id(int u, int e) const { return first + kT * VEC * u + e; }
};

// f(g, segment) for the segments of a part, the first of which is there.
template <class T, class F>
__device__ __forceinline__ void each_segment(const Row<T>& r, const Part& w, const Segment<T>& first, F f) {
  f(w.g0, first);
  for (int g = w.g0 + 1; g < w.g1; ++g) {
    const Segment<T> s(r, g);
    f(g, s);
  }
}

// The sums of a part's segments: each wave adds its own to LDS, and they are stored kSumBatch at a time.
constexpr int kSumBatch = 64;
struct SegmentSums {
  uint64_t* lds;   // [kSumBatch], zero
  uint64_t* sums;  // of the row
  int first;
  __device__ void clear() {
    if (threadIdx.x < kSumBatch) lds[threadIdx.x] = 0;
    __syncthreads();
  }
  __device__ __forceinline__ SegmentSums(uint64_t* l, const Part& w)
      : lds(l), sums(reinterpret_cast<uint64_t*>(w.ws + w.L.sum)), first(w.g0) {
    clear();
  }
  __device__ __forceinline__ void add(int g, double sum) {  // every thread, for g = first, first + 1, ...
    if (g - first == kSumBatch) {
      store(kSumBatch);
      clear();
      first = g;
    }
    const uint64_t s = wave_scan(static_cast<uint64_t>(sum), Add{});
    if (lane_id() == 63 && s)
      atomicAdd(reinterpret_cast<unsigned long long*>(&lds[g - first]), static_cast<unsigned long long>(s));
  }
  __device__ void store(int n) {
    __syncthreads();
    if (static_cast<int>(threadIdx.x) < n) sums[first + threadIdx.x] = lds[threadIdx.x];
    __syncthreads();
  }
};

template <class T>
__global__ __launch_bounds__(kT) void draw_top_kernel(const DrawArgs a, int G, int P, bool clear) {
  __shared__ Shared sh;
  const Part w(a, G, P);
  // The row's bins are cleared here, a piece by each part.
  if (clear) {
    const Params p(a, w.row);
    const bool counts = p.counts(a.V, G);
    if (counts || p.masses()) {
      uint4* const bins = reinterpret_cast<uint4*>(w.ws + (counts ? w.L.count : w.L.mass));
      for (int i = w.part * kT + threadIdx.x; i < kBins / (counts ? 4 : 2); i += P * kT) bins[i] = uint4{0, 0, 0, 0};
    }
  }
  const Row<T> r(a, w.row);
  float* const maxima = reinterpret_cast<float*>(w.ws + w.L.maxima);
  float top = -INFINITY;
  bool nan = false;
  each_segment(r, w, Segment<T>(r, w.g0), [&](int g, const Segment<T>& s) {
    float t = -INFINITY;
#pragma unroll
    for (int u = 0; u < s.PER; ++u)
#pragma unroll
      for (int e = 0; e < s.VEC; ++e) {
        t = fmaxf(t, s.x[u][e]);
        nan |= s.x[u][e] != s.x[u][e];
      }
    top = fmaxf(top, t);
    // Eight ids of each of 16 lanes: the row's last lane takes in those before it (itself, past the row's start).
    auto take = [&](auto ctrl) {
      const int v = __float_as_int(t);
      t = fmaxf(t, __int_as_float(__builtin_amdgcn_update_dpp(v, v, decltype(ctrl)::value, 0xf, 0xf, false)));
    };
    take(std::integral_constant<int, 0x111>{});
    take(std::integral_constant<int, 0x112>{});
    take(std::integral_constant<int, 0x114>{});
    take(std::integral_constant<int, 0x118>{});
    if ((threadIdx.x & 15) == 15) maxima[g * kGroups + (threadIdx.x >> 4)] = t;
  });
  const uint64_t best = block_max(nan ? 0xffffffffu : order_key(top), sh);
  if (threadIdx.x == 0) reinterpret_cast<uint64_t*>(w.ws + w.L.top)[w.part] = best;
}

// The key of the row's maximum from its parts'.
__device__ __forceinline__ uint32_t row_top(const char* ws, const Layout& L, int P, Shared& sh) {
  const uint64_t* top = reinterpret_cast<const uint64_t*>(ws + L.top);
  if (P <= 64) {
    return static_cast<uint32_t>(wave_all(top[min(lane_id(), P - 1)], Max{}));
  }
  uint64_t t = 0;
  for (int g = threadIdx.x; g < P; g += kT) t = top[g] > t ? top[g] : t;
  return static_cast<uint32_t>(block_max(t, sh));
}

// What a row's maximum says: without a distribution (NaN has the key that no number has; a maximum of
// infinity or minus infinity has none), greedy, or neither.
enum RowKind : int { kNone, kGreedy, kDraw };
struct Head {
  float x, m;
  RowKind kind;
  __device__ Head(const Params& p, uint32_t top) {
    x = key_value(top);
    m = p.T > 0.0f ? __fdiv_rn(x, p.T) : x;
    kind = !p.ok || top == 0xffffffffu || !(fabsf(m) < INFINITY) ? kNone : p.T > 0.0f ? kDraw : kGreedy;
  }
};

template <class T, bool FAST>
__device__ __forceinline__ void segment_sums(const Row<T>& r, const Part& w, const Segment<T>& first, const Dist& d,
                                             uint64_t* lds) {
  SegmentSums all(lds, w);
  each_segment(r, w, first, [&](int g, const Segment<T>& s) {
    double sum = 0.0;  // of eight whole numbers up to 2^40: exact
#pragma unroll
    for (int u = 0; u < s.PER; ++u)
#pragma unroll
      for (int e = 0; e < s.VEC; ++e)
        sum += static_cast<double>(d.weight_f(d.template below<FAST>(s.x[u][e])));
    all.add(g, sum);
  });
  all.store(w.g1 - all.first);
}

template <class T, bool FAST>
__device__ __forceinline__ void fill_bins(const Row<T>& r, const Part& w, const Segment<T>& first, const Dist& d,
                                          bool counts, uint64_t* bins) {
  each_segment(r, w, first, [&](int, const Segment<T>& s) {
#pragma unroll
    for (int u = 0; u < s.PER; ++u)
#pragma unroll
      for (int e = 0; e < s.VEC; ++e) {
        const float c = d.template below<FAST>(s.x[u][e]);
        const int b = bin_of(-c);
        if (b < kBins - 1)
          atomicAdd(reinterpret_cast<unsigned long long*>(&bins[b]),
                    static_cast<unsigned long long>(counts ? 1 : quant_detexp32(c)));
      }
  });
}

template <class T>
__global__ __launch_bounds__(kT) void draw_bins_kernel(const DrawArgs a, int G, int P) {
  __shared__ Shared sh;
  __shared__ uint64_t bins[kBins];
  const Part w(a, G, P);
  const Params p(a, w.row);
  const Row<T> r(a, w.row);
  const Segment<T> first(r, w.g0);  // in flight while the row's maximum is looked up
  const Head hd(p, row_top(w.ws, w.L, P, sh));
  if (hd.kind != kDraw) return;
  const Dist d(p.T, hd.m);
  if (!p.filtered()) {
    if (d.fast)
      segment_sums<T, true>(r, w, first, d, bins);
    else
      segment_sums<T, false>(r, w, first, d, bins);
    return;
  }
  const bool counts = p.counts(a.V, G);
  if (!counts && !p.masses()) return;
#pragma unroll
  for (int i = 0; i < kRun; ++i) bins[threadIdx.x + kT * i] = 0;
  __syncthreads();
  if (d.fast)
    fill_bins<T, true>(r, w, first, d, counts, bins);
  else
    fill_bins<T, false>(r, w, first, d, counts, bins);
  __syncthreads();
  uint32_t* const row_counts = reinterpret_cast<uint32_t*>(w.ws + w.L.count);
  uint64_t* const row_mass = reinterpret_cast<uint64_t*>(w.ws + w.L.mass);
#pragma unroll
  for (int i = 0; i < kRun; ++i) {
    const int b = threadIdx.x + kT * i;
    if (const uint64_t v = bins[b]) {
      if (counts)
        atomicAdd(&row_counts[b], static_cast<uint32_t>(v));
      else
        atomicAdd(reinterpret_cast<unsigned long long*>(&row_mass[b]), static_cast<unsigned long long>(v));
    }
  }
}

// A bound from below for the k-th largest of a row's logits, to 16 bits of its key: the k-th largest of its maxima.
__device__ __forceinline__ float kth_bound(const char* ws, const Layout& L, int G, int64_t k, Shared& sh) {
  const float* maxima = reinterpret_cast<const float*>(ws + L.maxima);
  constexpr int E = kKeyed * kGroups / kT;
  uint32_t key[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int i = threadIdx.x + kT * e;
    key[e] = i < G * kGroups ? order_key(maxima[min(i, G * kGroups - 1)]) : 0u;
  }
  uint32_t low = 0;
  for (int bit = 31; bit >= 16; --bit) {
    const uint32_t at = low | 1u << bit;
    int n = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) n += __popcll(__ballot(key[e] >= at));
    __syncthreads();
    if (lane_id() == 0) sh.red[threadIdx.x >> 6] = n;
    __syncthreads();
    uint64_t all = 0;
#pragma unroll
    for (int v = 0; v < kW; ++v) all += sh.red[v];
    if (all >= static_cast<uint64_t>(k)) low = at;
  }
  return key_value(low);
}

// Where the cut of a row under rank or mass falls, from its bins. Every thread of the workgroup calls it.
__device__ __forceinline__ void find_cut(const char* ws, const Layout& L, const Params& p, bool counts, Shared& sh,
                                         RowState* st) {
  // The row's bins, a run of them to each thread, summed from the maximum down.
  uint64_t q[kRun], mine = 0, total;
#pragma unroll
  for (int i = 0; i < kRun; i += 4) {
    if (counts) {
      const uint4 c = *reinterpret_cast<const uint4*>(ws + L.count + 4 * (kRun * threadIdx.x + i));
      q[i] = c.x, q[i + 1] = c.y, q[i + 2] = c.z, q[i + 3] = c.w;
    } else {
      const ulonglong2* m = reinterpret_cast<const ulonglong2*>(ws + L.mass + 8 * (kRun * threadIdx.x + i));
      const ulonglong2 u = m[0], v = m[1];
      q[i] = u.x, q[i + 1] = u.y, q[i + 2] = v.x, q[i + 3] = v.y;
    }
    mine += q[i] + q[i + 1] + q[i + 2] + q[i + 3];
  }
  uint64_t cum = block_scan(mine, sh, &total) - mine;
  const uint64_t limit = counts ? static_cast<uint64_t>(p.k)
                                : static_cast<uint64_t>(ceil(static_cast<double>(p.top_p) * static_cast<double>(total)));
  // The rank may lie among what weighs nothing: then nothing else is cut by it.
  if (threadIdx.x == 0) {
    st->cut_bin = kBins - 2;
    st->by = 0;
    st->need = total;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kRun; ++i) {
    if (cum < limit && cum + q[i] >= limit) {
      st->cut_bin = kRun * threadIdx.x + i;
      st->by = counts ? 1 : 2;
      st->need = limit - cum;
    }
    cum += q[i];
  }
  __syncthreads();
}

template <class T, bool FAST>
__device__ __forceinline__ void cut_segments(const Row<T>& r, const Part& w, const Segment<T>& first,
                                             const Params& p, const Dist& d,
                                             uint32_t mode, float low, int from, int cut,
                                             uint64_t* list, uint32_t* listed, uint64_t* lds) {
  SegmentSums all(lds, w);
  each_segment(r, w, first, [&](int g, const Segment<T>& s) {
    double sum = 0.0;
#pragma unroll
    for (int u = 0; u < s.PER; ++u)
#pragma unroll
      for (int e = 0; e < s.VEC; ++e) {
        const float x = s.x[u][e];
        if (!(x >= low)) continue;  // ids outside the row are minus infinity, `low` is finite
        if (mode == kSums) {
          const float c = d.template below<FAST>(x);
          const int b = bin_of(-c);
          if (b > cut) continue;
          if (b < from) {
            const double f = static_cast<double>(d.weight_f(c));
            sum += f >= static_cast<double>(p.min_w) ? f : 0.0;
            continue;
          }
        }
        const uint32_t slot = atomicAdd(listed, 1u);
        if (slot < kListMost)
          list[slot] = (static_cast<uint64_t>(~order_key(d.s(x))) << 32) | static_cast<uint32_t>(s.id(u, e));
      }
    if (mode == kSums) all.add(g, sum);
  });
  if (mode == kSums) all.store(w.g1 - all.first);
}

// One workgroup per row: what the next launch does with it.
__global__ __launch_bounds__(kT) void draw_find_kernel(const DrawArgs a, int G, int P) {
  __shared__ Shared sh;
  __shared__ RowState st;
  const int64_t row = blockIdx.x;
  const Layout L(G);
  char* const ws = a.ws + row * L.total;
  const Params p(a, row);
  const Head hd(p, row_top(ws, L, P, sh));
  if (hd.kind != kDraw || !p.filtered()) {
    if (threadIdx.x == 0) reinterpret_cast<RowState*>(ws)->mode = kNothing;
    return;
  }
  const bool both = p.k > 0 && p.top_p < 1.0f;  // top-p goes by the mass of all that top-k keeps
  if (threadIdx.x == 0) {
    st.count = 0;
    st.mode = kSums;
    st.cut_bin = kBins - 2;
    st.by = 0;
    st.need = 0;
  }
  __syncthreads();
  float low = -INFINITY;  // what is below it is not kept
  if (p.keyed(a.V, G)) {
    // Logits a little smaller may have the same quotient: half a step of it, normal or subnormal, at most.
    low = kth_bound(ws, L, G, p.k, sh);
    low = low - fabsf(low) * 0x1p-22f - p.T * 0x1p-148f;
    if (threadIdx.x == 0) st.mode = kList;
  } else if (p.k > 0 || p.top_p < 1.0f) {
    find_cut(ws, L, p, p.k > 0, sh, &st);
    if (threadIdx.x == 0 && both) st.mode = p.k <= kListMost / 2 ? kList : kRadix;
  }
  if (threadIdx.x != 0) return;
  if (p.min_w > 0 && !both) {
    // No weight of a bin after this one reaches min_p; the margin covers the logarithm's rounding and the
    // exponential's.
    const int by_m = min(bin_of(1e-3f - logf(p.min_p)) + 1, kBins - 2);
    if (by_m < static_cast<int>(st.cut_bin)) {
      st.cut_bin = by_m;
      st.by = 0;
    }
  }
  // The logit at the end of the cut's bin, less a bound for what the roundings between can make of it.
  const float end = static_cast<float>(st.cut_bin + 1) * (1.0f / kPerBin);
  low = fmaxf(low, p.T * (hd.m - end) - p.T * (fabsf(hd.m) + end) * 0x1p-18f);
  st.low = fmaxf(low, -3.4028234e38f);
  *reinterpret_cast<RowState*>(ws) = st;
}

template <class T>
__global__ __launch_bounds__(kT) void draw_cut_kernel(const DrawArgs a, int G, int P) {
  __shared__ Shared sh;
  __shared__ uint64_t list[kListMost], sums[kSumBatch];
  __shared__ uint32_t listed, base;
  const Part w(a, G, P);
  RowState* const out = reinterpret_cast<RowState*>(w.ws);
  const Row<T> r(a, w.row);
  const Segment<T> first(r, w.g0);  // in flight with what follows
  const RowState st = *out;
  const Params p(a, w.row);
  const Head hd(p, row_top(w.ws, w.L, P, sh));
  const uint32_t mode = st.mode;
  if (mode == kNothing) return;
  if (threadIdx.x == 0) listed = 0;
  __syncthreads();
  if (mode == kRadix) return;
  const int cut = static_cast<int>(st.cut_bin);
  const int from = st.by != 0 ? cut : cut + 1;  // bins before it are summed
  const float low = st.low;
  const Dist d(p.T, hd.m);
  if (d.fast)
    cut_segments<T, true>(r, w, first, p, d, mode, low, from, cut, list, &listed, sums);
  else
    cut_segments<T, false>(r, w, first, p, d, mode, low, from, cut, list, &listed, sums);
  __syncthreads();
  // A part that lists more than there is room for makes the row's count too large, too.
  const uint32_t n = min(listed, static_cast<uint32_t>(kListMost));
  if (threadIdx.x == 0 && n > 0) base = atomicAdd(&out->count, listed);
  __syncthreads();
  uint64_t* const entries = reinterpret_cast<uint64_t*>(w.ws + w.L.list);
  for (uint32_t i = threadIdx.x; i < n; i += kT)
    if (base + i < kListMost) entries[base + i] = list[i];
}

// Exact selection by radix over the keys of a row, by one workgroup: any filters, any number of ties.
template <class T>
__device__ void select_by_radix(const DrawArgs& a, int64_t row, const Params& p, const Dist& d, Keep* keep,
                                uint64_t* hist, Shared& sh) {
  const Row<T> r(a, row);
  constexpr int VEC = Row<T>::VEC;
  const int64_t words = (a.V + r.shift + VEC - 1) / VEC;
  // f(id, s) of every id of the row, in no order.
  auto each = [&](auto f) {
    constexpr int U = 4;  // loads in flight
    for (int64_t i = threadIdx.x; i < words; i += U * kT) {
      float x[U][VEC];
#pragma unroll
      for (int u = 0; u < U; ++u) r.load(i + u * kT, x[u]);
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const int64_t v = (i + u * kT) * VEC - r.shift + e;
          if (v >= 0 && v < a.V) f(static_cast<uint32_t>(v), d.s(x[u][e]));
        }
    }
  };
  // The largest key at which the sum of value(key, s) over the keys from the largest down to it reaches
  // `want`, and the sum over the keys above it.
  auto find = [&](uint64_t want, uint32_t low, bool mass, uint64_t* above) -> uint32_t {
    uint32_t prefix = 0;
    *above = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int i = threadIdx.x; i < 256; i += kT) hist[i] = 0;
      __syncthreads();
      const uint32_t mask = shift == 24 ? 0u : 0xffffffffu << (shift + 8);
      each([&](uint32_t, float s) {
        const uint32_t k = order_key(s);
        if ((k & mask) == prefix && k >= low)
          atomicAdd(reinterpret_cast<unsigned long long*>(&hist[(k >> shift) & 255]),
                    static_cast<unsigned long long>(mass ? d.weight(s) : 1));
      });
      __syncthreads();
      uint64_t all;
      const uint64_t v = threadIdx.x < 256 ? hist[255 - threadIdx.x] : 0;
      const uint64_t cum = block_scan(v, sh, &all) + *above;
      if (threadIdx.x < 256 && cum >= want && cum - v < want) {
        sh.out[0] = 255 - threadIdx.x;
        sh.out[1] = cum - v;
      }
      __syncthreads();
      prefix |= static_cast<uint32_t>(sh.out[0]) << shift;
      *above = sh.out[1];
      __syncthreads();
    }
    return prefix;
  };
  uint64_t above;
  if (p.k > 0) keep->kth = find(static_cast<uint64_t>(p.k), 0, false, &above);
  if (p.top_p < 1.0f) {
    uint64_t total = 0;
    each([&](uint32_t, float s) { total += order_key(s) >= keep->kth ? d.weight(s) : 0; });
    total = block_sum(total, sh);
    const uint64_t limit = static_cast<uint64_t>(ceil(static_cast<double>(p.top_p) * static_cast<double>(total)));
    keep->cut = find(limit, keep->kth, true, &above);
    // Equal keys have equal weights: so many of them, by increasing id.
    const uint64_t w = d.weight(key_value(keep->cut));
    uint64_t some = (limit - above + w - 1) / w;
    const int64_t per = (words + kT - 1) / kT, i0 = per * threadIdx.x, i1 = i0 + per < words ? i0 + per : words;
    uint64_t mine = 0, all;
    auto walk = [&](auto f) {
      for (int64_t i = i0; i < i1; ++i) {
        float x[VEC];
        r.load(i, x);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const int64_t v = i * VEC - r.shift + e;
          if (v >= 0 && v < a.V && order_key(d.s(x[e])) == keep->cut) f(v);
        }
      }
    };
    walk([&](int64_t) { ++mine; });
    const uint64_t upto = block_scan(mine, sh, &all);
    if (upto - mine < some && some <= upto) {
      uint64_t n = upto - mine;
      walk([&](int64_t v) {
        if (++n == some) sh.out[2] = static_cast<uint64_t>(v);
      });
    }
    __syncthreads();
    keep->last = static_cast<uint32_t>(sh.out[2]);
  }
}

constexpr int kListRun = kListMost / kT;
constexpr int kBuckets = 2048;
struct Lists {
  uint64_t bucket[kBuckets];
  uint32_t n;
};
__device__ __forceinline__ uint32_t entry_key(uint64_t e) { return ~static_cast<uint32_t>(e >> 32); }

// Buckets of a list's entries by s, from the largest down: kBuckets of equal width.
struct Bucket {
  float top, scale;
  __device__ Bucket(const uint64_t (&it)[kListRun], Shared& sh) {
    uint32_t low = 0xffffffffu, high = 0;
#pragma unroll
    for (int i = 0; i < kListRun; ++i)
      if (it[i] != ~0ull) {
        low = min(low, entry_key(it[i]));
        high = max(high, entry_key(it[i]));
      }
    top = key_value(static_cast<uint32_t>(block_max(high, sh)));
    const float width = top - key_value(static_cast<uint32_t>(block_min(low, sh)));
    scale = width > 0.0f ? (kBuckets - 1) / width : 0.0f;
  }
  __device__ __forceinline__ int operator()(uint64_t e) const {
    // NaN and what is past the last bucket: the last one.
    return static_cast<int>(fminf((top - key_value(entry_key(e))) * scale, static_cast<float>(kBuckets - 1)));
  }
};

struct Found {
  uint64_t entry, amount;
};
// Of n entries, it[threadIdx.x + kT i] of this thread, each in a bucket of an order, by increasing order(i): the first
// at which the sum of their amounts reaches `want` (at least 1, and reached). Sums by bucket give the bucket; only its entries are sorted.
// amount_of is amount for what order gave.
template <class B, class O, class A, class E>
__device__ __forceinline__ Found find_entry(int n, uint64_t want, Lists& l, uint64_t* some, Shared& sh, B bucket, O order, A amount,
                                            E amount_of) {
  constexpr int R = kBuckets / kT;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < R; ++i) l.bucket[threadIdx.x + kT * i] = 0;
  if (threadIdx.x == 0) l.n = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kListRun; ++i)
    if (static_cast<int>(threadIdx.x) + kT * i < n)
      atomicAdd(reinterpret_cast<unsigned long long*>(&l.bucket[bucket(i)]),
                static_cast<unsigned long long>(amount(i)));
  __syncthreads();
  uint64_t q[R], mine = 0, all;
#pragma unroll
  for (int i = 0; i < R; ++i) mine += q[i] = l.bucket[R * threadIdx.x + i];
  uint64_t cum = block_scan(mine, sh, &all) - mine;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    if (cum < want && want <= cum + q[i]) {
      sh.out[0] = R * threadIdx.x + i;
      sh.out[1] = cum;
    }
    cum += q[i];
  }
  __syncthreads();
  const int b = static_cast<int>(sh.out[0]);
  const uint64_t before = sh.out[1];
#pragma unroll
  for (int i = 0; i < kListRun; ++i)
    if (static_cast<int>(threadIdx.x) + kT * i < n && bucket(i) == b) some[atomicAdd(&l.n, 1u)] = order(i);
  __syncthreads();
  const int m = static_cast<int>(l.n);
  sort_lds(some, m);
  const int per = (m + kT - 1) / kT, i0 = min(m, static_cast<int>(threadIdx.x) * per), i1 = min(m, i0 + per);
  mine = 0;
  for (int i = i0; i < i1; ++i) mine += amount_of(some[i]);
  cum = block_scan(mine, sh, &all) - mine + before;
  for (int i = i0; i < i1; ++i) {
    const uint64_t v = amount_of(some[i]);
    if (cum < want && want <= cum + v) {
      sh.out[2] = some[i];
      sh.out[3] = v;
    }
    cum += v;
  }
  __syncthreads();
  return {sh.out[2], sh.out[3]};
}

// FILTERS: some row may have filters (without, the kernel is a small one, and four of its workgroups fit a CU).
template <class T, bool FILTERS>
__global__ __launch_bounds__(kT) void draw_finish_kernel(const DrawArgs a, int G, int P) {
  __shared__ Shared sh;
  __shared__ uint64_t sums[kMostSegments];  // or entries of one bucket of the list
  static_assert(kMostSegments >= kListMost, "");
  const int64_t row = blockIdx.x;
  const Layout L(G);
  char* const ws = a.ws + row * L.total;
  // All that may be needed is in flight at once.
  const Params p(a, row);
  const RowState st = *reinterpret_cast<const RowState*>(ws);
  const uint32_t word = a.words[row];
  uint64_t* const row_sums = reinterpret_cast<uint64_t*>(ws + L.sum);
  const uint64_t sum0 = row_sums[min(static_cast<int>(threadIdx.x), G - 1)];
  const uint64_t* const entries = reinterpret_cast<const uint64_t*>(ws + L.list);
  const uint64_t entry0 = FILTERS ? entries[threadIdx.x] : 0;
  const Head hd(p, row_top(ws, L, P, sh));
  if (hd.kind == kNone) {
    if (threadIdx.x == 0) give_none(a, row);
    return;
  }
  if (hd.kind == kGreedy) {  // the first segment with the maximum, and in it the first id
    const float* maxima = reinterpret_cast<const float*>(ws + L.maxima);
    uint64_t first = ~0ull;
    for (int i = threadIdx.x; i < G * kGroups; i += kT)
      if (maxima[i] == hd.x) first = min(first, static_cast<uint64_t>(i / kGroups));
    first = block_min(first, sh);
    const Segment<T> x(Row<T>(a, row), static_cast<int>(first));
    uint64_t id = ~0ull;
#pragma unroll
    for (int u = 0; u < x.PER; ++u)
#pragma unroll
      for (int e = 0; e < x.VEC; ++e)
        if (x.x[u][e] == hd.x) id = min(id, static_cast<uint64_t>(x.id(u, e)));
    id = block_min(id, sh);
    if (threadIdx.x == 0) give(a, row, static_cast<int64_t>(id), 1, 1);
    return;
  }
  const Dist d(p.T, hd.m);
  auto take_sums = [&]() {
    if (static_cast<int>(threadIdx.x) < G) sums[threadIdx.x] = sum0;
    for (int g = threadIdx.x + kT; g < G; g += kT) sums[g] = row_sums[g];
    __syncthreads();
  };
  if (!p.filtered()) {
    take_sums();
    draw_from_segments<T>(a, row, word, sums, G, d, Keep{}, sh);
    return;
  }
  if constexpr (FILTERS) {
  __shared__ Lists lists;
  const uint32_t listed = st.count, by = st.by;
  const uint32_t mode = listed > kListMost ? kRadix : st.mode;
  Keep keep;
  keep.min_w = p.min_w;
  if (mode == kRadix) {
    select_by_radix<T>(a, row, p, d, &keep, lists.bucket, sh);
    const Row<T> r(a, row);
    for (int g = 0; g < G; ++g) {
      const Segment<T> x(r, g);
      uint64_t s = 0;
#pragma unroll
      for (int u = 0; u < x.PER; ++u)
#pragma unroll
        for (int e = 0; e < x.VEC; ++e)
          s += keep.weight(d, d.s(x.x[u][e]), static_cast<uint32_t>(x.id(u, e)));
      s = block_sum(s, sh);
      if (threadIdx.x == 0) sums[g] = s;
    }
    __syncthreads();
    draw_from_segments<T>(a, row, word, sums, G, d, keep, sh);
    return;
  }
  // The list: a run of it to each thread, its weights in registers.
  const int n = static_cast<int>(listed);
  uint64_t it[kListRun], wt[kListRun];
#pragma unroll
  for (int i = 0; i < kListRun; ++i) {
    const int at = threadIdx.x + kT * i;
    it[i] = at >= n ? ~0ull : i == 0 ? entry0 : entries[at];
    wt[i] = at < n ? d.weight(key_value(entry_key(it[i]))) : 0;
  }
  const Bucket by_s(it, sh);
  const bool whole = mode == kList;
  const uint64_t rank = whole ? static_cast<uint64_t>(p.k) : by == 1 ? st.need : 0;
  if (rank > 0 && rank <= static_cast<uint64_t>(n)) {
    const uint64_t last = find_entry(
        n, rank, lists, sums, sh, [&](int i) { return by_s(it[i]); }, [&](int i) { return it[i]; },
        [&](int) { return 1ull; }, [](uint64_t) { return 1ull; }).entry;
    keep.kth = entry_key(last);
  }
  if (whole ? p.top_p < 1.0f : by == 2) {
    uint64_t limit = st.need;
    if (whole) {  // of what top-k keeps
      uint64_t t = 0;
#pragma unroll
      for (int i = 0; i < kListRun; ++i) t += entry_key(it[i]) >= keep.kth ? wt[i] : 0;
      limit = static_cast<uint64_t>(ceil(static_cast<double>(p.top_p) * static_cast<double>(block_sum(t, sh))));
    }
    const uint64_t last = find_entry(
        n, limit, lists, sums, sh, [&](int i) { return by_s(it[i]); }, [&](int i) { return it[i]; },
        [&](int i) { return entry_key(it[i]) >= keep.kth ? wt[i] : 0; },
        [&](uint64_t e) { return entry_key(e) >= keep.kth ? d.weight(key_value(entry_key(e))) : 0; }).entry;
    keep.cut = entry_key(last);
    keep.last = static_cast<uint32_t>(last);
  }
  auto kept = [&](uint64_t e, uint64_t w) {
    const uint32_t k = entry_key(e);
    return k >= keep.kth && (k > keep.cut || (k == keep.cut && static_cast<uint32_t>(e) <= keep.last)) &&
                   w >= p.min_w
               ? w
               : 0;
  };
  if (!whole) {
    const int shift = Row<T>(a, row).shift;
    __syncthreads();
    take_sums();
    if (by != 0) {
#pragma unroll
      for (int i = 0; i < kListRun; ++i)
        if (const uint64_t w = kept(it[i], wt[i]))
          atomicAdd(reinterpret_cast<unsigned long long*>(&sums[(static_cast<uint32_t>(it[i]) + shift) / kDrawSeg]),
                    static_cast<unsigned long long>(w));
      __syncthreads();
    }
    draw_from_segments<T>(a, row, word, sums, G, d, keep, sh);
    return;
  }
  // The draw: by id.
  uint64_t total = 0;
#pragma unroll
  for (int i = 0; i < kListRun; ++i) {
    wt[i] = kept(it[i], wt[i]);
    total += wt[i];
  }
  total = block_sum(total, sh);
  const uint64_t at = icdf_threshold(word, total);
  const float scale = static_cast<float>(kBuckets) / static_cast<float>(a.V);
  const Found f = find_entry(
      n, at + 1, lists, sums, sh,
      [&](int i) { return min(static_cast<int>(static_cast<float>(static_cast<uint32_t>(it[i])) * scale), kBuckets - 1); },
      [&](int i) { return it[i] << 32 | it[i] >> 32; }, [&](int i) { return wt[i]; },
      [&](uint64_t e) { return kept(e << 32 | e >> 32, d.weight(key_value(~static_cast<uint32_t>(e)))); });
  if (threadIdx.x == 0) give(a, row, static_cast<int64_t>(f.entry >> 32), f.amount, total);
  }
}

// Workgroups of a launch: twice what fits the GPU at a time, four of 512 threads to each of 256 CUs, so that the
// parts are small beside the whole (272 rows of 151,936 under one min-p 101 us with once as many, 94 with twice).
constexpr int64_t kFill = 2048;

template <class T>
hipError_t launch_draw_as(const DrawArgs& a, hipStream_t stream) {
  // Parts of a row: as many as give kFill workgroups in all, a segment at least.
  const int64_t G = draw_segments(a.V), most = (kFill + a.N - 1) / a.N, parts = most < G ? most : G;
  if (a.N * parts > kMaxThreads / kT || a.N * parts > 0x7fffffff) return hipErrorInvalidConfiguration;
  const dim3 grid(static_cast<unsigned>(a.N * parts)), rows(static_cast<unsigned>(a.N));
  const int g = static_cast<int>(G), p = static_cast<int>(parts);
  const bool greedy = !a.temperatures && a.temperature == 0.0f;
  const bool filters =
      !greedy && (a.top_ks || a.top_ps || a.min_ps || a.top_k > 0 || a.top_p < 1.0f || a.min_p > 0.0f);
  // Under one top-k or min-p for all rows nothing is binned.
  const bool one = !a.temperatures && !a.top_ks && !a.top_ps && !a.min_ps;
  const bool bins = !one || !filters || (a.top_k > 0 ? a.top_k > a.V / 128 || G > kKeyed : a.top_p < 1.0f);
  hipLaunchKernelGGL(draw_top_kernel<T>, grid, dim3(kT), 0, stream, a, g, p, filters && bins);
  if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  if (!greedy && bins) {
    hipLaunchKernelGGL(draw_bins_kernel<T>, grid, dim3(kT), 0, stream, a, g, p);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  if (filters) {
    hipLaunchKernelGGL(draw_find_kernel, rows, dim3(kT), 0, stream, a, g, p);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    hipLaunchKernelGGL(draw_cut_kernel<T>, grid, dim3(kT), 0, stream, a, g, p);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  if (filters)
    hipLaunchKernelGGL((draw_finish_kernel<T, true>), rows, dim3(kT), 0, stream, a, g, p);
  else
    hipLaunchKernelGGL((draw_finish_kernel<T, false>), rows, dim3(kT), 0, stream, a, g, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_draw(const DrawArgs& a, hipStream_t stream) {
  return a.bf16 ? launch_draw_as<__bf16>(a, stream) : launch_draw_as<float>(a, stream);
}

}  // namespace dbl
