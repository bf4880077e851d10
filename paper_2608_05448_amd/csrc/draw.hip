// One token per row of logits by temperature, top-k, top-p and min-p, from a given random word.
//
// The distribution is the target transform's (target.hip): s = fl32(logit / T), integer weights
// w = floor(detexp32(fl32(s - max)) 2^40), top-k with its ties, then top-p by decreasing s and
// increasing id; and then min-p. The token is the inverse CDF of the word over the kept weights in id
// order. Everything that decides is an integer, so the token depends neither on how a row is
// split nor on the other rows.
//
// What bounds it is reading the logits. A row is split into segments of kDrawSeg ids, one workgroup each,
// so that few rows still use the whole GPU, in three launches, the later of which read the logits
// from the caches:
//   top    maximum of each segment (with its lowest id: the greedy token)
//   bins   without filters the sum of each segment's weights; with them, counts and sums of weights in
//          bins of max - s. The row's last workgroup then draws the token, or finds the bin that the
//          cut falls into (a ticket per row; nobody waits)
//   cut    (only where there are filters) a list of what is above or at the cut, if that is at most
//          kListMost ids, else the sum of what is above it by segment and a list of the cut's bin.
//          The row's last workgroup sorts the list, finds the exact cut and draws. Rows that fit
//          neither (a large top-k together with top-p, more than kListMost ids in one bin) are
//          selected by radix over their order-preserving keys, by that workgroup alone.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "contract.hpp"
#include "kernels.hpp"
#include "wave.hpp"

namespace dbl {
namespace {

constexpr int kT = 512;        // threads of a workgroup
constexpr int kW = kT / 64;
constexpr int kBins = kDrawBins;  // of max - s
constexpr float kPerBin = 32;     // of width 1 / 32; the last one holds all that is 16 or more below the maximum
constexpr int kListMost = kDrawList;
static_assert(kBins == kT, "a thread per bin in the merge");

// kList: the list takes all bins up to cut_bin. kSums: the list takes cut_bin (by != 0), the bins before it are
// summed by segment. by: 0, nothing is cut inside that bin; 1, by rank: `need` is the last one's, from 1 within
// the bin; 2, by mass: an id is kept while less than `need` is kept before it (in the bin; kList: in the row).
enum RowMode : uint32_t { kDone = 0, kList = 1, kSums = 2, kRadix = 3 };
using RowState = DrawState;
using Layout = DrawLayout;

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
  // The values of word i, -inf outside the row.
  __device__ __forceinline__ void load(int64_t i, float (&x)[VEC]) const {
    const int64_t v0 = i * VEC - shift;
    const T* p = base + i * VEC;
    if (v0 < V && p + VEC <= end) {
      const uint4 q = *reinterpret_cast<const uint4*>(p);
      const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        if constexpr (sizeof(T) == 4)
          x[e] = __uint_as_float(w[e]);
        else
          x[e] = __uint_as_float((e & 1) ? (w[e / 2] & 0xffff0000u) : (w[e / 2] << 16));
      }
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
};

struct Shared {
  uint64_t red[kW + 1];
  uint64_t out[4];
  uint32_t flag;
};

template <class Op>
__device__ __forceinline__ uint64_t block_reduce(uint64_t v, Shared& sh, Op op) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = op(v, static_cast<uint64_t>(__shfl_xor(v, o)));
  __syncthreads();
  if (lane_id() == 0) sh.red[threadIdx.x >> 6] = v;
  __syncthreads();
  uint64_t r = sh.red[0];
#pragma unroll
  for (int w = 1; w < kW; ++w) r = op(r, sh.red[w]);
  return r;
}
__device__ __forceinline__ uint64_t block_sum(uint64_t v, Shared& sh) {
  return block_reduce(v, sh, [](uint64_t x, uint64_t y) { return x + y; });
}
__device__ __forceinline__ uint64_t block_max(uint64_t v, Shared& sh) {
  return block_reduce(v, sh, [](uint64_t x, uint64_t y) { return x > y ? x : y; });
}
// Sum over the threads up to and including this one; *all: of the workgroup.
__device__ __forceinline__ uint64_t block_scan(uint64_t v, Shared& sh, uint64_t* all) {
  uint64_t s = wave_incl_scan_u64(v);
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

// Whether this workgroup is the last of its row's n to come here; what the others wrote before they
// came is then visible to it.
__device__ __forceinline__ bool last_of_row(uint32_t* ticket, uint32_t n, Shared& sh) {
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0)
    sh.flag = __hip_atomic_fetch_add(ticket, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == n - 1;
  __syncthreads();
  const bool last = sh.flag != 0;
  if (last) __threadfence();
  return last;
}

// The distribution of a row: weight of a logit, its key, and what is kept.
struct Dist {
  float T, m;
  __device__ __forceinline__ float s(float x) const { return __fdiv_rn(x, T); }
  __device__ __forceinline__ uint64_t weight(float sv) const { return quant_detexp32(__fsub_rn(sv, m)); }
  __device__ __forceinline__ int bin(float sv) const {
    return static_cast<int>(fminf(__fsub_rn(m, sv) * kPerBin, static_cast<float>(kBins - 1)));
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

// Draws from the sums of a row's segments, seg[0 .. G): the segment that holds the threshold, and in it the id.
// Every thread of the workgroup calls it.
template <class T>
__device__ void draw_from_segments(const DrawArgs& a, int64_t row, const uint64_t* seg, int G, const Dist& d,
                                   const Keep& keep, Shared& sh) {
  uint64_t mine = 0, total;
  const int per = (G + kT - 1) / kT, g0 = min(G, static_cast<int>(threadIdx.x) * per), g1 = min(G, g0 + per);
  for (int g = g0; g < g1; ++g) mine += seg[g];
  const uint64_t incl = block_scan(mine, sh, &total);
  if (total == 0) {  // unreachable: the maximum weighs 2^40 and is kept
    if (threadIdx.x == 0) give_none(a, row);
    return;
  }
  const uint64_t at = icdf_threshold(a.words[row], total);
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

// Ascending sort of n keys in LDS, padded with ~0 to a power of two.
__device__ void sort_lds(uint64_t* v, int n) {
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
template <class T>
__global__ __launch_bounds__(kT) void draw_top_kernel(const DrawArgs a, int G) {
  __shared__ Shared sh;
  const int64_t row = blockIdx.x / G;
  const int g = blockIdx.x % G;
  const Layout L(G);
  char* const ws = a.ws + row * L.total;
  if (g == 0 && threadIdx.x == 0) {
    RowState* st = reinterpret_cast<RowState*>(ws);
    st->tickets[0] = st->tickets[1] = 0;
    st->count = 0;
    st->mode = kDone;
  }
  constexpr int VEC = Row<T>::VEC, PER = kDrawSeg / VEC / kT;
  const Row<T> r(a, row);
  float x[PER][VEC];
#pragma unroll
  for (int i = 0; i < PER; ++i)
    r.load(static_cast<int64_t>(g) * (kDrawSeg / VEC) + threadIdx.x + kT * i, x[i]);
  uint64_t top = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i)
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const int64_t v = (static_cast<int64_t>(g) * (kDrawSeg / VEC) + threadIdx.x + kT * i) * VEC - r.shift + e;
      // NaN of either sign comes before everything.
      const uint32_t k = x[i][e] != x[i][e] ? 0xffffffffu : order_key(x[i][e]);
      const uint64_t c = (static_cast<uint64_t>(k) << 32) | (0xffffffffu - static_cast<uint32_t>(v));
      if (v >= 0 && v < a.V) top = c > top ? c : top;
    }
  top = block_max(top, sh);
  if (threadIdx.x == 0) reinterpret_cast<uint64_t*>(ws + L.top)[g] = top;
}

// The row's maximum from its segments'.
__device__ __forceinline__ uint64_t row_top(const char* ws, const Layout& L, int G, Shared& sh) {
  const uint64_t* top = reinterpret_cast<const uint64_t*>(ws + L.top);
  if (G <= 64) {
    uint64_t t = top[min(lane_id(), G - 1)];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      const uint64_t u = __shfl_xor(t, o);
      t = u > t ? u : t;
    }
    return t;
  }
  uint64_t t = 0;
  for (int g = threadIdx.x; g < G; g += kT) t = top[g] > t ? top[g] : t;
  return block_max(t, sh);
}

struct Merge {  // of a row's bins, in LDS
  uint32_t count[kBins];
  uint64_t mass[kBins];
};

template <class T>
__global__ __launch_bounds__(kT) void draw_bins_kernel(const DrawArgs a, int G) {
  __shared__ Shared sh;
  __shared__ Merge bins;
  const int64_t row = blockIdx.x / G;
  const int g = blockIdx.x % G;
  const Layout L(G);
  char* const ws = a.ws + row * L.total;
  RowState* const st = reinterpret_cast<RowState*>(ws);
  const Params p(a, row);
  const uint64_t top = row_top(ws, L, G, sh);
  const float xm = key_value(static_cast<uint32_t>(top >> 32));
  const Dist d{p.T, p.T > 0.0f ? __fdiv_rn(xm, p.T) : xm};
  // NaN has the key that no number has; a maximum of infinity or minus infinity has no distribution.
  if (!p.ok || (top >> 32) == 0xffffffffu || !(fabsf(d.m) < INFINITY)) {
    if (g == 0 && threadIdx.x == 0) give_none(a, row);
    return;
  }
  if (p.T == 0.0f) {
    if (g == 0 && threadIdx.x == 0)
      give(a, row, 0xffffffffu - static_cast<uint32_t>(top), 1, 1);
    return;
  }
  constexpr int VEC = Row<T>::VEC, PER = kDrawSeg / VEC / kT;
  const Row<T> r(a, row);
  float x[PER][VEC];
#pragma unroll
  for (int i = 0; i < PER; ++i)
    r.load(static_cast<int64_t>(g) * (kDrawSeg / VEC) + threadIdx.x + kT * i, x[i]);
  uint64_t* const sums = reinterpret_cast<uint64_t*>(ws + L.sum);
  if (!p.filtered()) {
    uint64_t s = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i)
#pragma unroll
      for (int e = 0; e < VEC; ++e) s += d.weight(d.s(x[i][e]));
    s = block_sum(s, sh);
    if (threadIdx.x == 0) sums[g] = s;
    if (last_of_row(&st->tickets[0], G, sh)) draw_from_segments<T>(a, row, sums, G, d, Keep{}, sh);
    return;
  }
  bins.count[threadIdx.x] = 0;
  bins.mass[threadIdx.x] = 0;
  __syncthreads();
  const bool masses = p.top_p < 1.0f && p.k == 0;
#pragma unroll
  for (int i = 0; i < PER; ++i)
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const float s = d.s(x[i][e]);
      const int b = d.bin(s);
      atomicAdd(&bins.count[b], 1u);
      if (masses)
        atomicAdd(reinterpret_cast<unsigned long long*>(&bins.mass[b]),
                  static_cast<unsigned long long>(d.weight(s)));
    }
  __syncthreads();
  uint32_t* const counts = reinterpret_cast<uint32_t*>(ws + L.count);
  uint64_t* const mass = reinterpret_cast<uint64_t*>(ws + L.mass);
  counts[static_cast<int64_t>(g) * kBins + threadIdx.x] = bins.count[threadIdx.x];
  if (masses) mass[static_cast<int64_t>(g) * kBins + threadIdx.x] = bins.mass[threadIdx.x];
  if (!last_of_row(&st->tickets[0], G, sh)) return;

  // The row's bins, summed from the maximum down; where the cut falls.
  uint64_t c = 0, q = 0, all;
  for (int i = 0; i < G; ++i) c += counts[static_cast<int64_t>(i) * kBins + threadIdx.x];
  if (masses)
    for (int i = 0; i < G; ++i) q += mass[static_cast<int64_t>(i) * kBins + threadIdx.x];
  const uint64_t cum = block_scan(c, sh, &all);
  uint64_t total = 0, cum_mass = 0;
  if (masses) cum_mass = block_scan(q, sh, &total);
  const uint64_t limit =
      masses ? static_cast<uint64_t>(ceil(static_cast<double>(p.top_p) * static_cast<double>(total))) : 0;
  if (threadIdx.x == 0) sh.out[0] = sh.out[1] = kBins - 1;
  __syncthreads();
  const uint64_t rank = static_cast<uint64_t>(p.k);
  if (p.k > 0 && cum >= rank && cum - c < rank) sh.out[0] = threadIdx.x;
  if (masses && cum_mass >= limit && cum_mass - q < limit) sh.out[1] = threadIdx.x;
  __syncthreads();
  const int by_k = static_cast<int>(sh.out[0]), by_p = static_cast<int>(sh.out[1]);
  // No weight of a later bin than this one reaches min_p; the margin covers the logarithm's rounding and
  // the exponential's.
  const int by_m =
      p.min_w > 0 ? static_cast<int>(fminf((1e-3f - logf(p.min_p)) * kPerBin + 1.0f, kBins - 1)) : kBins - 1;
  int cut = by_k < by_p ? by_k : by_p;
  uint32_t by = p.k > 0 ? 1 : masses ? 2 : 0;
  if (by_m < cut && !(p.k > 0 && p.top_p < 1.0f)) {  // top-p goes by the mass of all that top-k keeps
    cut = by_m;
    by = 0;
  }
  if (threadIdx.x == cut) {
    st->cut_bin = cut;
    uint32_t mode = kRadix;
    uint64_t need = limit;
    if (cum <= kListMost) {
      mode = kList;
    } else if (by == 0 || (c <= kListMost && !(p.k > 0 && p.top_p < 1.0f))) {
      mode = kSums;
      need = by == 1 ? rank - (cum - c) : by == 2 ? limit - (cum_mass - q) : 0;
    }
    st->mode = mode;
    st->by = by;
    st->need = need;
  }
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
    for (int64_t i = threadIdx.x; i < words; i += kT) {
      float x[VEC];
      r.load(i, x);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const int64_t v = i * VEC - r.shift + e;
        if (v >= 0 && v < a.V) f(static_cast<uint32_t>(v), d.s(x[e]));
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

template <class T>
__global__ __launch_bounds__(kT) void draw_cut_kernel(const DrawArgs a, int G) {
  __shared__ Shared sh;
  __shared__ uint64_t list[kListMost];
  const int64_t row = blockIdx.x / G;
  const int g = blockIdx.x % G;
  const Layout L(G);
  char* const ws = a.ws + row * L.total;
  RowState* const st = reinterpret_cast<RowState*>(ws);
  const uint32_t mode = st->mode;
  if (mode == kDone) return;
  const Params p(a, row);
  const uint64_t top = row_top(ws, L, G, sh);
  const Dist d{p.T, __fdiv_rn(key_value(static_cast<uint32_t>(top >> 32)), p.T)};
  const int cut = static_cast<int>(st->cut_bin);
  const uint32_t by = st->by;
  uint64_t* const entries = reinterpret_cast<uint64_t*>(ws + L.list);
  uint64_t* const sums = reinterpret_cast<uint64_t*>(ws + L.sum);
  constexpr int VEC = Row<T>::VEC, PER = kDrawSeg / VEC / kT;
  if (mode != kRadix) {
    const Row<T> r(a, row);
    float x[PER][VEC];
#pragma unroll
    for (int i = 0; i < PER; ++i)
      r.load(static_cast<int64_t>(g) * (kDrawSeg / VEC) + threadIdx.x + kT * i, x[i]);
    uint64_t sum = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i)
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const int64_t v = (static_cast<int64_t>(g) * (kDrawSeg / VEC) + threadIdx.x + kT * i) * VEC - r.shift + e;
        const float s = d.s(x[i][e]);
        const int b = d.bin(s);
        if (b > cut || v < 0 || v >= a.V) continue;
        if (mode == kList || (by != 0 && b == cut)) {
          const uint32_t slot = atomicAdd(&st->count, 1u);
          if (slot < kListMost)  // always: the bins were counted
            entries[slot] = (static_cast<uint64_t>(~order_key(s)) << 32) | static_cast<uint32_t>(v);
        } else {
          const uint64_t w = d.weight(s);
          sum += w >= p.min_w ? w : 0;
        }
      }
    if (mode == kSums) {
      sum = block_sum(sum, sh);
      if (threadIdx.x == 0) sums[g] = sum;
    }
  }
  if (!last_of_row(&st->tickets[1], G, sh)) return;

  Keep keep;
  keep.min_w = p.min_w;
  if (mode == kRadix) {
    select_by_radix<T>(a, row, p, d, &keep, list, sh);
    const Row<T> r(a, row);
    for (int i = 0; i < G; ++i) {
      uint64_t s = 0;
      for (int u = 0; u < PER; ++u) {
        float x[VEC];
        const int64_t at = static_cast<int64_t>(i) * (kDrawSeg / VEC) + threadIdx.x + kT * u;
        r.load(at, x);
#pragma unroll
        for (int e = 0; e < VEC; ++e)
          s += keep.weight(d, d.s(x[e]), static_cast<uint32_t>(at * VEC - r.shift + e));
      }
      s = block_sum(s, sh);
      if (threadIdx.x == 0) sums[i] = s;
    }
    __syncthreads();
    draw_from_segments<T>(a, row, sums, G, d, keep, sh);
    return;
  }
  const int n = static_cast<int>(min(st->count, static_cast<uint32_t>(kListMost)));
  for (int i = threadIdx.x; i < n; i += kT) list[i] = entries[i];
  __syncthreads();
  if (n > 0) sort_lds(list, n);

  // The sorted list, a run of it to each thread: weights and their sums from the largest on.
  constexpr int RUN = kListMost / kT;
  const int per = (n + kT - 1) / kT, i0 = min(n, static_cast<int>(threadIdx.x) * per), i1 = min(n, i0 + per);
  uint64_t mine = 0, all = 0;
  uint64_t w[RUN];
#pragma unroll
  for (int i = 0; i < RUN; ++i) {
    w[i] = i0 + i < i1 ? d.weight(key_value(~static_cast<uint32_t>(list[i0 + i] >> 32))) : 0;
    mine += w[i];
  }
  const uint64_t start = block_scan(mine, sh, &all) - mine;
  int kept = n;
  auto key_of = [&](int i) { return ~static_cast<uint32_t>(list[i] >> 32); };
  auto count_if = [&](auto f) {  // entries of the list for which f(i, weight, sum before)
    uint64_t c = 0, before = start;
#pragma unroll
    for (int i = 0; i < RUN; ++i) {
      if (i0 + i < i1) c += f(i0 + i, w[i], before) ? 1 : 0;
      before += w[i];
    }
    return static_cast<int>(block_sum(c, sh));
  };
  const bool whole = mode == kList;
  const int64_t rank = whole ? p.k : by == 1 ? static_cast<int64_t>(st->need) : 0;
  if (rank > 0 && rank <= n) {
    const uint32_t kth = key_of(static_cast<int>(rank) - 1);
    kept = count_if([&](int i, uint64_t, uint64_t) { return key_of(i) >= kth; });
  }
  if (whole ? p.top_p < 1.0f : by == 2) {
    uint64_t limit = st->need;
    if (p.k > 0) {  // of what top-k keeps: the list's first `kept`
      uint64_t t = 0;
#pragma unroll
      for (int i = 0; i < RUN; ++i) t += i0 + i < kept ? w[i] : 0;
      limit = static_cast<uint64_t>(ceil(static_cast<double>(p.top_p) * static_cast<double>(block_sum(t, sh))));
    }
    kept = min(kept, count_if([&](int, uint64_t, uint64_t before) { return before < limit; }));
  }
  if (mode == kSums) {
    if (by != 0) {  // the cut's bin is not empty
      keep.cut = key_of(kept - 1);
      keep.last = static_cast<uint32_t>(list[kept - 1]);
#pragma unroll
      for (int i = 0; i < RUN; ++i)
        if (i0 + i < min(i1, kept) && w[i] >= p.min_w) {
          const Row<T> r(a, row);
          const int64_t at = static_cast<int64_t>(static_cast<uint32_t>(list[i0 + i])) + r.shift;
          atomicAdd(reinterpret_cast<unsigned long long*>(&sums[at / kDrawSeg]),
                    static_cast<unsigned long long>(w[i]));
        }
      __threadfence();
      __syncthreads();
    }
    draw_from_segments<T>(a, row, sums, G, d, keep, sh);
    return;
  }
  // What is drawn from, by id: id and weight in one word (24 and 40 bits; no weight is above 2^40).
  const int in_cut = kept;
  kept = count_if([&](int i, uint64_t wi, uint64_t) { return i < in_cut && wi >= p.min_w && wi > 0; });
  uint64_t packed[RUN];
#pragma unroll
  for (int i = 0; i < RUN; ++i)
    packed[i] = i0 + i < i1 && i0 + i < in_cut && w[i] >= p.min_w && w[i] > 0
                    ? (list[i0 + i] & 0xffffffffull) << 40 | (w[i] - 1)
                    : ~0ull;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < RUN; ++i)
    if (i0 + i < i1) list[i0 + i] = packed[i];
  __syncthreads();
  sort_lds(list, in_cut);
  const int pk = (kept + kT - 1) / kT, j0 = min(kept, static_cast<int>(threadIdx.x) * pk), j1 = min(kept, j0 + pk);
  uint64_t v[RUN], sum = 0, total;
#pragma unroll
  for (int i = 0; i < RUN; ++i) {
    v[i] = j0 + i < j1 ? (list[j0 + i] & 0xffffffffffull) + 1 : 0;
    sum += v[i];
  }
  uint64_t c = block_scan(sum, sh, &total) - sum;
  const uint64_t at = icdf_threshold(a.words[row], total);
#pragma unroll
  for (int i = 0; i < RUN; ++i) {
    if (c <= at && at < c + v[i]) give(a, row, static_cast<int64_t>(list[j0 + i] >> 40), v[i], total);
    c += v[i];
  }
}

template <class T>
hipError_t launch_draw_as(const DrawArgs& a, hipStream_t stream) {
  const int64_t G = draw_segments(a.V);
  if (a.N * G > kMaxThreads / kT || a.N * G > 0x7fffffff) return hipErrorInvalidConfiguration;
  const dim3 grid(static_cast<unsigned>(a.N * G));
  const int g = static_cast<int>(G);
  hipLaunchKernelGGL(draw_top_kernel<T>, grid, dim3(kT), 0, stream, a, g);
  if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  hipLaunchKernelGGL(draw_bins_kernel<T>, grid, dim3(kT), 0, stream, a, g);
  if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  const bool filters = a.top_ks || a.top_ps || a.min_ps || a.top_k > 0 || a.top_p < 1.0f || a.min_p > 0.0f;
  if (filters) hipLaunchKernelGGL(draw_cut_kernel<T>, grid, dim3(kT), 0, stream, a, g);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_draw(const DrawArgs& a, hipStream_t stream) {
  return a.bf16 ? launch_draw_as<__bf16>(a, stream) : launch_draw_as<float>(a, stream);
}

}  // namespace dbl
