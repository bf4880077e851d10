// C ABI of the training operators (declared in include/dblast.h): argument validation, workspace layout
// and status mapping around their launchers.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <new>
#include <string>
#include <utility>
#include <vector>

#include "abi_common.hpp"

using namespace dbl_abi;

namespace {

dbl_status check_nll(const dbl_shape& s, int dt) {
  if (dbl_status st = check_shape(s, true)) return st;
  if (dt != DBL_BF16 && dt != DBL_F32) return fail(DBL_EDTYPE, "dt must be DBL_BF16 or DBL_F32");
  if (dt == DBL_BF16 && s.d % 8 != 0) return fail(DBL_ESHAPE, "bf16 head needs d % 8 == 0");
  if (static_cast<double>(s.B) * s.K * s.R > static_cast<double>(dbl::kMaxTrainRows))
    return fail(DBL_ESHAPE, "B*K*R must be < 2^24");
  return ok();
}

dbl::NllArgs nll_args(const dbl_shape& s, int dt, const void* h, const void* w, const int32_t* x,
                      char* base, const WsLayout& L) {
  dbl::NllArgs a{};
  a.P = s.B * s.K;
  a.R = s.R;
  a.V = s.V;
  a.d = static_cast<int>(s.d);
  a.bf16 = dt == DBL_BF16;
  a.h = h;
  a.w = w;
  a.x = x;
  a.count = reinterpret_cast<int32_t*>(base + L.off[0]);
  a.inv = reinterpret_cast<int32_t*>(base + L.off[1]);
  a.rows = reinterpret_cast<dbl::TrainRow*>(base + L.off[2]);
  a.hc = base + L.off[3];
  return a;
}

// The tensors of a norm or clipping call: sizes, types and addresses.
dbl_status check_tensors(int64_t n, const void* const* grads, const int64_t* numel,
                         const int32_t* dt, void* const* out, bool clip,
                         std::vector<dbl::GradTensor>* to) {
  if (n < 0 || n > dbl::kMaxTensors) return fail(DBL_ESHAPE, "need 0 <= n <= 2^20 tensors");
  if (n > 0 && (!grads || !numel || !dt)) return fail(DBL_EINVAL, "NULL array");
  to->resize(static_cast<size_t>(n));
  int64_t all = 0;
  for (int64_t i = 0; i < n; ++i) {
    dbl::GradTensor& t = (*to)[static_cast<size_t>(i)];
    if (dt[i] != DBL_F32 && dt[i] != DBL_BF16)
      return fail(DBL_EDTYPE, "dt must be DBL_BF16 or DBL_F32");
    if (numel[i] < 0 || numel[i] >= dbl::kMaxGradElements - all)
      return fail(DBL_ESHAPE, "numel must be >= 0 and less than 2^40 together");
    all += numel[i];
    t.n = numel[i];
    t.bf16 = dt[i] == DBL_BF16;
    t.g = grads[i];
    t.out = !clip ? nullptr : out ? out[i] : const_cast<void*>(grads[i]);
    if (t.n == 0) continue;
    if (!t.g || (clip && !t.out)) return fail(DBL_EINVAL, "NULL tensor");
    const uintptr_t e = t.bf16 ? 2 : 4;
    if (reinterpret_cast<uintptr_t>(t.g) % e != 0 || reinterpret_cast<uintptr_t>(t.out) % e != 0)
      return fail(DBL_EINVAL, "a tensor is not aligned to its elements");
  }
  return ok();
}

}  // namespace

extern "C" {

dbl_status dbl_head_nll(dbl_shape s, int dt, const void* h, const void* w, const int32_t* x,
                        float* nll, float* lse, void* ws, size_t ws_bytes, void* stream) {
  return guarded([&]() -> dbl_status {
    if (dbl_status st = check_nll(s, dt)) return st;
    if (!w || (s.B > 0 && (!h || !x || !nll || !lse))) return fail(DBL_EINVAL, "NULL pointer");
    if (dbl_status st = check_aligned({{h, "h"}, {w, "w"}, {x, "x"}, {nll, "nll"}, {lse, "lse"}}))
      return st;
    const size_t e = dt == DBL_BF16 ? 2 : 4;
    const size_t rows = static_cast<size_t>(s.B) * s.K * s.R;
    std::vector<Span> spans = {{h, rows * s.d * e, false}, {w, static_cast<size_t>(s.V) * s.d * e, false},
                               {x, size_t(4) * s.B * s.K, false}, {nll, 4 * rows, true},
                               {lse, 4 * rows, true}};
    if (overlapping(spans)) return fail(DBL_EINVAL, "nll and lse must not overlap another array");
    if (s.B == 0) return ok();
    WsLayout L;
    if (dbl_status st = check_ws(DBL_OP_HEAD_NLL, s, ws, ws_bytes, &L)) return st;
    char* const base = static_cast<char*>(ws);
    dbl::NllArgs a = nll_args(s, dt, h, w, x, base, L);
    a.nll = nll;
    a.lse = lse;
    a.lmass = reinterpret_cast<float*>(base + L.off[4]);
    a.tgt = reinterpret_cast<float*>(base + L.off[5]);
    return hip_status(dbl::launch_nll(a, static_cast<hipStream_t>(stream)), "head nll launch");
  });
}

dbl_status dbl_head_nll_backward(dbl_shape s, int dt, const void* h, const void* w,
                                 const int32_t* x, const float* nll, const float* lse, const float* g,
                                 void* dh, void* dw, void* ws, size_t ws_bytes, void* stream) {
  return guarded([&]() -> dbl_status {
    if (dbl_status st = check_nll(s, dt)) return st;
    if (!w || (s.B > 0 && (!h || !x || !nll || !lse || !g || !dh)))
      return fail(DBL_EINVAL, "NULL pointer");
    if (dbl_status st = check_aligned({{h, "h"}, {w, "w"}, {x, "x"}, {nll, "nll"}, {lse, "lse"},
                                       {g, "g"}, {dh, "dh"}, {dw, "dw"}}))
      return st;
    const size_t e = dt == DBL_BF16 ? 2 : 4;
    const size_t rows = static_cast<size_t>(s.B) * s.K * s.R;
    const size_t hb = rows * s.d * e, wb = static_cast<size_t>(s.V) * s.d * e;
    std::vector<Span> spans = {{h, hb, false}, {w, wb, false}, {x, size_t(4) * s.B * s.K, false},
                               {nll, 4 * rows, false}, {lse, 4 * rows, false}, {g, 4 * rows, false},
                               {dh, hb, true}, {dw, wb, true}};
    if (overlapping(spans)) return fail(DBL_EINVAL, "dh and dw must not overlap another array");
    if (s.B == 0 && !dw) return ok();
    WsLayout L;
    if (dbl_status st = check_ws(DBL_OP_HEAD_NLL_BACKWARD, s, ws, ws_bytes, &L)) return st;
    char* const base = static_cast<char*>(ws);
    dbl::NllArgs a = nll_args(s, dt, h, w, x, base, L);
    a.nll = const_cast<float*>(nll);
    a.lse = const_cast<float*>(lse);
    a.g = g;
    a.dh = dh;
    a.dw = dw;
    a.hs = dw ? base + L.off[4] : nullptr;
    a.grad = base + L.off[5];
    a.part = reinterpret_cast<float*>(base + L.off[6]);
    const int64_t M = s.B * s.K * s.R;
    a.piece = dbl::nll_piece(M, s.V, static_cast<int>(e));
    const int64_t ids = a.piece < s.V ? a.piece : s.V;
    a.splits = a.bf16 ? dbl::grad_splits(s.d, M, ids) : dbl::grad_splits_f32(s.d, M, ids);
    a.dw_part = reinterpret_cast<float*>(base + L.off[7]);
    a.dw_splits = dbl::weight_splits(a.bf16, s.d, ids, M);
    return hip_status(dbl::launch_nll_backward(a, static_cast<hipStream_t>(stream)),
                      "head nll backward launch");
  });
}

dbl_status dbl_expand_branches_backward(dbl_shape s, const void* h, const void* W,
                                        const void* dout, void* dh, void* dW, void* dc, void* ws,
                                        size_t ws_bytes, void* stream) {
  return guarded([&]() -> dbl_status {
    if (s.B < 0 || s.K < 1 || s.K > (int64_t(1) << 20) || s.R < 1 || s.R > dbl::kMaxR)
      return fail(DBL_ESHAPE, "need B >= 0, 1 <= K <= 2^20 and 1 <= R <= 64");
    if (s.d < 32 || s.d % 32 != 0 || s.d > (int64_t(1) << 20) || s.R * s.d > (int64_t(1) << 23))
      return fail(DBL_ESHAPE, "expander needs d % 32 == 0, 32 <= d <= 2^20 and R*d <= 2^23");
    if (static_cast<double>(s.B) * s.K > static_cast<double>(dbl::kMaxTrainRows))
      return fail(DBL_ESHAPE, "B*K must be < 2^24");
    if (!W || (s.B > 0 && (!h || !dout))) return fail(DBL_EINVAL, "NULL input pointer");
    if (s.B > 0 && !dh && !dW && !dc) return fail(DBL_EINVAL, "no output");
    if (dbl_status st = check_aligned({{h, "h"}, {W, "W"}, {dout, "dout"}, {dh, "dh"}, {dW, "dW"},
                                       {dc, "dc"}}))
      return st;
    const size_t rows = static_cast<size_t>(s.B) * s.K, n = static_cast<size_t>(s.R) * s.d;
    std::vector<Span> spans = {{h, 2 * rows * s.d, false}, {W, 2 * n * s.d, false},
                               {dout, 2 * rows * n, false}, {dh, 2 * rows * s.d, true},
                               {dW, 2 * n * s.d, true}, {dc, 2 * n, true}};
    if (overlapping(spans)) return fail(DBL_EINVAL, "an output overlaps another array");
    dbl::ExpandBackwardArgs a{};
    if ((dh || dW) && s.B > 0) {
      WsLayout L;
      dbl_shape sv = s;
      sv.V = 1;
      if (dbl_status st = check_ws(DBL_OP_EXPAND_BACKWARD, sv, ws, ws_bytes, &L)) return st;
      a.part = reinterpret_cast<float*>(static_cast<char*>(ws) + L.off[0]);
      a.dW_part = reinterpret_cast<float*>(static_cast<char*>(ws) + L.off[1]);
      a.dh = dh;
    }
    a.P = s.B * s.K;
    a.R = s.R;
    a.d = static_cast<int>(s.d);
    a.h = h;
    a.W = W;
    a.dout = dout;
    a.dW = dW;
    a.dc = dc;
    a.splits = dbl::grad_splits(s.d, a.P, s.R * s.d);
    a.dW_splits = dbl::weight_splits(true, s.d, s.R * s.d, a.P);
    return hip_status(dbl::launch_expand_backward(a, static_cast<hipStream_t>(stream)),
                      "expander backward launch");
  });
}

dbl_status dbl_grad_norm(int64_t n, const void* const* grads, const int64_t* numel,
                         const int32_t* dt, float* norm, void* ws, size_t ws_bytes, void* stream) {
  return guarded([&]() -> dbl_status {
    std::vector<dbl::GradTensor> t;
    if (dbl_status st = check_tensors(n, grads, numel, dt, nullptr, false, &t)) return st;
    if (!norm || reinterpret_cast<uintptr_t>(norm) % 4 != 0)
      return fail(DBL_EINVAL, "norm is NULL or misaligned");
    const uintptr_t to = reinterpret_cast<uintptr_t>(norm);
    for (const dbl::GradTensor& g : t) {
      const uintptr_t at = reinterpret_cast<uintptr_t>(g.g);
      if (g.n > 0 && to + 4 > at && to < at + static_cast<uintptr_t>(g.n) * (g.bf16 ? 2 : 4))
        return fail(DBL_EINVAL, "norm overlaps a tensor");
    }
    WsLayout L;
    if (dbl_status st = check_ws(DBL_OP_GRAD_NORM, dbl_shape{n, 1, 1, 1, 1}, ws, ws_bytes, &L))
      return st;
    return hip_status(dbl::launch_grad_norm(t.data(), n, static_cast<double*>(ws), norm,
                                            static_cast<hipStream_t>(stream)),
                      "gradient norm launch");
  });
}

dbl_status dbl_clip_grads(int64_t n, const void* const* grads, void* const* out,
                          const int64_t* numel, const int32_t* dt, const float* norm,
                          float max_norm, void* stream) {
  return guarded([&]() -> dbl_status {
    std::vector<dbl::GradTensor> t;
    if (dbl_status st = check_tensors(n, grads, numel, dt, out, true, &t)) return st;
    if (!norm || reinterpret_cast<uintptr_t>(norm) % 4 != 0)
      return fail(DBL_EINVAL, "norm is NULL or misaligned");
    if (!(max_norm >= 0.0f)) return fail(DBL_EINVAL, "max_norm must be >= 0");
    std::vector<Span> spans;
    spans.reserve(2 * t.size() + 1);
    spans.emplace_back(norm, 4, false);
    for (const dbl::GradTensor& g : t) {
      const size_t bytes = static_cast<size_t>(g.n) * (g.bf16 ? 2 : 4);
      if (g.n == 0) continue;
      spans.emplace_back(g.out, bytes, true);
      if (g.out != g.g) spans.emplace_back(g.g, bytes, false);
    }
    if (overlapping(spans)) return fail(DBL_EINVAL, "tensors overlap");
    return hip_status(dbl::launch_clip_grads(t.data(), n, norm, max_norm,
                                             static_cast<hipStream_t>(stream)),
                      "gradient clipping launch");
  });
}

}  // extern "C"
