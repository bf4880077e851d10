// Argument checks, workspace layout and error text shared by the C ABI's translation units. Internal.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <initializer_list>
#include <string>
#include <utility>
#include <vector>

#include "../../include/dblast.h"
#include "kernels.hpp"

namespace dbl_abi {

inline thread_local std::string g_last_error;

inline dbl_status fail(dbl_status s, const std::string& msg) {
  g_last_error = std::string(dbl_status_string(s)) + ": " + msg;
  return s;
}

inline dbl_status ok() { return DBL_OK; }

constexpr size_t kAlign = 256;
inline size_t align_up(size_t n) { return (n + kAlign - 1) / kAlign * kAlign; }

inline int64_t ntiles(int64_t V) { return (V + DBL_VTILE - 1) / DBL_VTILE; }

// Shape checks shared by every call.
inline dbl_status check_shape(const dbl_shape& s, bool need_d) {
  if (s.B < 0) return fail(DBL_ESHAPE, "B must be >= 0");
  if (s.K < 1 || s.R < 1 || s.V < 1) return fail(DBL_ESHAPE, "K, R and V must be >= 1");
  if (s.R > dbl::kMaxR) return fail(DBL_ESHAPE, "R must be <= 64");
  if (s.V >= (int64_t(1) << 24)) return fail(DBL_ESHAPE, "V must be < 2^24");
  if (s.K > (int64_t(1) << 20)) return fail(DBL_ESHAPE, "K must be <= 2^20");
  // The bf16 head kernels address a tile's operand rows with 32-bit byte offsets (up to 512 d).
  if (need_d && (s.d < 1 || s.d > (int64_t(1) << 20)))
    return fail(DBL_ESHAPE, "d must be in [1, 2^20]");
  const double rows = static_cast<double>(s.B) * s.K * s.R;
  if (rows * static_cast<double>(s.V) >= 4.0e18) return fail(DBL_ESHAPE, "B*K*R*V too large");
  return ok();
}

// Every array is read and written with 16-byte vector accesses, so each must be 16-byte
// aligned. NULL (an optional array that is not passed) is not checked here.
inline dbl_status check_aligned(std::initializer_list<std::pair<const void*, const char*>> arrays) {
  for (const auto& a : arrays)
    if (reinterpret_cast<uintptr_t>(a.first) % 16 != 0)
      return fail(DBL_EINVAL, std::string(a.second) + " is not 16-byte aligned");
  return ok();
}

struct WsLayout {
  size_t total = 0;
  size_t off[12] = {};
};

inline WsLayout layout(int op, const dbl_shape& s) {
  WsLayout L;
  const size_t B = static_cast<size_t>(s.B), K = static_cast<size_t>(s.K);
  const size_t R = static_cast<size_t>(s.R);
  const size_t nT = static_cast<size_t>(ntiles(s.V));
  const size_t nchunk = static_cast<size_t>(dbl::n_chunks(static_cast<int>(nT)));
  size_t sizes[12] = {};
  int n = 0;
  switch (op) {
    case DBL_OP_HEAD:  // argmax keys, used only when argmax is requested
    case DBL_OP_MX_HEAD:
      sizes[0] = B * K * R * sizeof(uint64_t);
      n = 1;
      break;
    case DBL_OP_SAMPLE_GREEDY:
      n = 0;
      break;
    case DBL_OP_VERIFY_GREEDY:
      sizes[0] = B * K * R * sizeof(double);
      sizes[1] = B * nT * sizeof(uint64_t);
      sizes[2] = B * nT * sizeof(uint64_t);
      n = 3;
      break;
    case DBL_OP_EXPECTED_LEN_GREEDY:
      sizes[0] = B * K * R * sizeof(double);
      n = 1;
      break;
    case DBL_OP_SAMPLE:
      n = 0;
      break;
    case DBL_OP_VERIFY:
      sizes[0] = B * K * R * sizeof(double);
      sizes[1] = B * K * nchunk * sizeof(float);
      sizes[2] = B * nT * sizeof(uint64_t);
      sizes[3] = B * nT * sizeof(uint64_t);
      n = 4;
      break;
    case DBL_OP_EXPECTED_LEN:
      sizes[0] = B * K * R * sizeof(double);
      sizes[1] = B * K * nchunk * sizeof(float);
      n = 2;
      break;
    case DBL_OP_TARGET:  // rows B*K: segment results, lists or bins, and the cut
      sizes[0] = B * K * dbl::kFilterRowBytes;
      sizes[1] = B * K * sizeof(dbl::FilterCut);
      n = 2;
      break;
    case DBL_OP_HEAD_NLL:           // rows that count, and what the head leaves of them
    case DBL_OP_HEAD_NLL_BACKWARD:  // the same, a piece of the logits' gradient, the parts of dh
      if (s.B * s.K * s.R > dbl::kMaxTrainRows) {
        L.total = SIZE_MAX;
        return L;
      }
      sizes[0] = sizeof(int32_t);
      sizes[1] = B * K * sizeof(int32_t);
      sizes[2] = B * K * R * sizeof(dbl::TrainRow);
      sizes[3] = B * K * R * static_cast<size_t>(s.d) * sizeof(float);
      n = 6;
      if (op == DBL_OP_HEAD_NLL) {
        sizes[4] = B * K * R * dbl::nll_tiles(false, s.V) * sizeof(float);
        sizes[5] = B * K * R * sizeof(float);
      } else {
        const int64_t M = s.B * s.K * s.R;
        sizes[4] = sizes[3];
        for (int elem = 2; elem <= 4; elem += 2) {  // the call's type is not known here
          const int64_t piece = dbl::nll_piece(M, s.V, elem);
          const size_t grad = static_cast<size_t>(M) * piece * elem;
          const int64_t ids = piece < s.V ? piece : s.V;
          const size_t part =
              sizes[3] * (elem == 2 ? dbl::grad_splits(s.d, M, ids) : dbl::grad_splits_f32(s.d, M, ids));
          const int splits = dbl::weight_splits(elem == 2, s.d, ids, M);
          const size_t dw_part = splits > 1 ? static_cast<size_t>(splits) * ids * s.d * sizeof(float) : 0;
          sizes[5] = sizes[5] > grad ? sizes[5] : grad;
          sizes[6] = sizes[6] > part ? sizes[6] : part;
          sizes[7] = sizes[7] > dw_part ? sizes[7] : dw_part;
        }
        n = 8;
      }
      break;
    case DBL_OP_EXPAND_BACKWARD:  // the parts of the trunk gradient and of the weight's
      if (s.B * s.K > dbl::kMaxTrainRows) {
        L.total = SIZE_MAX;
        return L;
      }
      sizes[0] = B * K * static_cast<size_t>(s.d) * sizeof(float) *
                 dbl::grad_splits(s.d, s.B * s.K, s.R * s.d);
      if (const int splits = dbl::weight_splits(true, s.d, s.R * s.d, s.B * s.K); splits > 1)
        sizes[1] = static_cast<size_t>(splits) * s.R * s.d * s.d * sizeof(float);
      n = 2;
      break;
    case DBL_OP_GRAD_NORM:  // B tensors
      if (s.B > dbl::kMaxTensors) {
        L.total = SIZE_MAX;
        return L;
      }
      sizes[0] = static_cast<size_t>(dbl::norm_parts(s.B)) * sizeof(double);
      n = 1;
      break;
    case DBL_OP_SAMPLE_LOGITS: {  // rows B*K
      const size_t row = dbl::draw_row_bytes(s.V);
      if (B * K > SIZE_MAX / 2 / row) {
        L.total = SIZE_MAX;
        return L;
      }
      sizes[0] = B * K * row;
      n = 1;
      break;
    }
    default:
      L.total = SIZE_MAX;
      return L;
  }
  size_t at = 0;
  for (int i = 0; i < n; ++i) {
    L.off[i] = at;
    at += align_up(sizes[i]);
  }
  L.total = at;
  return L;
}

inline dbl_status check_ws(int op, const dbl_shape& s, void* ws, size_t ws_bytes, WsLayout* out) {
  *out = layout(op, s);
  if (out->total == 0) return ok();
  if (ws == nullptr) return fail(DBL_EWORKSPACE, "workspace pointer is NULL");
  if (reinterpret_cast<uintptr_t>(ws) % kAlign != 0)
    return fail(DBL_EWORKSPACE, "workspace must be 256-byte aligned");
  if (ws_bytes < out->total)
    return fail(DBL_EWORKSPACE, "workspace has " + std::to_string(ws_bytes) + " bytes, needs " +
                                    std::to_string(out->total));
  return ok();
}

inline dbl_status hip_status(hipError_t e, const char* what) {
  if (e == hipSuccess) return ok();
  return fail(DBL_EHIP, std::string(what) + ": " + hipGetErrorString(e));
}

// A piece of memory that a call reads or writes.
struct Span {
  uintptr_t at, end;
  bool written;
  Span(const void* p, size_t bytes, bool w)
      : at(reinterpret_cast<uintptr_t>(p)), end(at + (p ? bytes : 0)), written(w) {}
};

// Whether a written piece overlaps another one (sorted by address, the pieces written so far reach as far
// as `written`, all as far as `any`).
inline bool overlapping(std::vector<Span>& s) {
  std::sort(s.begin(), s.end(), [](const Span& a, const Span& b) { return a.at < b.at; });
  uintptr_t any = 0, written = 0;
  for (const Span& x : s) {
    if (x.at == x.end) continue;
    if (x.at < (x.written ? any : written)) return true;
    any = std::max(any, x.end);
    if (x.written) written = std::max(written, x.end);
  }
  return false;
}

// No C++ exception (a host allocation that fails) crosses the C boundary.
template <class F>
dbl_status guarded(F f) noexcept {
  try {
    return f();
  } catch (...) {
    g_last_error.clear();
    return DBL_EHIP;
  }
}

}  // namespace dbl_abi
