// C ABI of the low-precision serving operators and the token draw (declared in include/dblast.h): argument
// validation, workspace layout and status mapping around their launchers.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <vector>

#include "abi_common.hpp"

using namespace dbl_abi;

namespace {

dbl_status check_rows(int64_t M, int64_t d, int bits) {
  if (M < 0 || M >= (int64_t(1) << 40)) return fail(DBL_ESHAPE, "need 0 <= M < 2^40 rows");
  if (d < 1 || d > (int64_t(1) << 20)) return fail(DBL_ESHAPE, "d must be in [1, 2^20]");
  if (bits != 4 && bits != 8) return fail(DBL_EINVAL, "bits must be 4 or 8");
  return ok();
}

dbl_status check_type(int dt) {
  return dt == DBL_BF16 || dt == DBL_F32 ? ok() : fail(DBL_EDTYPE, "dt must be DBL_BF16 or DBL_F32");
}

size_t elem(int dt) { return dt == DBL_BF16 ? 2 : 4; }
size_t code_bytes(int64_t M, int64_t d, int bits) {
  return static_cast<size_t>(M) * dbl::mx_row(d) / 8 * bits;
}
size_t scale_bytes(int64_t M, int64_t d) { return static_cast<size_t>(M) * dbl::mx_row(d) / dbl::kMxBlock; }

dbl_status check_apart(std::vector<Span> spans) {
  return overlapping(spans) ? fail(DBL_EINVAL, "an output overlaps another array") : ok();
}

dbl_status quantize(int64_t M, int64_t d, int dt, const void* x, int bits, const void* codes,
                    const uint8_t* scales, bool back, void* stream) {
  return guarded([&]() -> dbl_status {
    if (dbl_status st = check_rows(M, d, bits)) return st;
    if (dbl_status st = check_type(dt)) return st;
    if (M == 0) return ok();
    if (!x || !codes || !scales) return fail(DBL_EINVAL, "NULL pointer");
    if (dbl_status st = check_aligned({{x, back ? "out" : "x"}, {codes, "codes"}, {scales, "scales"}}))
      return st;
    if (dbl_status st = check_apart({{x, static_cast<size_t>(M) * d * elem(dt), back},
                                     {codes, code_bytes(M, d, bits), !back},
                                     {scales, scale_bytes(M, d), !back}}))
      return st;
    const dbl::MxQuantArgs a{M, static_cast<int>(d), bits, dt == DBL_BF16, x, const_cast<void*>(codes),
                             const_cast<uint8_t*>(scales)};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    return hip_status(back ? dbl::launch_mx_dequantize(a, s) : dbl::launch_mx_quantize(a, s),
                      back ? "dequantisation launch" : "quantisation launch");
  });
}

}  // namespace

extern "C" {

int64_t dbl_mx_row(int64_t d) { return d < 1 || d > INT64_MAX - 127 ? 0 : dbl::mx_row(d); }

dbl_status dbl_mx_quantize(int64_t M, int64_t d, int dt, const void* x, int bits, void* codes,
                           uint8_t* scales, void* stream) {
  return quantize(M, d, dt, x, bits, codes, scales, false, stream);
}

dbl_status dbl_mx_dequantize(int64_t M, int64_t d, int bits, const void* codes, const uint8_t* scales,
                             int dt, void* out, void* stream) {
  return quantize(M, d, dt, out, bits, codes, scales, true, stream);
}

dbl_status dbl_add_rmsnorm_mx(int64_t M, int64_t d, int dt, const void* x, const void* residual,
                              const void* weight, float eps, void* sum, int bits, void* codes,
                              uint8_t* scales, void* y, void* stream) {
  return guarded([&]() -> dbl_status {
    if (dbl_status st = check_rows(M, d, bits)) return st;
    if (dbl_status st = check_type(dt)) return st;
    if (!(eps >= 0.0f && eps < INFINITY)) return fail(DBL_EINVAL, "eps must be finite and >= 0");
    if (sum && !residual) return fail(DBL_EINVAL, "sum needs a residual");
    if (M == 0) return ok();
    if (!x || !weight || !codes || !scales) return fail(DBL_EINVAL, "NULL pointer");
    if (dbl_status st = check_aligned({{x, "x"}, {residual, "residual"}, {weight, "weight"}, {sum, "sum"},
                                       {codes, "codes"}, {scales, "scales"}, {y, "y"}}))
      return st;
    const size_t all = static_cast<size_t>(M) * d * elem(dt);
    std::vector<Span> spans = {{weight, static_cast<size_t>(d) * elem(dt), false},
                               {sum, all, true},
                               {codes, code_bytes(M, d, bits), true},
                               {scales, scale_bytes(M, d), true},
                               {y, all, true}};
    if (x != sum) spans.emplace_back(x, all, false);
    if (residual != sum) spans.emplace_back(residual, all, false);
    if (dbl_status st = check_apart(std::move(spans))) return st;
    const dbl::MxNormArgs a{{M, static_cast<int>(d), bits, dt == DBL_BF16, x, codes, scales},
                            residual, weight, eps, sum, y};
    return hip_status(dbl::launch_mx_norm(a, static_cast<hipStream_t>(stream)), "norm launch");
  });
}

dbl_status dbl_mx_matmul(int64_t M, int64_t V, int64_t d, int bits, const void* h, const uint8_t* hs,
                         const void* w, const uint8_t* ws, int dt, void* logits, void* stream) {
  return guarded([&]() -> dbl_status {
    if (dbl_status st = check_rows(M, d, bits)) return st;
    if (V < 1 || V >= (int64_t(1) << 24)) return fail(DBL_ESHAPE, "V must be in [1, 2^24)");
    if (static_cast<double>(M) * static_cast<double>(V) >= 4.0e18) return fail(DBL_ESHAPE, "M*V too large");
    if (dbl_status st = check_type(dt)) return st;
    if (M == 0) return ok();
    if (!h || !hs || !w || !ws || !logits) return fail(DBL_EINVAL, "NULL pointer");
    if (dbl_status st = check_aligned({{h, "h"}, {hs, "hs"}, {w, "w"}, {ws, "ws"}, {logits, "logits"}}))
      return st;
    if (dbl_status st = check_apart({{h, code_bytes(M, d, bits), false},
                                     {hs, scale_bytes(M, d), false},
                                     {w, code_bytes(V, d, 4), false},
                                     {ws, scale_bytes(V, d), false},
                                     {logits, static_cast<size_t>(M) * V * elem(dt), true}}))
      return st;
    dbl::MxProductArgs a{};
    a.M = M;
    a.V = V;
    a.dp = static_cast<int>(dbl::mx_row(d));
    a.bits = bits;
    a.h = h;
    a.hs = hs;
    a.w = w;
    a.ws = ws;
    a.logits = logits;
    a.bf16 = dt == DBL_BF16;
    return hip_status(dbl::launch_mx_product(a, static_cast<hipStream_t>(stream)), "product launch");
  });
}

dbl_status dbl_mx_head_logprobs(dbl_shape s, int bits, const void* h, const uint8_t* hs, const void* w,
                                const uint8_t* ws, float* tls, float* lmass, float* lse, int32_t* argmax,
                                void* ws_mem, size_t ws_bytes, void* stream) {
  return guarded([&]() -> dbl_status {
    if (dbl_status st = check_shape(s, true)) return st;
    if (dbl_status st = check_rows(s.B * s.K * s.R, s.d, bits)) return st;
    if (s.B == 0) return ok();
    if (!h || !hs || !w || !ws || !tls || !lmass || !lse) return fail(DBL_EINVAL, "NULL pointer");
    if (dbl_status st = check_aligned({{h, "h"}, {hs, "hs"}, {w, "w"}, {ws, "ws"}, {tls, "tls"},
                                       {lmass, "lmass"}, {lse, "lse"}, {argmax, "argmax"}}))
      return st;
    const int64_t M = s.B * s.K * s.R;
    const size_t m = static_cast<size_t>(M);
    if (dbl_status st = check_apart({{h, code_bytes(M, s.d, bits), false},
                                     {hs, scale_bytes(M, s.d), false},
                                     {w, code_bytes(s.V, s.d, 4), false},
                                     {ws, scale_bytes(s.V, s.d), false},
                                     {tls, 4 * m * s.V, true},
                                     {lmass, 4 * m * ntiles(s.V), true},
                                     {lse, 4 * m, true},
                                     {argmax, 4 * m, true}}))
      return st;
    dbl::MxProductArgs a{};
    if (argmax) {
      WsLayout L;
      if (dbl_status st = check_ws(DBL_OP_MX_HEAD, s, ws_mem, ws_bytes, &L)) return st;
      a.amax_keys = static_cast<uint64_t*>(ws_mem);
    }
    a.M = M;
    a.V = s.V;
    a.dp = static_cast<int>(dbl::mx_row(s.d));
    a.bits = bits;
    a.h = h;
    a.hs = hs;
    a.w = w;
    a.ws = ws;
    a.tls = tls;
    a.lmass = lmass;
    a.lse = lse;
    a.argmax = argmax;
    return hip_status(dbl::launch_mx_product(a, static_cast<hipStream_t>(stream)), "head launch");
  });
}

dbl_status dbl_sample_logits(int64_t N, int64_t V, int dt, const void* logits, const uint32_t* words,
                             dbl_sampling p, int32_t* token, float* logprob, void* ws, size_t ws_bytes,
                             void* stream) {
  return guarded([&]() -> dbl_status {
    const dbl_shape s{N, 1, 1, 1, V};
    if (dbl_status st = check_shape(s, false)) return st;
    if (dbl_status st = check_type(dt)) return st;
    if (!p.temperatures && !(p.temperature >= 0.0f && p.temperature < INFINITY))
      return fail(DBL_EINVAL, "temperature must be finite and >= 0");
    if (!p.top_ks && p.top_k < 0) return fail(DBL_EINVAL, "top_k must be >= 0");
    if (!p.top_ps && !(p.top_p > 0.0f && p.top_p <= 1.0f))
      return fail(DBL_EINVAL, "top_p must be in (0, 1]");
    if (!p.min_ps && !(p.min_p >= 0.0f && p.min_p <= 1.0f))
      return fail(DBL_EINVAL, "min_p must be in [0, 1]");
    if (N == 0) return ok();
    if (!logits || !words || !token || !logprob) return fail(DBL_EINVAL, "NULL pointer");
    if (dbl_status st = check_aligned({{logits, "logits"}})) return st;
    const void* rows[] = {words, p.temperatures, p.top_ps, p.min_ps, p.top_ks, token, logprob};
    for (const void* r : rows)
      if (reinterpret_cast<uintptr_t>(r) % 4 != 0)
        return fail(DBL_EINVAL, "an array of a value per row is not aligned to its elements");
    const size_t n = 4 * static_cast<size_t>(N);
    if (dbl_status st = check_apart({{logits, static_cast<size_t>(N) * V * elem(dt), false},
                                     {words, n, false},
                                     {p.temperatures, n, false},
                                     {p.top_ps, n, false},
                                     {p.min_ps, n, false},
                                     {p.top_ks, n, false},
                                     {token, n, true},
                                     {logprob, n, true}}))
      return st;
    WsLayout L;
    if (dbl_status st = check_ws(DBL_OP_SAMPLE_LOGITS, s, ws, ws_bytes, &L)) return st;
    dbl::DrawArgs a{};
    a.N = N;
    a.V = V;
    a.bf16 = dt == DBL_BF16;
    a.logits = logits;
    a.words = words;
    a.temperature = p.temperature;
    a.top_p = p.top_p;
    a.min_p = p.min_p;
    a.top_k = p.top_k;
    a.temperatures = p.temperatures;
    a.top_ps = p.top_ps;
    a.min_ps = p.min_ps;
    a.top_ks = p.top_ks;
    a.token = token;
    a.logprob = logprob;
    a.ws = static_cast<char*>(ws);
    return hip_status(dbl::launch_draw(a, static_cast<hipStream_t>(stream)), "draw launch");
  });
}

}  // extern "C"
