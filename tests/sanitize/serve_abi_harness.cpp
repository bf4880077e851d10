// Host-only harness for the low-precision serving operators' validation layer (csrc/abi_serve.hip beside
// csrc/abi.hip), built under AddressSanitizer and UndefinedBehaviorSanitizer by
// tests/test_serve_abi_sanitized.py. The kernel launchers are stubs that record their arguments, so no
// GPU is touched: what valid calls hand over, what is refused, and shapes whose sizes do not fit 64 bits.
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include <cmath>

#include "../../include/dblast.h"
#include "../../paper_2608_05448_amd/csrc/kernels.hpp"

namespace {
int g_launches = 0, g_fail = 0;
hipError_t g_result = hipSuccess;
dbl::MxQuantArgs g_quant;
dbl::MxNormArgs g_norm;
dbl::MxProductArgs g_product;
dbl::DrawArgs g_draw;

void check(bool ok, const char* what, int line) {
  if (!ok) {
    ++g_fail;
    fprintf(stderr, "FAILED line %d: %s (last error: %s)\n", line, what, dbl_last_error());
  }
}
#define CHECK(x) check((x), #x, __LINE__)

void* P(uintptr_t a) { return reinterpret_cast<void*>(a); }
float* F(uintptr_t a) { return reinterpret_cast<float*>(a); }
int32_t* I(uintptr_t a) { return reinterpret_cast<int32_t*>(a); }
uint8_t* U(uintptr_t a) { return reinterpret_cast<uint8_t*>(a); }
uint32_t* W(uintptr_t a) { return reinterpret_cast<uint32_t*>(a); }
}  // namespace

namespace dbl {
hipError_t launch_head(const HeadArgs&, hipStream_t) { return g_result; }
hipError_t launch_sample(const SampleArgs&, hipStream_t) { return g_result; }
hipError_t launch_verify(const VerifyArgs&, hipStream_t) { return g_result; }
hipError_t launch_sample_greedy(const GreedyArgs&, hipStream_t) { return g_result; }
hipError_t launch_verify_greedy(const GreedyArgs&, hipStream_t) { return g_result; }
hipError_t launch_objective(const ObjectiveArgs&, hipStream_t) { return g_result; }
hipError_t launch_expand(const ExpandArgs&, hipStream_t) { return g_result; }
hipError_t launch_prior_head(const PriorHeadArgs&, hipStream_t) { return g_result; }
hipError_t launch_filter(const FilterArgs&, hipStream_t) { return g_result; }
hipError_t launch_determinism(const DeterminismArgs&, hipStream_t) { return g_result; }
hipError_t launch_read_probe(const void*, int64_t, float*, int64_t, hipStream_t) { return g_result; }
hipError_t launch_mx_quantize(const MxQuantArgs& a, hipStream_t) { ++g_launches; g_quant = a; return g_result; }
hipError_t launch_mx_dequantize(const MxQuantArgs& a, hipStream_t) { ++g_launches; g_quant = a; return g_result; }
hipError_t launch_mx_norm(const MxNormArgs& a, hipStream_t) { ++g_launches; g_norm = a; return g_result; }
hipError_t launch_mx_product(const MxProductArgs& a, hipStream_t) { ++g_launches; g_product = a; return g_result; }
hipError_t launch_draw(const DrawArgs& a, hipStream_t) { ++g_launches; g_draw = a; return g_result; }
}  // namespace dbl

int main(int argc, char** argv) {
  if (argc > 1 && strcmp(argv[1], "--plant-overflow") == 0) {
    // Shows that the sanitizer is active: one read past a heap array.
    volatile int* v = new int[4];
    const int x = v[argc + 2];
    delete[] v;
    return x == 12345 ? 3 : 2;
  }
  // Fake, aligned device addresses 64 GB apart (never dereferenced).
  auto a = [&](int i) { return uintptr_t(1) << 44 | static_cast<uintptr_t>(i) << 36; };
  constexpr int64_t kMost = (int64_t(1) << 40) - 1, kWide = int64_t(1) << 20;

  // --- rows: what is handed over, and the largest sizes (2^60 values) ------------------------
  for (int bits : {4, 8}) {
    CHECK(dbl_mx_quantize(17, 1000, DBL_BF16, P(a(0)), bits, P(a(1)), U(a(2)), nullptr) == DBL_OK);
    CHECK(g_quant.M == 17 && g_quant.d == 1000 && g_quant.bits == bits && g_quant.bf16);
    CHECK(dbl_mx_dequantize(17, 1000, bits, P(a(1)), U(a(2)), DBL_F32, P(a(0)), nullptr) == DBL_OK);
    CHECK(g_quant.x == P(a(0)) && !g_quant.bf16);
    int before = g_launches;
    CHECK(dbl_mx_quantize(kMost, kWide, DBL_F32, P(a(0)), bits, P(a(1)), U(a(2)), nullptr) == DBL_EINVAL);
    CHECK(dbl_mx_quantize(kMost + 1, 1, DBL_F32, P(a(0)), bits, P(a(1)), U(a(2)), nullptr) == DBL_ESHAPE);
    CHECK(dbl_mx_quantize(INT64_MAX, INT64_MAX, DBL_F32, P(a(0)), bits, P(a(1)), U(a(2)), nullptr) == DBL_ESHAPE);
    CHECK(dbl_mx_quantize(INT64_MIN, 1, DBL_F32, P(a(0)), bits, P(a(1)), U(a(2)), nullptr) == DBL_ESHAPE);
    CHECK(dbl_add_rmsnorm_mx(kMost, kWide, DBL_F32, P(a(0)), nullptr, P(a(1)), 0.0f, nullptr, bits, P(a(2)),
                             U(a(3)), nullptr, nullptr) == DBL_EINVAL);
    CHECK(g_launches == before);
  }
  // In place is the same rows exactly; an absent residual, sum or y is no overlap.
  CHECK(dbl_add_rmsnorm_mx(3, 64, DBL_BF16, P(a(0)), P(a(1)), P(a(2)), 1e-6f, P(a(0)), 8, P(a(3)), U(a(4)),
                           nullptr, nullptr) == DBL_OK);
  CHECK(g_norm.sum == P(a(0)) && g_norm.residual == P(a(1)) && !g_norm.y && g_norm.q.d == 64);
  CHECK(dbl_add_rmsnorm_mx(3, 64, DBL_BF16, P(a(0)), nullptr, P(a(2)), 1e-6f, nullptr, 8, P(a(3)), U(a(4)),
                           P(a(5)), nullptr) == DBL_OK);
  CHECK(!g_norm.sum && !g_norm.residual && g_norm.y == P(a(5)));

  // --- products ------------------------------------------------------------------------------
  CHECK(dbl_mx_matmul(17, 151936, 2560, 8, P(a(0)), U(a(1)), P(a(2)), U(a(3)), DBL_F32, P(a(4)), nullptr) ==
        DBL_OK);
  CHECK(g_product.dp == 2560 && g_product.logits == P(a(4)) && !g_product.tls && !g_product.amax_keys);
  const dbl_shape s{2, 3, 4, 1000, 50257};
  const size_t hw = dbl_workspace_bytes(DBL_OP_MX_HEAD, s);
  auto head = [&](dbl_shape q, int bits, int32_t* argmax, void* ws, size_t n) {
    return dbl_mx_head_logprobs(q, bits, P(a(0)), U(a(1)), P(a(2)), U(a(3)), F(a(4)), F(a(5)), F(a(6)), argmax, ws,
                                n, nullptr);
  };
  CHECK(head(s, 8, nullptr, nullptr, 0) == DBL_OK && g_product.M == 24 && g_product.dp == 1024);
  CHECK(head(s, 8, I(a(7)), P(a(8)), hw) == DBL_OK && g_product.amax_keys == P(a(8)));
  int before = g_launches;
  CHECK(head(s, 8, I(a(7)), P(a(8)), hw - 1) == DBL_EWORKSPACE);
  CHECK(head(s, 8, I(a(7)), P(a(8) + 16), hw) == DBL_EWORKSPACE);
  CHECK(head(s, 8, I(a(7)), nullptr, hw) == DBL_EWORKSPACE);
  CHECK(head(s, 5, nullptr, nullptr, 0) == DBL_EINVAL);
  // More rows than any array holds: their bytes do not fit 64 bits.
  CHECK(head({int64_t(1) << 61, 1, 1, 1 << 20, 1}, 8, nullptr, nullptr, 0) == DBL_ESHAPE);
  CHECK(head({int64_t(1) << 61, 1, 1, 64, 1}, 8, I(a(7)), nullptr, 0) == DBL_ESHAPE);
  CHECK(head({int64_t(1) << 40, 1, 1, 64, 1}, 8, nullptr, nullptr, 0) == DBL_ESHAPE);
  CHECK(dbl_mx_matmul(kMost, (1 << 24) - 1, 1, 8, P(a(0)), U(a(1)), P(a(2)), U(a(3)), DBL_F32, P(a(4)), nullptr) ==
        DBL_ESHAPE);
  CHECK(g_launches == before);

  // --- draw ----------------------------------------------------------------------------------
  const size_t dw = dbl_workspace_bytes(DBL_OP_SAMPLE_LOGITS, dbl_shape{17, 1, 1, 1, 151936});
  dbl_sampling p{};
  p.temperature = 1.0f;
  p.top_p = 1.0f;
  auto draw = [&](int64_t N, int64_t V, dbl_sampling q, void* ws, size_t n) {
    return dbl_sample_logits(N, V, DBL_F32, P(a(0)), W(a(1)), q, I(a(2)), F(a(3)), ws, n, nullptr);
  };
  CHECK(draw(17, 151936, p, P(a(9)), dw) == DBL_OK && g_draw.N == 17 && g_draw.ws == P(a(9)));
  dbl_sampling rows = p;  // numbers beside arrays are not looked at
  rows.temperature = rows.top_p = rows.min_p = std::nanf("");
  rows.top_k = -1;
  rows.temperatures = F(a(4) + 4);
  rows.top_ps = F(a(5));
  rows.min_ps = F(a(6));
  rows.top_ks = I(a(7));
  CHECK(draw(17, 151936, rows, P(a(9)), dw) == DBL_OK && g_draw.temperatures == F(a(4) + 4));
  before = g_launches;
  rows.temperatures = F(a(4) + 2);
  CHECK(draw(17, 151936, rows, P(a(9)), dw) == DBL_EINVAL);
  rows.temperatures = reinterpret_cast<const float*>(I(a(2)));  // an output over a parameter
  CHECK(draw(17, 151936, rows, P(a(9)), dw) == DBL_EINVAL);
  CHECK(draw(17, 151936, p, P(a(9)), dw - 1) == DBL_EWORKSPACE);
  for (int64_t N : {int64_t(1) << 47, int64_t(1) << 61}) {
    CHECK(dbl_workspace_bytes(DBL_OP_SAMPLE_LOGITS, dbl_shape{N, 1, 1, 1, 1}) == SIZE_MAX);
    CHECK(draw(N, 1, p, P(a(9)), size_t(1) << 60) != DBL_OK);
  }
  CHECK(g_launches == before);

  // --- a launcher's error comes back; no rows launch nothing ----------------------------------
  g_result = hipErrorInvalidConfiguration;
  CHECK(draw(17, 151936, p, P(a(9)), dw) == DBL_EHIP && head(s, 8, nullptr, nullptr, 0) == DBL_EHIP);
  before = g_launches;
  CHECK(draw(0, 10, p, nullptr, 0) == DBL_OK && head({0, 1, 1, 64, 10}, 8, nullptr, nullptr, 0) == DBL_OK);
  CHECK(g_launches == before);

  if (g_fail) {
    fprintf(stderr, "%d checks failed\n", g_fail);
    return 1;
  }
  printf("all checks passed\n");
  return 0;
}
