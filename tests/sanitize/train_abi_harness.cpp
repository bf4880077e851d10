// Host-only harness for the training operators' validation layer (csrc/abi_train.hip beside
// csrc/abi.hip), built under AddressSanitizer and UndefinedBehaviorSanitizer by
// tests/test_train_abi_sanitized.py. The kernel launchers are stubs that record their arguments, so no
// GPU is touched: valid and invalid calls, the workspaces' carve-up, tensors that overlap.
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include <algorithm>
#include <cmath>
#include <limits>
#include <vector>

#include "../../include/dblast.h"
#include "../../paper_2608_05448_amd/csrc/kernels.hpp"

namespace {
int g_launches = 0, g_fail = 0;
hipError_t g_result = hipSuccess;
dbl::NllArgs g_nll;
dbl::ExpandBackwardArgs g_expand;
std::vector<dbl::GradTensor> g_tensors;

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
hipError_t launch_nll(const NllArgs& a, hipStream_t) { ++g_launches; g_nll = a; return g_result; }
hipError_t launch_nll_backward(const NllArgs& a, hipStream_t) { ++g_launches; g_nll = a; return g_result; }
hipError_t launch_expand_backward(const ExpandBackwardArgs& a, hipStream_t) {
  ++g_launches;
  g_expand = a;
  return g_result;
}
hipError_t launch_grad_norm(const GradTensor* t, int64_t n, double*, float*, hipStream_t) {
  ++g_launches;
  g_tensors.assign(t, t + n);
  return g_result;
}
hipError_t launch_clip_grads(const GradTensor* t, int64_t n, const float*, float, hipStream_t) {
  ++g_launches;
  g_tensors.assign(t, t + n);
  return g_result;
}
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
  const size_t bad = SIZE_MAX;

  // --- head: the workspaces' parts lie in order, apart and inside ---------------------------
  for (dbl_shape s : {dbl_shape{2, 4, 3, 64, 1000}, dbl_shape{16, 16, 8, 4096, 151936},
                      dbl_shape{1, 1, 1, 8, 1}, dbl_shape{512, 16, 4, 256, 151936}}) {
    const size_t M = static_cast<size_t>(s.B) * s.K * s.R;
    for (int dt : {DBL_BF16, DBL_F32}) {
      const size_t fws = dbl_workspace_bytes(DBL_OP_HEAD_NLL, s);
      const size_t bws = dbl_workspace_bytes(DBL_OP_HEAD_NLL_BACKWARD, s);
      CHECK(fws != bad && bws != bad && fws % 256 == 0 && bws % 256 == 0);
      const size_t e = dt == DBL_BF16 ? 2 : 4;
      auto apart = [&](std::vector<std::pair<const void*, size_t>> parts, size_t total) {
        uintptr_t at = a(20);
        for (const auto& p : parts) {
          const uintptr_t q = reinterpret_cast<uintptr_t>(p.first);
          CHECK(q >= at && q % 256 == 0);
          at = q + p.second;
        }
        CHECK(at <= a(20) + total);
      };
      CHECK(dbl_head_nll(s, dt, P(a(0)), P(a(1)), I(a(2)), F(a(3)), F(a(4)), P(a(20)), fws,
                         nullptr) == DBL_OK);
      CHECK(g_nll.P == s.B * s.K && g_nll.R == s.R && g_nll.bf16 == (dt == DBL_BF16) && !g_nll.g);
      apart({{g_nll.count, 4},
             {g_nll.inv, 4 * M / s.R},
             {g_nll.rows, 16 * M},
             {g_nll.hc, e * M * s.d},
             {g_nll.lmass, 4 * M * dbl::nll_tiles(g_nll.bf16, s.V)},
             {g_nll.tgt, 4 * M}}, fws);
      CHECK(dbl_head_nll_backward(s, dt, P(a(0)), P(a(1)), I(a(2)), F(a(3)), F(a(4)), F(a(5)),
                                  P(a(6)), P(a(7)), P(a(20)), bws, nullptr) == DBL_OK);
      CHECK(g_nll.piece % 256 == 0 && g_nll.piece > 0 && g_nll.splits >= 1 && g_nll.hs);
      apart({{g_nll.count, 4},
             {g_nll.inv, 4 * M / s.R},
             {g_nll.rows, 16 * M},
             {g_nll.hc, e * M * s.d},
             {g_nll.hs, e * M * s.d},
             {g_nll.grad, e * M * g_nll.piece},
             {g_nll.part, 4 * M * s.d * g_nll.splits},
             {g_nll.dw_part, g_nll.dw_splits > 1 ? 4 * std::min<size_t>(g_nll.piece, s.V) * s.d *
                                                       g_nll.dw_splits : 0}}, bws);
      CHECK(g_nll.dw_splits >= 1);
      CHECK(dbl_head_nll_backward(s, dt, P(a(0)), P(a(1)), I(a(2)), F(a(3)), F(a(4)), F(a(5)),
                                  P(a(6)), nullptr, P(a(20)), bws, nullptr) == DBL_OK);
      CHECK(!g_nll.dw && !g_nll.hs);
      int before = g_launches;
      CHECK(dbl_head_nll(s, dt, P(a(0)), P(a(1)), I(a(2)), F(a(3)), F(a(4)), P(a(20)), fws - 1,
                         nullptr) == DBL_EWORKSPACE);
      CHECK(dbl_head_nll_backward(s, dt, P(a(0)), P(a(1)), I(a(2)), F(a(3)), F(a(4)), F(a(5)),
                                  P(a(6)), P(a(7)), P(a(20)), bws - 1, nullptr) == DBL_EWORKSPACE);
      CHECK(dbl_head_nll_backward(s, dt, P(a(0)), P(a(1)), I(a(2)), F(a(3)), F(a(4)), F(a(5)),
                                  P(a(6)), P(a(7)), P(a(20) + 16), bws, nullptr) == DBL_EWORKSPACE);
      // outputs over inputs or each other
      CHECK(dbl_head_nll_backward(s, dt, P(a(0)), P(a(1)), I(a(2)), F(a(3)), F(a(4)), F(a(5)),
                                  P(a(0)), P(a(7)), P(a(20)), bws, nullptr) == DBL_EINVAL);
      CHECK(dbl_head_nll_backward(s, dt, P(a(0)), P(a(1)), I(a(2)), F(a(3)), F(a(4)), F(a(5)),
                                  P(a(6)), P(a(6)), P(a(20)), bws, nullptr) == DBL_EINVAL);
      CHECK(g_launches == before);
    }
  }
  dbl_shape hs{2, 4, 3, 64, 1000};
  const size_t fws = dbl_workspace_bytes(DBL_OP_HEAD_NLL, hs);
  const size_t bws = dbl_workspace_bytes(DBL_OP_HEAD_NLL_BACKWARD, hs);
  int before = g_launches;
  for (int i = 0; i < 5; ++i) {
    void* p[5] = {P(a(0)), P(a(1)), P(a(2)), P(a(3)), P(a(4))};
    for (uintptr_t off : {uintptr_t(0), uintptr_t(8)}) {
      p[i] = off ? P(a(i) + off) : nullptr;
      CHECK(dbl_head_nll(hs, DBL_BF16, p[0], p[1], static_cast<int32_t*>(p[2]),
                         static_cast<float*>(p[3]), static_cast<float*>(p[4]), P(a(20)), fws,
                         nullptr) == DBL_EINVAL);
    }
  }
  CHECK(dbl_head_nll(hs, DBL_BF16, P(a(0)), P(a(1)), I(a(2)), F(a(3)), F(a(3)), P(a(20)), fws, nullptr) ==
        DBL_EINVAL);
  CHECK(dbl_head_nll(hs, DBL_BF16, P(a(0)), P(a(1)), I(a(2)), F(a(3)), F(a(1) + 16), P(a(20)), fws,
                     nullptr) == DBL_EINVAL);
  CHECK(dbl_head_nll(dbl_shape{2, 4, 3, 60, 1000}, DBL_BF16, P(a(0)), P(a(1)), I(a(2)), F(a(3)),
                     F(a(4)), P(a(20)), fws, nullptr) == DBL_ESHAPE);
  CHECK(dbl_head_nll(hs, 5, P(a(0)), P(a(1)), I(a(2)), F(a(3)), F(a(4)), P(a(20)), fws, nullptr) ==
        DBL_EDTYPE);
  CHECK(dbl_head_nll(dbl_shape{1 << 14, 1 << 10, 1, 8, 8}, DBL_BF16, P(a(0)), P(a(1)), I(a(2)),
                     F(a(3)), F(a(4)), P(a(20)), bad, nullptr) == DBL_ESHAPE);
  for (dbl_shape s : {dbl_shape{1, 1, 65, 8, 8}, dbl_shape{1, 1, 1, (1 << 20) + 8, 8},
                      dbl_shape{1, 1, 1, 8, 1 << 24}, dbl_shape{-1, 1, 1, 8, 8},
                      dbl_shape{1, 0, 1, 8, 8}, dbl_shape{1, 1, 1, 0, 8}}) {
    CHECK(dbl_head_nll(s, DBL_F32, P(a(0)), P(a(1)), I(a(2)), F(a(3)), F(a(4)), P(a(20)), fws,
                       nullptr) == DBL_ESHAPE);
    CHECK(dbl_workspace_bytes(DBL_OP_HEAD_NLL, s) == bad);
  }
  CHECK(dbl_workspace_bytes(DBL_OP_HEAD_NLL, dbl_shape{1 << 14, 1 << 10, 1, 8, 8}) == bad);
  CHECK(g_launches == before);
  // no rows: nothing to do, except dw = 0
  CHECK(dbl_head_nll(dbl_shape{0, 4, 3, 64, 1000}, DBL_BF16, nullptr, P(a(1)), nullptr, nullptr,
                     nullptr, nullptr, 0, nullptr) == DBL_OK);
  CHECK(dbl_head_nll_backward(dbl_shape{0, 4, 3, 64, 1000}, DBL_BF16, nullptr, P(a(1)), nullptr,
                              nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, 0, nullptr) == DBL_OK);
  CHECK(g_launches == before);
  CHECK(dbl_head_nll_backward(dbl_shape{0, 4, 3, 64, 1000}, DBL_BF16, nullptr, P(a(1)), nullptr,
                              nullptr, nullptr, nullptr, nullptr, P(a(7)), P(a(20)), bws,
                              nullptr) == DBL_OK);
  CHECK(g_launches == before + 1);
  g_result = hipErrorInvalidConfiguration;
  CHECK(dbl_head_nll(hs, DBL_BF16, P(a(0)), P(a(1)), I(a(2)), F(a(3)), F(a(4)), P(a(20)), fws,
                     nullptr) == DBL_EHIP);
  CHECK(strstr(dbl_last_error(), "DBL_EHIP") != nullptr);
  g_result = hipSuccess;

  // --- expander ----------------------------------------------------------------------------
  dbl_shape es{3, 5, 4, 96, 1};
  const size_t ews = dbl_workspace_bytes(DBL_OP_EXPAND_BACKWARD, es);
  CHECK(dbl_expand_branches_backward(es, P(a(0)), P(a(1)), P(a(2)), P(a(3)), P(a(4)), P(a(5)),
                                     P(a(20)), ews, nullptr) == DBL_OK);
  CHECK(g_expand.P == 15 && g_expand.R == 4 && g_expand.d == 96 && g_expand.part == P(a(20)) &&
        g_expand.splits >= 1 && ews >= static_cast<size_t>(g_expand.splits) * 15 * 96 * 4);
  CHECK(dbl_expand_branches_backward(es, P(a(0)), P(a(1)), P(a(2)), nullptr, P(a(4)), nullptr, P(a(20)), ews,
                                     nullptr) == DBL_OK);
  CHECK(!g_expand.dh && !g_expand.dc && g_expand.dW);
  before = g_launches;
  CHECK(dbl_expand_branches_backward(es, P(a(0)), P(a(1)), P(a(2)), nullptr, nullptr, nullptr, P(a(20)),
                                     ews, nullptr) == DBL_EINVAL);
  CHECK(dbl_expand_branches_backward(es, P(a(0)), P(a(1)), P(a(2)), P(a(3)), nullptr, nullptr, P(a(20)),
                                     ews - 1, nullptr) == DBL_EWORKSPACE);
  CHECK(dbl_expand_branches_backward(es, P(a(0)), P(a(1)), P(a(2)), P(a(2)), nullptr, nullptr, P(a(20)),
                                     ews, nullptr) == DBL_EINVAL);
  CHECK(dbl_expand_branches_backward(es, P(a(0)), P(a(1)), P(a(2)), P(a(3)), P(a(4)), P(a(4)), P(a(20)),
                                     ews, nullptr) == DBL_EINVAL);
  CHECK(dbl_expand_branches_backward(es, P(a(0) + 2), P(a(1)), P(a(2)), P(a(3)), P(a(4)), P(a(5)),
                                     P(a(20)), ews, nullptr) == DBL_EINVAL);
  CHECK(dbl_expand_branches_backward(es, P(a(0)), P(a(1)), P(a(2)), nullptr, P(a(4)), nullptr, nullptr, 0,
                                     nullptr) == DBL_EWORKSPACE);
  CHECK(g_launches == before);
  CHECK(dbl_expand_branches_backward(es, P(a(0)), P(a(1)), P(a(2)), nullptr, nullptr, P(a(5)), nullptr, 0,
                                     nullptr) == DBL_OK);
  dbl_shape ms{256, 16, 4, 512, 1};  // a small weight gradient of many rows, in parts
  const size_t mws = dbl_workspace_bytes(DBL_OP_EXPAND_BACKWARD, ms);
  CHECK(dbl_expand_branches_backward(ms, P(a(0)), P(a(1)), P(a(2)), P(a(3)), P(a(4)), P(a(5)), P(a(20)), mws,
                                     nullptr) == DBL_OK);
  CHECK(g_expand.dW_splits > 1 &&
        reinterpret_cast<uintptr_t>(g_expand.dW_part) >=
            a(20) + static_cast<size_t>(g_expand.splits) * 4096 * 512 * 4 &&
        reinterpret_cast<uintptr_t>(g_expand.dW_part) + static_cast<size_t>(g_expand.dW_splits) * 4 * 512 * 512 * 4 <=
            a(20) + mws);
  before = g_launches;
  for (dbl_shape s : {dbl_shape{3, 5, 4, 100, 1}, dbl_shape{3, 5, 65, 96, 1}, dbl_shape{-1, 5, 4, 96, 1},
                      dbl_shape{3, 5, 64, 1 << 18, 1}, dbl_shape{1 << 14, 1 << 10, 1, 32, 1}})
    CHECK(dbl_expand_branches_backward(s, P(a(0)), P(a(1)), P(a(2)), P(a(3)), P(a(4)), P(a(5)), P(a(20)),
                                       bad, nullptr) == DBL_ESHAPE);
  CHECK(g_launches == before);
  CHECK(dbl_expand_branches_backward(dbl_shape{0, 5, 4, 96, 1}, nullptr, P(a(1)), nullptr, nullptr,
                                     P(a(4)), P(a(5)), nullptr, 0, nullptr) == DBL_OK);

  // --- gradient norm and clipping --------------------------------------------------------------
  for (int n : {0, 1, 179, 180, 181, 1000}) {
    std::vector<const void*> g;
    std::vector<void*> out;
    std::vector<int64_t> numel;
    std::vector<int32_t> dt;
    for (int i = 0; i < n; ++i) {
      numel.push_back(i % 7 == 3 ? 0 : 1 + i);
      dt.push_back(i % 2);
      g.push_back(i % 7 == 3 ? nullptr : P(a(1) + 65536u * i + 4));
      out.push_back(i % 7 == 3 ? nullptr : P(a(2) + 65536u * i + 8));
    }
    const size_t nws = dbl_workspace_bytes(DBL_OP_GRAD_NORM, dbl_shape{n, 1, 1, 1, 1});
    CHECK(nws == static_cast<size_t>((n + 179) / 180) * 8192);
    CHECK(dbl_grad_norm(n, g.data(), numel.data(), dt.data(), F(a(0)), n ? P(a(20)) : nullptr, nws,
                        nullptr) == DBL_OK);
    CHECK(static_cast<int>(g_tensors.size()) == n);
    CHECK(dbl_clip_grads(n, g.data(), nullptr, numel.data(), dt.data(), F(a(0)), 1.0f, nullptr) == DBL_OK);
    for (int i = 0; i < n; ++i) CHECK(g_tensors[i].out == g_tensors[i].g && g_tensors[i].n == numel[i]);
    CHECK(dbl_clip_grads(n, g.data(), out.data(), numel.data(), dt.data(), F(a(0)), INFINITY, nullptr) ==
          DBL_OK);
    if (n < 2) continue;
    before = g_launches;
    CHECK(dbl_grad_norm(n, g.data(), numel.data(), dt.data(), F(a(0)), P(a(20)), nws - 1, nullptr) ==
          DBL_EWORKSPACE);
    const void* keep = g[0];
    g[0] = g[1];  // the same tensor twice (fewer elements)
    CHECK(dbl_clip_grads(n, g.data(), nullptr, numel.data(), dt.data(), F(a(0)), 1.0f, nullptr) == DBL_EINVAL);
    g[0] = P(a(1) + 1);
    CHECK(dbl_grad_norm(n, g.data(), numel.data(), dt.data(), F(a(0)), P(a(20)), nws, nullptr) == DBL_EINVAL);
    g[0] = nullptr;
    CHECK(dbl_grad_norm(n, g.data(), numel.data(), dt.data(), F(a(0)), P(a(20)), nws, nullptr) == DBL_EINVAL);
    g[0] = keep;
    CHECK(dbl_grad_norm(n, g.data(), numel.data(), dt.data(), static_cast<float*>(const_cast<void*>(g[1])),
                        P(a(20)), nws, nullptr) == DBL_EINVAL);  // the norm inside a gradient
    void* okeep = out[1];
    out[1] = const_cast<void*>(g[0]);  // an output over another gradient
    CHECK(dbl_clip_grads(n, g.data(), out.data(), numel.data(), dt.data(), F(a(0)), 1.0f, nullptr) == DBL_EINVAL);
    out[1] = okeep;
    CHECK(dbl_clip_grads(n, g.data(), nullptr, numel.data(), dt.data(), static_cast<const float*>(g[0]), 1.0f,
                         nullptr) == DBL_EINVAL);  // the norm inside a gradient
    CHECK(dbl_clip_grads(n, g.data(), nullptr, numel.data(), dt.data(), F(a(0)), -1.0f, nullptr) == DBL_EINVAL);
    CHECK(dbl_clip_grads(n, g.data(), nullptr, numel.data(), dt.data(), F(a(0)), std::nanf(""), nullptr) ==
          DBL_EINVAL);
    CHECK(dbl_clip_grads(n, g.data(), nullptr, numel.data(), dt.data(), nullptr, 1.0f, nullptr) == DBL_EINVAL);
    dt[0] = 7;
    CHECK(dbl_grad_norm(n, g.data(), numel.data(), dt.data(), F(a(0)), P(a(20)), nws, nullptr) == DBL_EDTYPE);
    dt[0] = 0;
    numel[0] = -1;
    CHECK(dbl_grad_norm(n, g.data(), numel.data(), dt.data(), F(a(0)), P(a(20)), nws, nullptr) == DBL_ESHAPE);
    numel[0] = std::numeric_limits<int64_t>::max();
    CHECK(dbl_grad_norm(n, g.data(), numel.data(), dt.data(), F(a(0)), P(a(20)), nws, nullptr) == DBL_ESHAPE);
    CHECK(g_launches == before);
  }
  CHECK(dbl_grad_norm(-1, nullptr, nullptr, nullptr, F(a(0)), nullptr, 0, nullptr) == DBL_ESHAPE);
  CHECK(dbl_grad_norm(1, nullptr, nullptr, nullptr, F(a(0)), nullptr, 0, nullptr) == DBL_EINVAL);

  if (g_fail) {
    fprintf(stderr, "%d checks failed\n", g_fail);
    return 1;
  }
  printf("all checks passed\n");
  return 0;
}
