// Host-side check of the C entries of low-rank adapters, gradient norms and the
// verification of drafts, built with AddressSanitizer and
// UndefinedBehaviorSanitizer on the host code (tests/test_more_operators_sanitized.py):
// arguments at and past their limits, sizes of scratch, and, on a machine
// without a GPU, calls that fail at their first launch.  Nothing here touches
// device memory.
#include <cstdint>
#include <cstdio>
#include <limits>
#include <vector>
#include "internal.h"

// What the operators' sources take from the rest of the library.
static thread_local std::string g_text;
namespace hav {
thread_local LaunchTiming g_launch_timing;
void set_error(const std::string& s) { g_text = s; }
}  // namespace hav
extern "C" const char* hieravg_last_error(void) { return g_text.c_str(); }

int main() {
  int fails = 0;
  auto expect = [&](bool ok, const char* what) { if (!ok) { std::printf("FAIL %s (%s)\n", what, hieravg_last_error()); ++fails; } };
  alignas(64) static char mem[4096];
  char* p = mem;
  float* f = (float*)mem;
  const int64_t big = std::numeric_limits<int64_t>::max(), low = std::numeric_limits<int64_t>::min();
  const size_t huge = std::numeric_limits<size_t>::max();
  const int64_t sizes[] = {low, -1, 0, 1, 2, 63, 64, 65, 2047, 2049, 131072, 1 << 23, (1 << 23) + 1, 1 << 24, (1 << 24) + 1, int64_t(1) << 31, big};
  const int32_t counts[] = {std::numeric_limits<int32_t>::min(), -1, 0, 1, 16, 17, 64, 65, 128, 129, 8192, 8193, std::numeric_limits<int32_t>::max()};
  size_t sum = 0;
  // Drafts.
  for (int64_t s : sizes)
    for (int32_t d : counts)
      for (int64_t c : sizes) {
        const size_t n = hieravg_verify_drafts_scratch(s, d, c, 1);
        if (s < 1 || s > 1 << 24 || d < 0 || d > HIERAVG_DRAFTS_MAX || c < 1 || c > 1 << 23) expect(n == 0, "scratch of refused drafts");
        sum += n;
        for (int64_t stride : {c, big, low, int64_t(0)})
          expect(hieravg_verify_drafts(p, 0, s, d, c, stride, p, 1, stride, p, 4, f, nullptr, f, (int32_t*)p, (int32_t*)p, f, p, huge, nullptr) != HIERAVG_OK || s == 0, "drafts");
      }
  // Adapters.
  for (int64_t r : sizes)
    for (int32_t n : counts)
      for (int32_t k : counts)
        for (int64_t i : {int64_t(1), int64_t(7), int64_t(4096), int64_t(1) << 24, (int64_t(1) << 24) + 1, big, low})
          for (int32_t type : {0, 1, 2, 3}) {
            const hieravg_adapters w{p, p, f, i, i, n, k, type};
            const size_t a = hieravg_adapter_product_scratch(r, &w), b = hieravg_adapter_grad_scratch(r, &w, 0), c = hieravg_adapter_grad_scratch(r, &w, 1);
            if (r < 1 || r > 1 << 24 || n < 1 || n > HIERAVG_ADAPTERS_MAX || k < 1 || k > HIERAVG_RANK_MAX || i < 1 || i > 1 << 24 || type > 2)
              expect(a == 0 && b == 0 && c == 0, "scratch of refused adapters");
            sum += a + b + c;
            if (r == 0) continue;
            for (int64_t stride : {i, big, low}) {
              expect(hieravg_adapter_product(&w, p, r, stride, p, 8, p, stride, p + 64, 0, stride, f, p, huge, nullptr) != HIERAVG_OK, "product");
              expect(hieravg_adapter_grad(&w, p, r, stride, p, stride, p, 4, nullptr, nullptr, 0, p + 64, 2, stride, p, p, 0, p, huge, nullptr) != HIERAVG_OK, "gradient");
              expect(hieravg_adapter_grad(&w, p, r, stride, p, stride, p, 4, f, nullptr, 0, nullptr, 2, stride, p, p, 1, p, huge, nullptr) != HIERAVG_OK, "gradient of weights");
            }
          }
  expect(hieravg_adapter_product(nullptr, p, 1, 1, p, 4, nullptr, 1, p, 0, 1, nullptr, p, huge, nullptr) == HIERAVG_EINVAL, "no adapters");
  // Norms and scaling.
  for (int64_t n : sizes)
    for (int32_t count : {std::numeric_limits<int32_t>::min(), 0, 1, 3, 300}) {
      std::vector<hieravg_tensor> t(300, hieravg_tensor{p, n, 2});
      t[1] = {nullptr, 5, 0};
      std::vector<void*> out(300, p);
      sum += hieravg_grad_norm_scratch(t.data(), count);
      expect(hieravg_grad_norm(t.data(), count, 1.0, f, f, f, p, huge, nullptr) != HIERAVG_OK, "norm");
      expect(hieravg_scale_tensors(t.data(), out.data(), count, f, nullptr) != HIERAVG_OK || n == 0, "scaling");
    }
  expect(hieravg_grad_norm(nullptr, 1, 1.0, f, f, f, p, huge, nullptr) == HIERAVG_EINVAL && hieravg_scale_tensors(nullptr, nullptr, 1, f, nullptr) == HIERAVG_EINVAL, "no tensors");
  std::vector<hieravg_tensor> many(1 << 20, hieravg_tensor{p, 1, 0});
  expect(hieravg_grad_norm_scratch(many.data(), 1 << 20) == size_t(12) << 20, "scratch of many tensors");
  expect(hieravg_grad_norm_scratch(many.data(), (1 << 20) + 1) == 0, "scratch of too many tensors");
  expect(sum > 0, "scratch at all");
  std::printf("%s\n", fails ? "host checks FAILED" : "host checks ok");
  return fails != 0;
}
