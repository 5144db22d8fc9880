// Host-side check of the tensor operators' C entries, built with
// AddressSanitizer and UndefinedBehaviorSanitizer on the host code
// (tests/test_operators_sanitized.py): arguments at and past their limits,
// sizes of scratch and states, and, on a machine without a GPU, calls that fail
// at their first launch or allocation.  Nothing here touches device memory.
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <limits>
#include <vector>
#include "hieravg.h"

int main() {
  int fails = 0;
  auto expect = [&](bool ok, const char* what) { if (!ok) { std::printf("FAIL %s (%s)\n", what, hieravg_last_error()); ++fails; } };
  alignas(64) static char mem[1024];
  void* p = mem;
  const int64_t big = std::numeric_limits<int64_t>::max(), low = std::numeric_limits<int64_t>::min();
  const int64_t sizes[] = {low, -1, 0, 1, 2, 64, 65, 127, 128, 129, 1024, 1025, 8192, 8193, 131072, 131073, 1 << 23, (1 << 23) + 1,
                           0x7FFFFF00, 0x7FFFFFFF, int64_t(1) << 31, int64_t(1) << 40, big - 127, big};
  const int32_t tops[] = {std::numeric_limits<int32_t>::min(), -1, 0, 1, 8, 9, 64, 65, std::numeric_limits<int32_t>::max()};
  // Sizes of scratch: any arguments; 0 for those that a call refuses.
  size_t sum = 0;
  for (int64_t r : sizes)
    for (int64_t c : sizes) {
      for (int32_t t : tops) {
        const size_t s = hieravg_log_probs_scratch(r, c, t);
        if (r < 1 || r > 0x7FFFFFFF || c < 1 || c > 1 << 23 || t < 0 || t > HIERAVG_TOP_MAX) expect(s == 0, "scratch of refused log_probs");
        sum += s;
      }
      for (int64_t k : sizes) {
        const size_t s = hieravg_block_product_scratch(r, c, k);
        if (r < 1 || c < 1 || k < 1 || r > 0x7FFFFF00 || c > 0x7FFFFF00 || k > 1 << 23) expect(s == 0, "scratch of a refused product");
        sum += s;
      }
    }
  expect(sum > 0, "scratch at all");
  expect(hieravg_log_probs_scratch(1, 1 << 23, 64) == 64 * (16 + 8 * 64), "scratch of the longest row");
  // Calls with every argument at its limits: refused, or, without a GPU, failed.
  for (int64_t r : sizes)
    for (int64_t c : sizes)
      for (int64_t s : {c, big, low, int64_t(0)}) {
        expect(r == 0 || hieravg_log_probs(p, 0, r, c, s, p, 8, 3, (float*)p, (float*)p, (float*)p, (int32_t*)p, (float*)p, nullptr, 0, nullptr) != HIERAVG_OK, "log_probs");
        expect(r == 0 || hieravg_log_probs_grad(p, 3, r, c, s, p, 8, (float*)p, (float*)p, (float*)p, (float*)p, p, s, nullptr) != HIERAVG_OK, "log_probs_grad");
        expect(r == 0 || hieravg_quantize_blocks(p, 2, r, c, s, 2, (uint8_t*)p, (uint8_t*)p, nullptr, nullptr, nullptr) != HIERAVG_OK, "quantize_blocks");
        expect(hieravg_block_product((uint8_t*)p, (uint8_t*)p, 0, (uint8_t*)p, (uint8_t*)p, 1, r, c, 200, nullptr, 1, s, nullptr, 0, nullptr) != HIERAVG_OK || r == 0 || c == 0, "block_product");
      }
  // Strides and pointers whose rows end past any address.
  expect(hieravg_log_probs_grad(p, 0, 0x7FFFFFFF, 4, big, p, 8, nullptr, (float*)p, (float*)p, (float*)p, p, big - 4, nullptr) == HIERAVG_EINVAL, "strides");
  // Sizes of states.
  std::vector<int64_t> n(1 << 10, int64_t(1) << 40);
  expect(hieravg_adamw_state_size(n.data(), 1 << 10) == int64_t(1) << 50, "state size");
  n.assign(3, big);
  expect(hieravg_adamw_state_size(n.data(), 3) == HIERAVG_EINVAL, "state size past the limit");
  n.assign(3, low);
  expect(hieravg_adamw_state_size(n.data(), 3) == HIERAVG_EINVAL, "negative state size");
  // AdamW: refusals, and a create that fails at its first HIP call.
  hieravg_adamw_config cfg{0.1, 0.9, 0.999, 1e-8, 0.01, 5, 8};
  hieravg_adamw_tensor t{mem, nullptr, 4, 0, 0, 0};
  for (int64_t k : {low, int64_t(-1), (int64_t(1) << 40) + 1, big}) {
    t.n = k;
    expect(!hieravg_adamw_create(&cfg, &t, 1, p, p, (uint8_t*)p, (uint8_t*)p), "size");
  }
  t.n = 4;
  cfg.state_bits = 7;
  expect(!hieravg_adamw_create(&cfg, &t, 1, p, p, (uint8_t*)p, (uint8_t*)p), "bits");
  cfg.state_bits = 8;
  hieravg_adamw_t h = hieravg_adamw_create(&cfg, &t, 1, p, p, (uint8_t*)p, (uint8_t*)p);
  std::printf("create without device: %p (%s)\n", (void*)h, hieravg_last_error());
  expect(!h, "create without a device");
  hieravg_adamw_destroy(h);
  double lr = 0;
  expect(hieravg_adamw_step(nullptr, nullptr, nullptr) == HIERAVG_EINVAL && hieravg_adamw_lr(nullptr, &lr) == HIERAVG_EINVAL &&
             hieravg_adamw_set_steps(nullptr, big, nullptr) == HIERAVG_EINVAL && hieravg_adamw_steps(nullptr) == HIERAVG_EINVAL &&
             hieravg_adamw_set_lr(nullptr, 0.1, nullptr) == HIERAVG_EINVAL, "NULL handles");
  expect(hieravg_scores(nullptr, 0, 0, 4, 0, (float*)p, (float*)p, nullptr, nullptr) == HIERAVG_EINVAL, "scores null");
  std::printf("%s\n", fails ? "host checks FAILED" : "host checks ok");
  return fails != 0;
}
