// Host check of meet() (csrc/ops.h), by which the tensor operators refuse results
// that share memory with other operands: against a search over all bytes, for
// matrices of up to three rows and blocks.  Built with sanitizers
// (tests/test_more_operator_limits_abi.py).
#include <cstdio>
#include <vector>
#include "ops.h"

namespace hav {
thread_local LaunchTiming g_launch_timing;
void set_error(const std::string&) {}
}  // namespace hav
using namespace hav;

static bool share(const Area& a, const Area& b) {
  if (!a.len || !b.len) return false;  // rows of no bytes
  for (int64_t i = 0; i < a.rows; ++i)
    for (int64_t j = 0; j < b.rows; ++j) {
      const char *x = (const char*)a.p + i * a.stride, *y = (const char*)b.p + j * b.stride;
      if (x < y + b.len && y < x + a.len) return true;
    }
  return false;
}

int main() {
  static char mem[64];
  std::vector<Area> all;
  for (int at = 0; at < 14; ++at)
    for (int64_t rows = 1; rows <= 3; ++rows)
      for (int64_t len = 0; len <= 4; ++len)
        for (int64_t stride = len; stride <= 7; ++stride) all.push_back({mem + at, rows, stride, len});
  all.push_back({nullptr, 3, 4, 4});
  int64_t fails = 0, met = 0, apart = 0;
  for (const Area& a : all)
    for (const Area& b : all) {
      const bool want = a.p && b.p && share(a, b), got = meet(a, b);
      const bool exact = a.rows == 1 || b.rows == 1 || a.stride == a.len || b.stride == b.len;
      met += want;
      apart += !want && !got;
      if ((want && !got) || (exact && want != got)) ++fails;
    }
  // far apart and near the end of the addresses
  const Area low{(const void*)16, 1 << 24, int64_t(1) << 32, 8}, block{(const void*)(uintptr_t(5) << 32), 1, 16, 16};
  if (meet(low, block) || !meet(low, {(const void*)((uintptr_t(5) << 32) + 15), 1, 2, 2})) ++fails;
  if (meet_any(block, Area{}, Area{}) || !meet_any(block, Area{}, block)) ++fails;
  std::printf("%s %lld %lld\n", fails ? "FAILED" : "overlap ok", (long long)met, (long long)apart);
  return fails != 0;
}
