// CPU check of compact_tokens (paper_2511_20982_amd/csrc/plan_masked.hpp) at the limits of
// its arguments: every move within the page table is among the tokens, and the kernel's
// places and loop counters stay ints.  Prints "ok" or the first failure.
#include <cstdio>

#include "../paper_2511_20982_amd/csrc/plan_masked.hpp"

using namespace dopd;

constexpr int kPage = 16;

int main() {
  const int edge[] = {INT32_MIN, -1, 0, 1, 2, 15, 16, 17, 128, 1 << 20, (1 << 26) - 1, 1 << 26, 1 << 27, kMaMaxPos - 1,
                      kMaMaxPos, kMaMaxPos + 1, INT32_MAX - 8, INT32_MAX - 1, INT32_MAX};
  for (int count : edge)
    for (int most : edge)
      for (int pre : edge)
        for (int stride : edge) {
          if (most < 1 || pre < 0 || pre >= kMaMaxPos || stride < 0) continue;  // (refused, or left out before)
          const int64_t m = compact_tokens(count, most, pre, (int64_t)stride * kPage), room = (int64_t)stride * kPage - pre;
          const int64_t all = std::min<int64_t>(count, most), in = std::min({all, room, (int64_t)kMaMaxPos});
          if (m > 0 ? m != in : in > 0) return std::printf("FAIL tokens %d %d %d %d\n", count, most, pre, stride), 1;
          // last page, last slot of it, the counter behind the last group of eight tokens
          if (m > 0 && ((pre + m - 1) / kPage * kPage + kPage - 1 > INT32_MAX || (m + 7) / 8 * 8 > INT32_MAX))
            return std::printf("FAIL overflow %d %d %d %d\n", count, most, pre, stride), 1;
        }
  std::printf("ok\n");
  return 0;
}
