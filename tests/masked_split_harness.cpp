// Prints how ma_split (paper_2511_20982_amd/csrc/plan_masked.hpp) deals requests of `rows`
// packed rows (g = 8) and 1000 keys, beside one chunk of 512 tokens, to kernels: a line
// "<requests> <hi16> <hi64>" for 1 to 40 of them.
// Usage: masked_split_harness <cus> <hkv> <rows> <mid>
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "../paper_2511_20982_amd/csrc/plan_masked.hpp"

using namespace dopd;

int main(int argc, char** argv) {
  if (argc < 5) return 2;
  const MachineShape mach{std::atoi(argv[1]), 1};
  const int hkv = std::atoi(argv[2]), tokens = std::atoi(argv[3]) / 8;
  std::vector<int32_t> cu{0, 512}, pre{0};
  for (int n = 1; n <= 40; ++n) {
    cu.push_back(cu.back() + tokens);
    pre.push_back(1000 - tokens);
    const MaSplit s = ma_split(MaskRule{1, 0, 0}, cu.data(), pre.data(), n + 1, 8, hkv, std::atoi(argv[4]) != 0, mach);
    std::printf("%d %d %d\n", n, s.hi16, s.hi64);
  }
  return 0;
}
