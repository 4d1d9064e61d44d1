// Which gathers go by the norm's units, under AddressSanitizer and UndefinedBehaviorSanitizer (no GPU involved).  Built and run by
// tests/test_gather_rule_host.py.
#include <cstdio>
#include <vector>

#include "thc.h"
#include "thc_tensorplan.hpp"

using namespace thc;

static bool by_norm_units(uint64_t bytes, uint64_t tensors, uint32_t type, uint32_t flat_bytes, uint64_t zeros) {
  std::vector<void*> data;
  std::vector<uint64_t> numel;
  std::vector<uint32_t> types(tensors, type);
  uint64_t at = 1ull << 32, left = bytes / type_bytes(type);
  for (uint64_t i = 0; i < tensors; ++i) {
    data.push_back(reinterpret_cast<void*>(at));
    numel.push_back(left / (tensors - i));
    left -= numel.back();
    at += numel.back() * type_bytes(type) + 256;
  }
  const thc_tensors t{tensors, data.data(), numel.data(), types.data()};
  Scan scan;
  if (scan_tensors(&t, &scan) != THC_OK) return false;
  return gather_behind_norm(scan, flat_bytes, zeros);
}

int main() {
  int problems = 0;
  auto check = [&](bool ok, const char* what) {
    if (!ok) ++problems, std::printf("%s\n", what);
  };
  constexpr uint64_t MB = 1 << 20;
  for (uint32_t type : {(uint32_t)THC_DTYPE_F32, (uint32_t)THC_DTYPE_BF16}) {
    const uint32_t size = type_bytes(type);
    check(by_norm_units(51 * MB, 161, type, size, 5), "a list in one launch behind its norm");
    check(by_norm_units(12 * MB, 1, type, size, 0) && by_norm_units(128 * MB, 1, type, size, 0), "the shortest and the longest");
    check(!by_norm_units(12 * MB - 4, 1, type, size, 0) && !by_norm_units(8 * MB, 160, type, size, 0), "shorter lists");
    check(!by_norm_units(128 * MB + 4, 1, type, size, 0), "longer lists");
    check(!by_norm_units(51 * MB, 400, type, size, 0), "lists of more than one launch");
    check(by_norm_units(51 * MB, TABLE, type, size, 0) && !by_norm_units(51 * MB, TABLE, type, size, 1), "zeros take a place of their own");
    check(!by_norm_units(51 * MB, 10, type, 6 - size, 0), "elements of another size");
  }
  std::printf("%d problem(s)\n", problems);
  return problems != 0;
}
