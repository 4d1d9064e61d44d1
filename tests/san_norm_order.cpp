// What the order of a norm's sums depends on, under AddressSanitizer and UndefinedBehaviorSanitizer (no GPU involved).  A kernel of the
// norm takes from its table each tensor's first unit, type, place and address, and of the address only the part below a line decides which
// of its elements a thread adds up; the host goes by bytes and entries besides.  Built and run by tests/test_norm_order_host.py.
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "thc.h"
#include "thc_tensorplan.hpp"

using namespace thc;

struct Tensor {
  uint64_t numel;
  uint32_t type;
  uint64_t gap;   // bytes between the end of the tensor before it and its start
};

// Everything that the order of the sums goes by, for a list that starts at `base`.
static std::vector<uint64_t> order(const std::vector<Tensor>& list, uint64_t base, uint64_t* entries = nullptr) {
  std::vector<void*> data;
  std::vector<uint64_t> numel, found;
  std::vector<uint32_t> type;
  for (const Tensor& x : list) {
    base += x.gap;
    data.push_back(x.numel ? reinterpret_cast<void*>(base) : nullptr);
    numel.push_back(x.numel);
    type.push_back(x.type);
    base += x.numel * type_bytes(x.type);
  }
  const thc_tensors t{list.size(), data.data(), numel.data(), type.data()};
  Scan scan;
  if (scan_tensors(&t, &scan) != THC_OK) {
    std::printf("refused\n");
    std::exit(1);
  }
  if (entries) *entries = scan.entries;
  found = {scan.bytes, scan.entries};
  for (uint32_t log_unit : {LOG_NORM_UNIT, LOG_WAVE_UNIT})
    for_tables(&t, scan, Grid::TENSOR, 0, 0, log_unit, [&](const TensorTable<TABLE>& tab, uint32_t count, uint32_t units) {
      found.push_back(count);
      found.push_back(units);
      for (uint32_t k = 0; k < count; ++k) {
        found.push_back(tab.unit[k]);
        found.push_back(tab.at[k]);
        found.push_back((tab.ptr[k] & ~PTR_MASK) | (tab.ptr[k] & PTR_MASK) % LINE);
      }
    });
  return found;
}

static int problems = 0;
static void check(bool ok, const char* what, long long a = 0) {
  if (ok) return;
  ++problems;
  std::printf("%s (%lld)\n", what, a);
}

int main() {
  std::srand(11);
  auto rnd = [](uint64_t n) { return (uint64_t)std::rand() % n; };
  const uint64_t base = 1ull << 32;
  // lists that agree in sizes, types, addresses modulo 128 and in which tensors adjoin: the same order wherever they lie
  for (int round = 0; round < 300; ++round) {
    std::vector<Tensor> list;
    uint64_t at = base;
    const int count = round % 5 == 0 ? 250 + (int)rnd(300) : 1 + (int)rnd(40);
    for (int i = 0; i < count; ++i) {
      const uint32_t type = round % 2 ? (uint32_t)rnd(3) : (uint32_t)(round % 3);
      uint64_t gap = rnd(2) ? 0 : 4 * (1 + rnd(60));
      gap += (at + gap) % type_bytes(type);
      list.push_back({rnd(9) ? 1 + rnd(count > 40 ? 3000 : 50000) : 0, type, gap});
      at += gap + list.back().numel * type_bytes(type);
    }
    std::vector<Tensor> moved = list;
    bool behind = false;                      // whether a tensor with elements came before
    uint64_t between = 0;                     // bytes since its end
    for (Tensor& x : moved) {
      between += x.gap;
      if (x.numel) {
        if (behind && between) x.gap += LINE * rnd(1000);   // what adjoins stays together
        behind = true;
        between = 0;
      }
    }
    check(order(list, base) == order(moved, base + LINE * rnd(1 << 20)), "another order for the same list further on", round);
  }
  // the same addresses modulo 128, adjoining and 128 bytes apart: another order
  uint64_t one = 0, two = 0;
  const auto joined = order({{1000512, THC_DTYPE_F32, 0}, {1000512, THC_DTYPE_F32, 0}}, base, &one);
  const auto apart = order({{1000512, THC_DTYPE_F32, 0}, {1000512, THC_DTYPE_F32, LINE}}, base, &two);
  check(joined != apart && one == 1 && two == 2, "tensors that adjoin are cut as if they did not");
  // adjoining goes by the types and past tensors without elements
  order({{64, THC_DTYPE_BF16, 0}, {64, THC_DTYPE_F16, 0}}, base, &two);
  order({{64, THC_DTYPE_BF16, 0}, {0, THC_DTYPE_F32, 0}, {64, THC_DTYPE_BF16, 0}}, base, &one);
  check(one == 1 && two == 2, "what counts as adjoining");
  std::printf("%d problem(s)\n", problems);
  return problems != 0;
}
