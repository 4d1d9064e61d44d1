// Host side of the calls that take lists of tensors under AddressSanitizer and UndefinedBehaviorSanitizer (no GPU involved): the checks
// of a list, and its tables, walked as the kernels walk them.  Built and run by tests/test_tensors_host.py.
#include <cstdio>
#include <cstdlib>
#include <utility>
#include <vector>

#include "thc.h"
#include "thc_tensorplan.hpp"

using namespace thc;

struct List {
  std::vector<void*> data;
  std::vector<uint64_t> numel;
  std::vector<uint32_t> dtype;
  void add(uint64_t at, uint64_t n, uint32_t type) {
    data.push_back(reinterpret_cast<void*>(at));
    numel.push_back(n);
    dtype.push_back(type);
  }
  thc_tensors get() const { return {data.size(), data.data(), numel.data(), dtype.data()}; }
};

static int overlap(const thc_tensors* t, bool each_other, std::initializer_list<Range> others) {
  Scan scan;
  const int rc = scan_tensors(t, &scan);
  return rc ? rc : check_overlap(t, scan, each_other, others);
}

static int problems = 0;
static void check(bool ok, const char* what, long long a = 0, long long b = 0) {
  if (ok) return;
  ++problems;
  std::printf("%s (%lld, %lld)\n", what, a, b);
}

// What a unit's threads take of a tensor of `len` bytes whose grid starts at `lo`: take(first byte, bytes)
template <class Take>
static void walk_unit(int64_t lo, int64_t len, uint32_t log_unit, int slot, int size, Take&& take) {
  const int64_t first = lo < 0 ? lo & (slot - 1) : 0, last = len - ((len - lo) & (slot - 1));
  for (int t = 0; t < slot / size; ++t) {
    if (lo < 0 && t * size < first && t * size < len) take(t * size, size);
    if (last >= first && last - lo < (1 << log_unit) && last + t * size < len) take(last + t * size, size);
  }
  for (int64_t at = 0; at < (1 << log_unit); at += slot)
    if (lo + at >= 0 && lo + at + slot <= len) take(lo + at, slot);
}

// Every element of a short list is taken once, in the units that locate() would find for it, and lies where the list has it.
static void check_cover(const List& l, Grid grid, uint32_t flat_bytes, uint64_t zeros, uint32_t log_unit, int slot16) {
  const thc_tensors t = l.get();
  Scan scan;
  check(scan_tensors(&t, &scan) == THC_OK, "refused");
  const uint64_t total = scan.total;
  std::vector<int> seen(total + zeros, 0);
  std::vector<uint64_t> address(total + zeros, 0);
  for (uint64_t i = 0, pos = 0; i < t.count; ++i)
    for (uint64_t j = 0; j < t.numel[i]; ++j) address[pos++] = reinterpret_cast<uintptr_t>(t.data[i]) + j * type_bytes(t.dtype[i]);
  uint32_t most = 0, least = ~0u, launches = 0;
  uint64_t entries = 0, bytes = 0;
  for_tables(&t, scan, grid, flat_bytes, zeros, log_unit, [&](const TensorTable<TABLE>& tab, uint32_t count, uint32_t units) {
    ++launches;
    entries += count;
    most = count > most ? count : most;
    least = count < least ? count : least;
    check(count >= 1 && count <= TABLE, "tensors of a table", count);
    TensorTable<SHORT_TABLE> small;
    if (count <= SHORT_TABLE) shorten(tab, count, &small);
    for (uint32_t u = 0; u < units; ++u) {
      uint32_t n = 0, m = 0;
      for (uint32_t k = 0; k < 64 * tab.LANES; ++k) n += tab.unit[k] <= u;
      if (count <= SHORT_TABLE) {
        for (uint32_t k = 0; k < 64 * small.LANES; ++k) m += small.unit[k] <= u;
        check(n == m && small.ptr[n] == tab.ptr[n] && small.at[n] == tab.at[n], "short table", n, m);
      }
      check(n >= 1 && n <= count, "unit without a tensor", u, n);
      const uint32_t i = n - 1;
      auto place = [&](uint32_t k) { return (tab.ptr[k] >> PTR_BITS & 0xFF) << 32 | tab.at[k]; };
      const uint32_t type = (uint32_t)(tab.ptr[i] >> (PTR_BITS + 8));
      const uint64_t ptr = tab.ptr[i] & PTR_MASK, at = place(i);
      const uint32_t size = grid == Grid::FLAT ? flat_bytes : type_bytes(type);
      const int64_t len = (int64_t)((place(i + 1) - at) * size);
      const uint64_t start = grid == Grid::FLAT ? at * size : ptr;
      const int64_t lo = (int64_t)((uint64_t)(u - tab.unit[i]) << log_unit) - (int64_t)(start % LINE);
      check(lo < len, "empty unit", u, i);
      check((start + (uint64_t)lo) % LINE == 0, "unit off its line", u, lo);
      walk_unit(lo, len, log_unit, size == 2 ? slot16 : 16, (int)size, [&](int64_t byte, int bytes) {
        for (int64_t b = byte; b < byte + bytes; b += size) {
          const uint64_t e = at + (uint64_t)b / size;
          check(b >= 0 && b < len && e < seen.size(), "outside its tensor", b, len);
          if (e >= seen.size()) return;
          ++seen[e];
          if (e < total) check(ptr + (uint64_t)b / size * type_bytes(type) == address[e], "wrong address", (long long)e);
          else check(type == TYPE_ZEROS, "no zeros behind the list", (long long)e);
        }
      });
    }
  });
  for (uint64_t i = 0; i < t.count; ++i) bytes += t.numel[i] * type_bytes(t.dtype[i]);
  check(entries == scan.entries + (zeros != 0) && bytes == scan.bytes, "entries or bytes", (long long)entries, (long long)scan.entries);
  for (uint64_t e = 0; e < seen.size(); ++e) check(seen[e] == 1, "element not taken once", (long long)e, seen[e]);
  check(launches < 2 || most - least <= launches, "launches of different lengths", most, least);
}

static void check_long() {
  // more than one launch can hold, by units and by elements; 2^39 bytes apart, nothing is read
  List l;
  l.add(1ull << 32, 5, THC_DTYPE_F32);
  l.add((1ull << 33) + 4, (3ull << 33) + 7, THC_DTYPE_F32);
  l.add(1ull << 40, 3ull << 34, THC_DTYPE_BF16);
  const thc_tensors t = l.get();
  uint64_t sum = 0, next = 0;
  Scan scan;
  check(scan_tensors(&t, &scan) == THC_OK, "long list refused");
  const uint64_t total = scan.total;
  int launches = 0;
  for (Grid grid : {Grid::TENSOR, Grid::FLAT}) {
    sum = next = 0;
    for_tables(&t, scan, grid, 4, 9, LOG_MOVE_UNIT, [&](const TensorTable<TABLE>& tab, uint32_t count, uint32_t units) {
      ++launches;
      check(units && units <= MOST_UNITS && (uint64_t)units * 256 < 1ull << 32, "units of a launch", units);
      auto place = [&](uint32_t k) { return (tab.ptr[k] >> PTR_BITS & 0xFF) << 32 | tab.at[k]; };
      check(place(0) == next, "launches do not follow each other", (long long)next);
      next = place(count);
      for (uint32_t k = 0; k < count; ++k) sum += place(k + 1) - place(k);
    });
    check(sum == total + 9, "long list's elements", (long long)sum, (long long)total);
  }
  check(launches > 4, "long list's launches", launches);
}

int main() {
  std::srand(7);
  auto rnd = [](uint64_t n) { return (uint64_t)std::rand() % n; };
  for (int round = 0; round < 120; ++round) {
    List l;
    uint64_t at = 1 << 20;
    const int count = round % 6 == 0 ? 200 + (int)rnd(400) : (int)rnd(12);
    for (int i = 0; i < count; ++i) {
      const uint32_t type = round % 3 == 0 ? (uint32_t)rnd(3) : (uint32_t)(round % 3);
      const uint64_t n = rnd(8) == 0 ? 0 : rnd(count > 20 ? 60 : rnd(2) ? 40 : 12000);
      if (rnd(3)) at += rnd(400) * 2;          // otherwise right behind the one before
      at += at % type_bytes(type);
      l.add(n ? at : 0, n, type);
      at += n * type_bytes(type);
    }
    const uint64_t zeros = rnd(2) ? rnd(3000) : 0;
    check_cover(l, Grid::TENSOR, 0, 0, LOG_NORM_UNIT, 16);
    check_cover(l, Grid::TENSOR, 0, 0, LOG_WAVE_UNIT, 16);
    check_cover(l, Grid::TENSOR, 0, 0, LOG_MOVE_UNIT, 8);
    for (uint32_t b : {2u, 4u}) check_cover(l, Grid::FLAT, b, zeros, LOG_MOVE_UNIT, round % 2 ? 16 : 8);
    for (uint32_t b : {2u, 4u}) check_cover(l, Grid::FLAT, b, zeros, LOG_NORM_UNIT, 16);
    const thc_tensors t = l.get();
    Scan scan;
    bool wide = false, narrow = false;
    for (uint64_t i = 0; i < t.count; ++i)
      if (t.numel[i]) (t.dtype[i] == THC_DTYPE_F32 ? wide : narrow) = true;
    check(scan_tensors(&t, &scan) == THC_OK && same_size(scan, 4) == !narrow && same_size(scan, 2) == !wide, "sizes of elements");
    check(overlap(&t, true, {}) == THC_OK, "overlap where there is none");
    if (count > 1) {                           // in another order, and then one of them twice
      std::swap(l.data.front(), l.data.back());
      std::swap(l.numel.front(), l.numel.back());
      std::swap(l.dtype.front(), l.dtype.back());
      const thc_tensors s = l.get();
      check(overlap(&s, true, {}) == THC_OK, "overlap where there is none, in another order");
      for (int i = 0; i < count; ++i)
        if (l.numel[i]) {
          const char* const p = static_cast<char*>(l.data[i]);
          const uint64_t n = l.numel[i] * type_bytes(l.dtype[i]);
          check(overlap(&s, false, {Range(nullptr, 4), Range(p + n - 1, 1)}) == THC_EINVAL, "range over a tensor's end not seen");
          check(overlap(&s, false, {Range(p - 3, 4)}) == THC_EINVAL, "range over a tensor's start not seen");
          check(overlap(&s, false, {Range(reinterpret_cast<void*>(1 << 19), 1 << 19)}) == THC_OK, "range in front of the list");
          l.add(reinterpret_cast<uintptr_t>(l.data[i]) + (l.numel[i] - 1) * type_bytes(l.dtype[i]), 1, l.dtype[i]);
          const thc_tensors d = l.get();
          check(overlap(&d, true, {}) == THC_EINVAL, "overlap not seen");
          check(overlap(&d, false, {}) == THC_OK, "overlap of what is only read");
          break;
        }
    }
  }
  check_long();
  check(norm_keeps((24ull << 20) - 1, true) == 0 && norm_keeps(24ull << 20, true) == 256ull << 20 && norm_keeps(1, false) == 256ull << 20,
        "norm_keeps");
  check(behind_norm(128ull << 20) && !behind_norm((128ull << 20) + 1), "behind_norm");
  std::printf("%d problem(s)\n", problems);
  return problems != 0;
}
