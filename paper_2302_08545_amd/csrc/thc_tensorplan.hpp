// Host side of the calls that take a list of tensors: validation, and the tables of tensors that travel with each launch.
// Plain C++ (no GPU types), so that it can be built and run under the host sanitizers.
#pragma once

#include <algorithm>
#include <cstdint>
#include <new>
#include <vector>

#include "thc.h"

namespace thc {

// The work of a launch is counted in units of UNIT elements.  A tensor's units lie on a grid that starts on a 128-byte line of
// what the kernel accesses in whole lines (its own memory, or its place in the flat vector), up to one line before its first
// element, so that no line but a tensor's first and last is shared by two units.
constexpr uint32_t LOG_UNIT = 13, UNIT = 1u << LOG_UNIT;
constexpr uint32_t LINE = 128;

// Tensors of one launch, passed by value (a captured graph keeps them): a kernel's arguments have to stay within 4 KB.
constexpr uint32_t TABLE = 192;
constexpr int AT_BITS = 40;
constexpr uint64_t AT_MASK = (1ull << AT_BITS) - 1;
enum { TYPE_F32 = THC_DTYPE_F32, TYPE_BF16 = THC_DTYPE_BF16, TYPE_F16 = THC_DTYPE_F16, TYPE_ZEROS = 3 };

struct TensorTable {
  void* ptr[TABLE];
  uint64_t at[TABLE + 1];     // first element's place in the flat vector, and above AT_BITS the tensor's type
  uint32_t unit[TABLE + 1];   // first unit; behind the last tensor the number of units
  uint32_t count;
};

inline uint32_t type_bytes(uint32_t type) { return type == TYPE_F32 ? 4 : 2; }

inline int validate_tensors(const thc_tensors* t, uint64_t* total) {
  *total = 0;
  if (!t) return THC_EINVAL;
  if (t->count && (!t->data || !t->numel || !t->dtype)) return THC_EINVAL;
  for (uint64_t i = 0; i < t->count; ++i) {
    if (t->dtype[i] > THC_DTYPE_F16 || t->numel[i] > AT_MASK) return THC_EINVAL;
    if (t->numel[i] && (!t->data[i] || reinterpret_cast<uintptr_t>(t->data[i]) % type_bytes(t->dtype[i]))) return THC_EINVAL;
    *total += t->numel[i];
    if (*total > AT_MASK) return THC_EINVAL;
  }
  return THC_OK;
}

// Whether memory that a call writes overlaps other memory of the call: the tensors each other (`each_other`), or the range
// [flat, flat + bytes).  THC_EINVAL if so.
inline int check_overlap(const thc_tensors* t, bool each_other, const void* flat, uint64_t bytes) {
  const uintptr_t f0 = reinterpret_cast<uintptr_t>(flat), f1 = f0 + bytes;
  bool sorted = true;
  uintptr_t last = 0;
  for (uint64_t i = 0; i < t->count; ++i) {
    if (!t->numel[i]) continue;
    const uintptr_t a = reinterpret_cast<uintptr_t>(t->data[i]), b = a + t->numel[i] * type_bytes(t->dtype[i]);
    if (a < f1 && f0 < b) return THC_EINVAL;
    sorted = sorted && a >= last;
    last = b;
  }
  if (!each_other || sorted) return THC_OK;      // in the order of their addresses, one behind the other: nothing left to compare
  try {
    std::vector<std::pair<uintptr_t, uintptr_t>> r;
    r.reserve(t->count);
    for (uint64_t i = 0; i < t->count; ++i) {
      const uintptr_t a = reinterpret_cast<uintptr_t>(t->data[i]);
      if (t->numel[i]) r.emplace_back(a, a + t->numel[i] * type_bytes(t->dtype[i]));
    }
    std::sort(r.begin(), r.end());
    for (size_t i = 1; i < r.size(); ++i)
      if (r[i].first < r[i - 1].second) return THC_EINVAL;
  } catch (const std::bad_alloc&) {
    return THC_EUNSUPPORTED;
  }
  return THC_OK;
}

// Which memory a call's units are aligned to.
enum class Grid { TENSOR, FLAT };

// The tables of a call, one after another: launch(table, units of the table).  Tensors without elements take no place, and one
// that starts where the one before it ends, with the same type, is part of it.  `zeros`: that many zeros follow the last tensor
// in the flat vector.  `flat_bytes`: bytes per element of the flat vector (Grid::FLAT).
template <class Launch>
inline void for_tables(const thc_tensors* t, Grid grid, uint32_t flat_bytes, uint64_t zeros, Launch&& launch) {
  TensorTable tab;
  uint32_t k = 0, units = 0;
  uint64_t at = 0;
  auto flush = [&] {
    if (!k) return;
    tab.at[k] = at;
    tab.unit[k] = units;
    tab.count = k;
    launch(tab, units);
    k = units = 0;
  };
  auto add = [&](void* ptr, uint64_t numel, uint32_t type) {
    // a launch's units are numbered in 32 bits; 2^40 elements are 2^27 units, and a tensor adds at most one
    if (k == TABLE) flush();
    const uint32_t size = grid == Grid::FLAT ? flat_bytes : type_bytes(type);
    const uint64_t addr = grid == Grid::FLAT ? at * size : reinterpret_cast<uintptr_t>(ptr);
    tab.ptr[k] = ptr;
    tab.at[k] = at | (uint64_t)type << AT_BITS;
    tab.unit[k] = units;
    units += (uint32_t)((addr % LINE / size + numel + UNIT - 1) >> LOG_UNIT);
    at += numel;
    ++k;
  };
  void* run = nullptr;
  uint64_t len = 0;
  uint32_t type = 0;
  for (uint64_t i = 0; i < t->count; ++i) {
    if (!t->numel[i]) continue;
    if (len && t->dtype[i] == type && t->data[i] == static_cast<char*>(run) + len * type_bytes(type)) {
      len += t->numel[i];
      continue;
    }
    if (len) add(run, len, type);
    run = t->data[i];
    len = t->numel[i];
    type = t->dtype[i];
  }
  if (len) add(run, len, type);
  if (zeros) add(nullptr, zeros, TYPE_ZEROS);
  flush();
}

}  // namespace thc
