// Host side of the calls that take a list of tensors: validation, and the tables of tensors that travel with each launch.
// Plain C++ (no GPU types), so that it can be built and run under the host sanitizers.
#pragma once

#include <algorithm>
#include <cstdint>
#include <initializer_list>
#include <utility>
#include <vector>

#include "thc.h"

namespace thc {

// The work of a launch is counted in units of a power of two of bytes.  A tensor's units lie on a grid that starts on a 128-byte
// line of what the kernel accesses in whole lines (its own memory, or its place in the flat vector), up to one line before its first
// element, so that no line but a tensor's first and last is shared by two units.
// A move has a workgroup for each unit, in the order of memory, so that consecutive workgroups, which go to the eight XCDs in turn, write
// consecutive 8 KB: us by the unit's bytes, 4 / 8 / 16 / 32 KB, scatter of 553 MB in binary32 176.9 / 180 / 182 / 188, gather of 3.1 GB in
// bf16 1077 / 1040 / 1047 / 1081 (256 to 2048 workgroups that walk the units: 183 to 219, and 1130 to 1254).
// The norm has one workgroup of 512 threads on each of the 256 compute units, which walk the units together: 8 MB in flight are enough, and
// memory answers fewer at a time faster.  us, 1.5 GB in binary32 / bf16: 256 x 512 threads with units of 16 KB 336 / 367, 32 KB 229 / 229,
// 64 KB 240 / 241; 256 x 256 threads 227 / 249 (the multiply-adds of bf16 then take longer than its bytes); 256 x 1024 240 / 243;
// 512 x 256 241 / 241; 1792 x 256 239 / 242; 8192 x 256 237 / 238.  256 MB, plainly read: 256 x 512 44.8 / 45.2, 8192 x 256 48.1 / 48.7.
constexpr uint32_t LINE = 128;
constexpr uint32_t LOG_NORM_UNIT = 15, LOG_MOVE_UNIT = 13, LOG_WAVE_UNIT = 12;

// A launch holds fewer than 2^32 threads, 2^24 workgroups of 256: longer lists take several, and longer tensors several places in
// the table, of whole lines.
constexpr uint32_t MOST_UNITS = 1u << 23;
constexpr uint64_t MOST_NUMEL = 1ull << 33;
static_assert((MOST_NUMEL * 4 >> LOG_MOVE_UNIT) < MOST_UNITS);

// Tensors of one launch, passed by value (a captured graph keeps them): a kernel's arguments have to stay within 4 KB, which 16 bytes
// a tensor let hold 244.  Short lists travel in a table of their own: a third of the arguments to write and, per wave, a quarter of
// the places to look at.
constexpr uint32_t TABLE = 244, SHORT_TABLE = 63;
constexpr int PTR_BITS = 48, AT_BITS = 40;     // of a device address, and of a place in the flat vector
constexpr uint64_t PTR_MASK = (1ull << PTR_BITS) - 1, AT_MASK = (1ull << AT_BITS) - 1;
enum { TYPE_F32 = THC_DTYPE_F32, TYPE_BF16 = THC_DTYPE_BF16, TYPE_F16 = THC_DTYPE_F16, TYPE_ZEROS = 3 };

template <uint32_t N>
struct TensorTable {
  static constexpr uint32_t LANES = (N + 64) / 64;   // places that one of 64 lanes looks at
  uint32_t unit[64 * LANES];   // each tensor's first unit; behind the last one no unit is as large
  uint64_t ptr[N + 1];         // address; above PTR_BITS the upper 8 bits of the place in the flat vector, then the type
  uint32_t at[N + 1];          // the lower 32 bits of the first element's place in the flat vector; behind the last tensor its end
  void set(uint32_t k, const void* p, uint64_t place, uint32_t type, uint32_t first) {
    unit[k] = first;
    ptr[k] = (reinterpret_cast<uintptr_t>(p) & PTR_MASK) | (place >> 32) << PTR_BITS | (uint64_t)type << (PTR_BITS + 8);
    at[k] = (uint32_t)place;
  }
  void end(uint32_t k, uint64_t place) {
    set(k, nullptr, place, 0, ~0u);
    std::fill(unit + k, unit + 64 * LANES, ~0u);
  }
};

inline void shorten(const TensorTable<TABLE>& from, uint32_t count, TensorTable<SHORT_TABLE>* to) {
  std::copy(from.unit, from.unit + 64, to->unit);
  std::copy(from.ptr, from.ptr + count + 1, to->ptr);
  std::copy(from.at, from.at + count + 1, to->at);
}

inline uint32_t type_bytes(uint32_t type) { return type == TYPE_F32 ? 4 : 2; }

// What one walk over a list finds out.  An entry of a launch's table is a run of memory: a tensor that starts where the one before it ends,
// with the same type, is part of it, and tensors without elements take no place.
struct Scan {
  uint64_t total = 0, bytes = 0, entries = 0;
  uintptr_t begin = ~(uintptr_t)0, end = 0;   // all tensors lie between these
  bool ascending = true;                      // in the order of their addresses, none over another
  bool wide = false, narrow = false;          // whether any element has four bytes, and two
};

inline int scan_tensors(const thc_tensors* t, Scan* out) {
  if (!t) return THC_EINVAL;
  if (t->count && (!t->data || !t->numel || !t->dtype)) return THC_EINVAL;
  Scan s;
  uintptr_t last = 0;
  uint32_t type = ~0u;
  for (uint64_t i = 0; i < t->count; ++i) {
    if (t->dtype[i] > THC_DTYPE_F16 || t->numel[i] > AT_MASK) return THC_EINVAL;
    if (!t->numel[i]) continue;
    const uintptr_t a = reinterpret_cast<uintptr_t>(t->data[i]);
    const uint64_t bytes = t->numel[i] * type_bytes(t->dtype[i]);
    if (!a || a >> PTR_BITS || (a & (type_bytes(t->dtype[i]) - 1))) return THC_EINVAL;
    s.entries += a != last || t->dtype[i] != type;
    s.ascending = s.ascending && a >= last;
    s.begin = std::min(s.begin, a);
    s.total += t->numel[i];
    s.bytes += bytes;
    last = a + bytes;
    s.end = std::max(s.end, last);
    type = t->dtype[i];
    (type == TYPE_F32 ? s.wide : s.narrow) = true;
    if (s.total > AT_MASK) return THC_EINVAL;
  }
  *out = s;
  return THC_OK;
}

// whether all elements have that size
inline bool same_size(const Scan& s, uint32_t bytes) { return !(bytes == 4 ? s.narrow : s.wide); }

// Bytes at the start of a list that the norm's pass reads with plain loads, so that the 256 MB memory-side cache holds them for the
// call that moves the list next; the rest is read non-temporally, which is up to 9 % faster and does not push out what is kept.
// us on one binary32 tensor, nothing kept / 256 MB kept (bf16 differs by up to 6 %):
//              8 MB         16 MB         24 MB         32 MB         64 MB         96 MB         224 MB          512 MB           1 GB
//   norm      5.8 / 5.9    6.9 / 7.3     8.2 / 8.7     9.3 / 10.0   13.9 / 15.0   18.4 / 20.0   36.7 / 39.5     78.1 / 81.0    152 / 155
//   + gather 10.8 / 9.9   14.5 / 12.1   18.7 / 14.7   22.8 / 17.1   37.7 / 32.1   52.7 / 46.7   110.9 / 103.7   247.6 / 239.2   493 / 487
//   clip      8.9 / 9.9   13.1 / 13.9   17.1 / 16.8   21.0 / 20.4   36.1 / 32.2   51.2 / 47.4   112.3 / 105.3   247.8 / 242.4   493 / 490
// A norm by itself pays up to 9 % for it.  That no factor is wanted from it tells nothing: norms of several lists may be combined, and the
// list then moved by a factor of the caller's.
inline uint64_t norm_keeps(uint64_t bytes, bool in_place) { return in_place && bytes < 24ull << 20 ? 0 : 256ull << 20; }

// Lists that are scaled behind their norm by its units of 32 KB: a unit is then read by the same one of the eight XCDs, whose L2 may still
// have it, and each wave of the scaling adds the partials up, which saves a launch.  The rest goes by units of 8 KB, behind a launch that
// adds the partials up.  us, units of 8 KB and that launch / units of 32 KB, tensors of binary32 (bf16 differs by up to 5 %):
//                         4 MB          16 MB         32 MB         51 MB         102 MB        127 MB        160 MB         512 MB
//   clipped, one       11.1 / 10.2   15.7 / 14.1   26.2 / 20.6   34.4 / 27.5   54.3 / 49.6   64.2 / 60.9   78.3 / 78.4   242.2 / 248.2
//   clipped, 400       22.3 / 21.0   25.3 / 25.7   34.5 / 32.6   41.8 / 38.2   64.3 / 59.2   74.8 / 69.8
//   below limit, one   11.4 / 9.8    11.5 / 9.8    13.5 / 12.0   16.9 / 14.9   25.0 / 22.4   29.6 / 26.5   35.8 / 32.2    96.9 / 89.0
//   below limit, 400   21.8 / 20.3   23.2 / 21.6   23.3 / 21.8   24.5 / 24.4   33.7 / 32.5   37.7 / 35.7
inline bool behind_norm(uint64_t bytes) { return bytes <= 128ull << 20; }

// Gathers by those units, for the same XCD's sake: those that are given a factor, which as a rule is that of a norm before them.
// us, units of 8 KB / 32 KB, tensors:
//                                 8 MB          12 MB         16 MB         32 MB         51 MB         102 MB        127 MB
//   norm + gather, f32     1   12.2 / 12.0                 14.4 / 13.7   20.6 / 18.6   29.5 / 27.3   51.3 / 49.3   62.1 / 60.6
//                        160   13.8 / 13.9   14.7 / 14.2   17.1 / 15.0   24.1 / 21.6   32.7 / 30.3   57.8 / 54.8   69.0 / 66.1
//                        400                 23.4 / 23.7   24.8 / 24.7   32.5 / 32.7   41.0 / 41.8   65.1 / 65.4   76.7 / 76.5
//                 bf16     1   12.4 / 12.2                 15.0 / 14.1   21.2 / 19.0   29.9 / 28.1   51.9 / 49.9   62.6 / 61.1
//                        160   14.7 / 16.0   15.4 / 14.1   18.1 / 16.8   25.4 / 24.4   34.4 / 33.6   60.5 / 58.4   74.3 / 71.3
//                        400                 25.0 / 26.1   26.3 / 28.1   34.1 / 37.4   43.2 / 46.6   67.9 / 71.6   82.4 / 85.0
//   gather alone, f32    160    6.2 / 7.1     7.6 / 8.2     9.3 / 9.9    14.7 / 15.3   21.3 / 21.3   37.8 / 37.6   45.5 / 45.8
//                 bf16   160    6.6 / 9.7     8.2 / 10.7    9.3 / 12.4   14.6 / 18.2   21.1 / 24.1   37.4 / 41.1   45.7 / 49.0
//                        400                 12.5 / 18.0   13.6 / 19.6   19.1 / 24.4   24.8 / 30.8   42.6 / 49.0   50.2 / 56.5
// Each launch of the large units costs some us that a second launch does not win back, so lists of more than one go by 8 KB, and so do
// short ones, which win nothing behind a norm, and gathers that change the size of their elements, which take longer.  A gather of bf16 by
// a factor with no norm before it is what the rule costs: up to 4 us.
inline bool gather_behind_norm(const Scan& s, uint32_t flat_bytes, uint64_t zeros) {
  return same_size(s, flat_bytes) && s.bytes >= 12ull << 20 && behind_norm(s.bytes) && s.entries + (zeros != 0) <= TABLE;
}

// Shared memory that these gathers ask for and do not use: three workgroups run on a compute unit instead of five.  us of norm and gather,
// nothing asked for / 53000: binary32, 160 tensors 24 MB 18.4 / 18.5, 32 MB 22.2 / 21.6, 51 MB 33.0 / 30.3, 76 MB 45.6 / 42.7, 102 MB
// 57.5 / 54.8, 127 MB 68.6 / 66.1, 40 tensors 51 MB 31.4 / 29.6, 127 MB 67.3 / 65.2; bf16, 160 tensors 51 MB 34.8 / 33.6, 102 MB 59.7 / 58.4,
// 127 MB 72.6 / 71.3; one tensor of either type 32 MB 18.4 / 18.6 and 18.6 / 19.0, from 51 MB on the same.  By themselves these gathers differ
// by up to 3 % one way or the other.  Asking for less does less: binary32, 160 tensors, 102 MB 57.1 / 56.8 / 55.5 / 54.7 with 26000 / 32000 /
// 40000 / 53000.
constexpr uint32_t BEHIND_NORM_LDS = 53000;

// Shared memory that a move of a long list asks for and does not use: 26000 of a compute unit's 160 KB let six workgroups run there instead
// of eight, and memory answers fewer accesses at a time faster.  us, nothing asked for / 26000 / 32000 bytes (six, five workgroups):
// one tensor of 512 MB gather binary32 174.3 / 168.1 / 165.4, bf16 171.5 / 169.2 / 165.7, scatter 172.3 / 166.1 / 166.1, to bf16
// 255.1 / 251.2 / 247.8, clip 244.0 / 242.2 / 241.4; scatter of VGG16's gradient 177.6 / 175.1 / 174.6; gather of GPT-2 XL's 1040 / 1036 /
// 1052, which five are too few for.  At 160 MB gather gains 2 %, at 128 MB nothing; scatter to bf16 loses 1.5 % at 64 and 96 MB.
inline uint32_t move_lds(uint64_t bytes) { return bytes > 128ull << 20 ? 26000 : 0; }

struct Range {
  uintptr_t begin, end;
  Range(const void* p, uint64_t bytes) : begin(reinterpret_cast<uintptr_t>(p)), end(begin + (p ? bytes : 0)) {}
  bool meets(const Range& r) const { return begin < r.end && r.begin < end; }
};

// Whether memory that a call writes overlaps other memory of the call: the tensors each other (`each_other`), or `others`, among which the
// caller has seen to it that nothing overlaps.  THC_EINVAL if so.
inline int check_overlap(const thc_tensors* t, const Scan& s, bool each_other, std::initializer_list<Range> others) {
  for (const Range& o : others) {
    if (o.begin >= s.end || s.begin >= o.end) continue;
    for (uint64_t i = 0; i < t->count; ++i)
      if (t->numel[i] && o.meets(Range(t->data[i], t->numel[i] * type_bytes(t->dtype[i])))) return THC_EINVAL;
  }
  if (!each_other || s.ascending) return THC_OK;
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
  } catch (...) {                                // no memory for it: nothing is thrown through the C entry
    return THC_EUNSUPPORTED;
  }
  return THC_OK;
}

// Which memory a call's units are aligned to.
enum class Grid { TENSOR, FLAT };

// The tables of a call, one after another: launch(table, its tensors, its units).  Longer lists are cut into as many entries a launch: 391
// as 196 and 195, not 244 and 147.  `flat_bytes`: bytes per element of the flat vector (Grid::FLAT).  `zeros`: that many zeros follow the
// last tensor in the flat vector.  `log_unit`: of a unit's bytes.  2.5 ns an entry (and 1.8 for scan_tensors), which every call pays.
template <class Launch>
inline void for_tables(const thc_tensors* t, const Scan& s, Grid grid, uint32_t flat_bytes, uint64_t zeros, uint32_t log_unit, Launch&& launch) {
  const uint64_t entries = s.entries + (zeros != 0), launches = (entries + TABLE - 1) / TABLE;
  const uint32_t most = launches ? (uint32_t)((entries + launches - 1) / launches) : TABLE;
  TensorTable<TABLE> tab;
  uint32_t k = 0, units = 0;
  uint64_t at = 0;
  auto flush = [&] {
    if (!k) return;
    tab.end(k, at);
    launch(tab, k, units);
    k = units = 0;
  };
  uint64_t i = 0;
  while (i < t->count || zeros) {
    const char* ptr = nullptr;
    uint64_t numel = zeros;
    uint32_t type = TYPE_ZEROS;
    if (i < t->count) {
      numel = t->numel[i];
      if (!numel) {
        ++i;
        continue;
      }
      ptr = static_cast<const char*>(t->data[i]);
      type = t->dtype[i];
      for (++i; i < t->count; ++i) {
        if (!t->numel[i]) continue;
        if (t->data[i] != ptr + numel * type_bytes(type) || t->dtype[i] != type) break;
        numel += t->numel[i];
      }
    } else {
      zeros = 0;
    }
    for (uint64_t left = numel; left; left -= numel) {
      numel = left < MOST_NUMEL ? left : MOST_NUMEL;
      const uint32_t size = grid == Grid::FLAT ? flat_bytes : type_bytes(type);
      const uint64_t addr = grid == Grid::FLAT ? at * size : reinterpret_cast<uintptr_t>(ptr);
      const uint32_t own = (uint32_t)((addr % LINE + numel * size + (1u << log_unit) - 1) >> log_unit);
      if (k == most || units + own > MOST_UNITS) flush();
      tab.set(k++, ptr, at, type, units);
      units += own;
      at += numel;
      if (ptr) ptr += numel * type_bytes(type);
    }
  }
  flush();
}

}  // namespace thc
