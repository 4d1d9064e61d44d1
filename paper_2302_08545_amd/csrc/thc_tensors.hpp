// Kernels between a model's tensors and the flat vectors of the path: the global norm of a list of tensors, scaling it in place,
// gathering it into a flat vector and scattering one over it.
//
//   norm     v = sqrt(sum x^2) in binary64, or max |x|;  c = 1 where v <= max_norm, else max_norm / v, rounded once to binary32
//   moves    y = round(fl32(x * c)): the product rounded to binary32, then to the type, as elementary operations would
//
// Bound by memory, with one operation per element (the norm: a conversion and a multiply-add in binary64, a quarter of the ALU at full
// rate); small lists by launches.  Rates of large lists (MI355X): the norm reads 6.9 TB/s (7.3 from one tensor of 4 GB), moves 6.0 to 6.4.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "thc_device.hpp"
#include "thc_tensorplan.hpp"

namespace thc {

constexpr int TNT = 256;                   // threads per workgroup of a move
// A norm launch has at most one workgroup, and one partial, for each of the GPU's 256 compute units.
constexpr int NORM_NT = 512, ONE_NT = 1024;
constexpr uint32_t NORM_PARTIALS = 256;

struct Bf16 { uint16_t bits; };
struct F16 { _Float16 v; };
__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(Bf16 x) { return bf16_to_f32(x.bits); }
__device__ __forceinline__ float widen(F16 x) { return (float)x.v; }
template <class T> __device__ __forceinline__ T narrow(float x);
template <> __device__ __forceinline__ float narrow<float>(float x) { return x; }
template <> __device__ __forceinline__ Bf16 narrow<Bf16>(float x) { return Bf16{__builtin_bit_cast(uint16_t, (__bf16)x)}; }
template <> __device__ __forceinline__ F16 narrow<F16>(float x) {
  asm("" : "+v"(x));   // the product is rounded to binary32 first, as everywhere: a fused multiply and conversion would round it once
  return F16{(_Float16)x};
}

template <class T, uint32_t N>
struct Pack { T x[N]; };

template <int WORDS, int ALIGN> struct Words;
template <> struct Words<2, 2> { typedef uint32_t type __attribute__((ext_vector_type(2), aligned(2))); };
template <> struct Words<4, 2> { typedef uint32_t type __attribute__((ext_vector_type(4), aligned(2))); };
template <> struct Words<4, 4> { typedef uint32_t type __attribute__((ext_vector_type(4), aligned(4))); };

// N consecutive elements, non-temporal, aligned as one of them is: the GPU takes global accesses of any alignment
template <class T, int N>
__device__ __forceinline__ Pack<T, N> load_pack(const T* p) {
  using U = typename Words<sizeof(T) * N / 4, sizeof(T)>::type;
  const U v = __builtin_nontemporal_load(reinterpret_cast<const U*>(p));
  return __builtin_bit_cast(Pack<T, N>, v);
}

// Non-temporal, aligned to its size.  Plain stores would leave the lines to whoever reads them next, but they cost the call more: gather
// of 128 MB 45.1 -> 48.7 us, with the norm before it 60.6 -> 77.8, scatter of 128 MB 43.3 -> 48.3, scaling in place 66.2 -> 86.8.  Together
// with the next reading, us plain / non-temporal: norm, gather and compress 32 MB 46.2 / 46.9, 128 MB 138 / 142, 256 MB 266 / 262, bf16
// 128 MB 179 / 178; decompress, scatter and an addition to every tensor 32 MB 54.7 / 55.8, 128 MB 166 / 172, 512 MB 656 / 649; scaling in
// place and the addition 64 MB 58.0 / 58.0.
template <class T, int N>
__device__ __forceinline__ void store_pack(T* p, const Pack<T, N>& v) {
  typedef uint32_t U __attribute__((ext_vector_type(sizeof(T) * N / 4)));
  __builtin_nontemporal_store(__builtin_bit_cast(U, v), reinterpret_cast<U*>(p));
}

// The tensor that a unit belongs to, and the unit's place in it.
struct Piece {
  char* ptr;
  uint64_t at;      // of the tensor's first element in the flat vector
  int64_t len;      // of the tensor, in bytes of the memory that the grid goes by
  int64_t lo;       // the unit's first byte there, counted from the tensor's: negative where the grid starts before it
  uint32_t type;
};

// Each wave counts the tensors that start at or before the unit: a lane reads the starts of a few in one access.
template <uint32_t LOG_UNIT, Grid GRID, uint32_t FLAT_BYTES, class Table>
__device__ __forceinline__ Piece locate(const Table& tab, uint32_t u) {
  const auto starts = reinterpret_cast<const Pack<uint32_t, Table::LANES>*>(tab.unit)[threadIdx.x & 63u];
  uint32_t n = 0;
#pragma unroll
  for (uint32_t k = 0; k < Table::LANES; ++k) n += (uint32_t)__popcll(__ballot(starts.x[k] <= u));
  const uint32_t i = __builtin_amdgcn_readfirstlane(n - 1u);
  const uint64_t w = tab.ptr[i], next = tab.ptr[i + 1];
  const uint32_t lo = tab.at[i], lo_next = tab.at[i + 1];
  Piece p;
  p.ptr = (char*)(__attribute__((address_space(1))) char*)(w & PTR_MASK);   // global memory: a plain cast leaves that open, and the accesses slower
  p.at = (w >> PTR_BITS & 0xFF) << 32 | lo;
  p.type = (uint32_t)(w >> (PTR_BITS + 8));
  const uint32_t size = GRID == Grid::FLAT ? FLAT_BYTES : p.type == TYPE_F32 ? 4 : 2;
  p.len = (int64_t)((((next >> PTR_BITS & 0xFF) << 32 | lo_next) - p.at) * size);
  const uint64_t addr = GRID == Grid::FLAT ? p.at * size : w;
  p.lo = (int64_t)((uint64_t)(u - tab.unit[i]) << LOG_UNIT) - (int64_t)(addr % LINE);
  return p;
}

// Units are cut into slots of SLOT bytes that lie on the grid.  The elements in front of a tensor's first whole slot and behind its
// last one are taken one to a thread: the offset of this thread's, in bytes, or -1.
template <uint32_t LOG_UNIT, int N, int SLOT, int SIZE>
__device__ __forceinline__ int64_t edge(const Piece& p) {
  constexpr int E = SLOT / SIZE;
  static_assert(2 * E <= N);
  const int t = (int)(threadIdx.x % N);
  const int64_t first = p.lo < 0 ? p.lo & (SLOT - 1) : 0;          // where the first whole slot starts
  const int64_t last = p.len - ((p.len - p.lo) & (SLOT - 1));      // where the last one ends
  if (t < E) return p.lo < 0 && t * SIZE < first && t * SIZE < p.len ? t * SIZE : -1;
  const int64_t j = last + (t - E) * SIZE;
  return t < 2 * E && last >= first && last - p.lo < (1 << LOG_UNIT) && j < p.len ? j : -1;
}
__device__ __forceinline__ bool whole(const Piece& p, int64_t bytes) { return p.lo >= 0 && p.lo + bytes <= p.len; }
template <int SLOT>
__device__ __forceinline__ bool whole_slot(const Piece& p, uint32_t at) {
  return p.lo + at >= 0 && p.lo + at + SLOT <= p.len;
}

// ---- norm ---------------------------------------------------------------------------------------------------------
// L2: squares of binary32 values are exact in binary64, and so are those of bf16 and f16.  MAX: magnitudes as bit patterns,
// whose order is that of the magnitudes, with NaN above infinity.
template <int KIND> struct Acc;
template <> struct Acc<THC_NORM_L2> {
  double v = 0.0;
  __device__ __forceinline__ void add(float x) { v = __builtin_fma((double)x, (double)x, v); }
  __device__ __forceinline__ double get() const { return v; }
  static __device__ __forceinline__ double join(double a, double b) { return a + b; }
};
template <> struct Acc<THC_NORM_MAX> {
  uint32_t v = 0;
  __device__ __forceinline__ void add(float x) {
    const uint32_t m = __float_as_uint(x) & 0x7FFFFFFFu;
    v = m > v ? m : v;
  }
  __device__ __forceinline__ double get() const { return (double)__uint_as_float(v); }
  static __device__ __forceinline__ double join(double a, double b) {
    return __double_as_longlong(a) > __double_as_longlong(b) ? a : b;   // both are positive
  }
};

template <int CTRL>
__device__ __forceinline__ double dpp(double v) {
  const uint64_t w = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_mov_dpp((int)w, CTRL, 0xF, 0xF, true), hi = (uint32_t)__builtin_amdgcn_mov_dpp((int)(w >> 32), CTRL, 0xF, 0xF, true);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// Fixed order; every lane gets the total.  The first four exchanges pair lanes, pairs, fours and eights inside a row of 16.
template <int KIND>
__device__ __forceinline__ double wave_join(double v) {
  v = Acc<KIND>::join(v, dpp<0xB1>(v));    // lane ^ 1
  v = Acc<KIND>::join(v, dpp<0x4E>(v));    // lane ^ 2
  v = Acc<KIND>::join(v, dpp<0x141>(v));   // the other four of eight
  v = Acc<KIND>::join(v, dpp<0x140>(v));   // the other eight of sixteen
  v = Acc<KIND>::join(v, __shfl_xor(v, 16, 64));
  return Acc<KIND>::join(v, __shfl_xor(v, 32, 64));
}

// fixed order; every thread of the workgroup gets the total
template <int KIND, int N>
__device__ __forceinline__ double group_join(double v) {
  __shared__ double part[N / 64];
  v = wave_join<KIND>(v);
  if ((threadIdx.x & 63u) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  v = part[0];
#pragma unroll
  for (int w = 1; w < N / 64; ++w) v = Acc<KIND>::join(v, part[w]);
  return v;
}

template <class T, int S, class A>
__device__ __forceinline__ void add_words(const uint4 (&v)[S], uint32_t one, A& acc) {
  acc.add(widen(__builtin_bit_cast(Pack<T, 4 / sizeof(T)>, one).x[0]));
#pragma unroll
  for (int k = 0; k < S; ++k) {
    const auto x = __builtin_bit_cast(Pack<T, 16 / sizeof(T)>, v[k]);
#pragma unroll
    for (int e = 0; e < 16 / (int)sizeof(T); ++e) acc.add(widen(x.x[e]));
    __builtin_amdgcn_sched_barrier(0);   // 16 bytes after the other: all of them widened at once do not fit the registers
  }
}

// One unit, by N threads: its words are read the same way whatever they hold.
template <uint32_t LOG_UNIT, int N, class A>
__device__ __forceinline__ void norm_unit(const Piece& p, bool keep, A& acc) {
  constexpr int S = (1 << LOG_UNIT) / 16 / N;
  const char* const x = p.ptr + p.lo;
  uint32_t t = threadIdx.x % N * 16;
  asm("" : "+v"(t));   // offsets that are not worth a register between two units
  uint4 v[S];
  uint32_t one = 0;
  if (!whole(p, 1 << LOG_UNIT)) {
    const int64_t e = p.type == TYPE_F32 ? edge<LOG_UNIT, N, 16, 4>(p) : edge<LOG_UNIT, N, 16, 2>(p);
    if (e >= 0) one = p.type == TYPE_F32 ? *reinterpret_cast<const uint32_t*>(p.ptr + e) : *reinterpret_cast<const uint16_t*>(p.ptr + e);
#pragma unroll
    for (int k = 0; k < S; ++k) {
      v[k] = make_uint4(0, 0, 0, 0);
      if (whole_slot<16>(p, t + k * N * 16)) v[k] = load_u4<KEEP>(x + (t + k * N * 16));
    }
  } else if (keep) {
#pragma unroll
    for (int k = 0; k < S; ++k) v[k] = load_u4<KEEP>(x + (t + k * N * 16));
  } else {
#pragma unroll
    for (int k = 0; k < S; ++k) v[k] = load_u4<STREAM>(x + (t + k * N * 16));
  }
  if (p.type == TYPE_F32) add_words<float>(v, one, acc);
  else if (p.type == TYPE_BF16) add_words<Bf16>(v, one, acc);
  else add_words<F16>(v, one, acc);
}

template <class Table>
struct NormArgs {
  Table tab;
  double* partials;
  uint32_t units;
  uint32_t keep;        // units that the caches are to hold on to: the launch's first ones
  uint32_t before;      // partials that an earlier launch of the call has written: these are added to
};
static_assert(sizeof(NormArgs<TensorTable<TABLE>>) <= 4096, "kernel arguments");

template <int KIND, class Table>
__global__ __launch_bounds__(NORM_NT) void k_norm(const NormArgs<Table> a) {
  Acc<KIND> acc;
  for (uint32_t u = blockIdx.x; u < a.units; u += gridDim.x) {
    const Piece p = locate<LOG_NORM_UNIT, Grid::TENSOR, 0>(a.tab, u);
    norm_unit<LOG_NORM_UNIT, NORM_NT>(p, u < a.keep, acc);
  }
  const double v = group_join<KIND, NORM_NT>(acc.get());
  if (threadIdx.x == 0) a.partials[blockIdx.x] = blockIdx.x < a.before ? Acc<KIND>::join(a.partials[blockIdx.x], v) : v;
}

struct NormOut {
  float* norm;
  float* scale;         // or null
  float max_norm;
};

// the factor that clips, from the sum of squares or the largest magnitude; one thread of the launch writes both
template <int KIND>
__device__ __forceinline__ float finish(const NormOut& o, double v, bool writes) {
  const double limit = o.max_norm;
  // a sum that exceeds the limit's square by less than its root's rounding has the factor 1 too, by way of the quotient
  if (!writes && v <= (KIND == THC_NORM_L2 ? limit * limit : limit)) return 1.f;
  const double norm = KIND == THC_NORM_L2 ? __builtin_sqrt(v) : v;
  const float c = norm <= limit ? 1.f : (float)(limit / norm);
  if (writes) {
    *o.norm = (float)norm;
    if (o.scale) *o.scale = c;
  }
  return c;
}

// the partials added up by a wave, which gets the total in every lane
template <int KIND>
__device__ __forceinline__ double join_partials(const double* partials, uint32_t count) {
  const uint32_t lane = threadIdx.x & 63u;
  double x[NORM_PARTIALS / 64];
#pragma unroll
  for (uint32_t k = 0; k < NORM_PARTIALS / 64; ++k) x[k] = lane + 64 * k < count ? partials[lane + 64 * k] : 0.0;
  double v = x[0];
#pragma unroll
  for (uint32_t k = 1; k < NORM_PARTIALS / 64; ++k) v = Acc<KIND>::join(v, x[k]);
  return wave_join<KIND>(v);
}

struct FinalArgs {
  NormOut out;
  const double* partials;
  uint32_t count;
};

template <int KIND>
__global__ __launch_bounds__(64) void k_norm_final(const FinalArgs a) {
  finish<KIND>(a.out, join_partials<KIND>(a.partials, a.count), threadIdx.x == 0);
}

// ---- moves --------------------------------------------------------------------------------------------------------
// dst[j] = round(src[j] * c) over one unit of dst, by N threads: whole lines but at a tensor's ends
template <uint32_t LOG_UNIT, int N, class S, class D>
__device__ __forceinline__ void move_unit(const S* src, D* dst, const Piece& p, float c) {
  constexpr int V = 16 / (sizeof(S) > sizeof(D) ? sizeof(S) : sizeof(D)), SLOT = V * sizeof(D), K = (1 << LOG_UNIT) / SLOT / N;
  const S* const x = src + (p.lo >> (sizeof(D) / 2));            // a whole number of elements
  D* const y = dst + (p.lo >> (sizeof(D) / 2));
  const uint32_t t = threadIdx.x % N * V;
  auto scaled = [&](const Pack<S, V>& v) {
    Pack<D, V> o;
#pragma unroll
    for (int e = 0; e < V; ++e) o.x[e] = narrow<D>(widen(v.x[e]) * c);
    return o;
  };
  Pack<S, V> v[K];
  if (whole(p, 1 << LOG_UNIT)) {
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = load_pack<S, V>(x + (t + k * N * V));
#pragma unroll
    for (int k = 0; k < K; ++k) store_pack<D, V>(y + (t + k * N * V), scaled(v[k]));
    return;
  }
  const int64_t at = edge<LOG_UNIT, N, SLOT, sizeof(D)>(p);
  S one{};
  if (at >= 0) one = src[at >> (sizeof(D) / 2)];
#pragma unroll
  for (int k = 0; k < K; ++k)
    if (whole_slot<SLOT>(p, (t + k * N * V) * sizeof(D))) v[k] = load_pack<S, V>(x + (t + k * N * V));
  if (at >= 0) dst[at >> (sizeof(D) / 2)] = narrow<D>(widen(one) * c);
#pragma unroll
  for (int k = 0; k < K; ++k)
    if (whole_slot<SLOT>(p, (t + k * N * V) * sizeof(D))) store_pack<D, V>(y + (t + k * N * V), scaled(v[k]));
}

// zeros, likewise
template <uint32_t LOG_UNIT, class D>
__device__ __forceinline__ void zero_unit(D* dst, const Piece& p) {
  constexpr int V = 16 / sizeof(D), K = (1 << LOG_UNIT) / 16 / TNT;
  const int64_t e = edge<LOG_UNIT, TNT, 16, sizeof(D)>(p);
  if (e >= 0) dst[e >> (sizeof(D) / 2)] = D{};
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const uint32_t i = (threadIdx.x + k * TNT) * V;
    if (whole_slot<16>(p, i * sizeof(D))) store_pack<D, V>(dst + ((p.lo >> (sizeof(D) / 2)) + i), Pack<D, V>{});
  }
}

template <uint32_t LOG_UNIT, int N>
__device__ __forceinline__ void scale_piece(const Piece& p, float c) {
  if (p.type == TYPE_F32) move_unit<LOG_UNIT, N>(reinterpret_cast<const float*>(p.ptr), reinterpret_cast<float*>(p.ptr), p, c);
  else if (p.type == TYPE_BF16) move_unit<LOG_UNIT, N>(reinterpret_cast<const Bf16*>(p.ptr), reinterpret_cast<Bf16*>(p.ptr), p, c);
  else move_unit<LOG_UNIT, N>(reinterpret_cast<const F16*>(p.ptr), reinterpret_cast<F16*>(p.ptr), p, c);
}

// flat: the vector, or null where the tensors are scaled in place
template <class Table>
struct MoveArgs {
  Table tab;
  void* flat;
  const float* scale;   // or null
};
static_assert(sizeof(MoveArgs<TensorTable<TABLE>>) <= 4096, "kernel arguments");

// Scaling with the partials added up by each wave: the launch of k_norm_final is saved (see behind_norm).
template <class Table>
struct FinishArgs {
  Table tab;
  NormOut out;
  const double* partials;
  uint32_t count;
};

template <int KIND, class Table>
__global__ __launch_bounds__(TNT, 4) void k_finish_scale(const FinishArgs<Table> a) {
  const float c = finish<KIND>(a.out, join_partials<KIND>(a.partials, a.count), blockIdx.x == 0 && threadIdx.x == 0);
  if (c == 1.f) return;
  scale_piece<LOG_NORM_UNIT, TNT>(locate<LOG_NORM_UNIT, Grid::TENSOR, 0>(a.tab, blockIdx.x), c);
}

template <class Table>
__global__ __launch_bounds__(TNT, 8) void k_scale(const MoveArgs<Table> a) {
  const float c = *a.scale;
  if (c == 1.f) return;
  scale_piece<LOG_MOVE_UNIT, TNT>(locate<LOG_MOVE_UNIT, Grid::TENSOR, 0>(a.tab, blockIdx.x), c);
}

// units of LOG_NORM_UNIT: lists whose elements have the vector's size
template <uint32_t LOG_UNIT, class D, class Table>
__global__ __launch_bounds__(TNT, LOG_UNIT == LOG_MOVE_UNIT ? 8 : 4) void k_gather(const MoveArgs<Table> a) {
  constexpr bool WIDE = LOG_UNIT == LOG_MOVE_UNIT || sizeof(D) == 4, NARROW = LOG_UNIT == LOG_MOVE_UNIT || sizeof(D) == 2;
  const float c = a.scale ? *a.scale : 1.f;
  const Piece p = locate<LOG_UNIT, Grid::FLAT, sizeof(D)>(a.tab, blockIdx.x);
  D* const dst = static_cast<D*>(a.flat) + p.at;
  if (p.type == TYPE_ZEROS) zero_unit<LOG_UNIT>(dst, p);
  if constexpr (WIDE) {
    if (p.type == TYPE_F32) move_unit<LOG_UNIT, TNT>(reinterpret_cast<const float*>(p.ptr), dst, p, c);
  }
  if constexpr (NARROW) {
    if (p.type == TYPE_BF16) move_unit<LOG_UNIT, TNT>(reinterpret_cast<const Bf16*>(p.ptr), dst, p, c);
    else if (p.type == TYPE_F16) move_unit<LOG_UNIT, TNT>(reinterpret_cast<const F16*>(p.ptr), dst, p, c);
  }
}

template <class Table>
__global__ __launch_bounds__(TNT, 8) void k_scatter(const MoveArgs<Table> a) {
  const float c = a.scale ? *a.scale : 1.f;
  const Piece p = locate<LOG_MOVE_UNIT, Grid::TENSOR, 0>(a.tab, blockIdx.x);
  const float* const src = static_cast<const float*>(a.flat) + p.at;
  if (p.type == TYPE_F32) move_unit<LOG_MOVE_UNIT, TNT>(src, reinterpret_cast<float*>(p.ptr), p, c);
  else if (p.type == TYPE_BF16) move_unit<LOG_MOVE_UNIT, TNT>(src, reinterpret_cast<Bf16*>(p.ptr), p, c);
  else move_unit<LOG_MOVE_UNIT, TNT>(src, reinterpret_cast<F16*>(p.ptr), p, c);
}

// ---- small lists ----------------------------------------------------------------------------------------------------
// One workgroup, a unit to a wave, takes a list through the norm and, with SCALE, the scaling.  With up to two units a wave it is done
// before the two launches would be.  us, this / the launches: binary32, 4 KB in one tensor 2.3 / 3.8 (with the scaling 2.2 / 3.8), 64 KB in 8
// 2.8 / 4.2 (2.6 / 4.3), 128 KB in one 3.6 / 3.9 (3.4 / 3.9); bf16 128 KB 4.4 / 4.0 (4.5 / 4.3), in 8 4.3 / 4.4 (4.4 / 4.6); three units a
// wave: 4 KB in 48 tensors 5.3 / 4.2 (5.2 / 4.5), bf16 6.6 / 4.7 (7.1 / 4.9); four: 256 KB 5.2 / 4.0 (5.0 / 4.2).
constexpr uint32_t ONE_MOST_UNITS = 2 * ONE_NT / 64;

struct OneArgs {
  TensorTable<SHORT_TABLE> tab;
  NormOut out;
  uint32_t units;
};

template <int KIND, bool SCALE>
__global__ __launch_bounds__(ONE_NT) void k_norm_one(const OneArgs a) {
  const uint32_t wave = threadIdx.x >> 6;
  Acc<KIND> acc;
  for (uint32_t u = wave; u < a.units; u += ONE_NT / 64)
    norm_unit<LOG_WAVE_UNIT, 64>(locate<LOG_WAVE_UNIT, Grid::TENSOR, 0>(a.tab, u), true, acc);
  const float c = finish<KIND>(a.out, group_join<KIND, ONE_NT>(acc.get()), threadIdx.x == 0);   // behind a barrier: everything has been read
  if constexpr (SCALE) {
    if (c == 1.f) return;
    for (uint32_t u = wave; u < a.units; u += ONE_NT / 64)
      scale_piece<LOG_WAVE_UNIT, 64>(locate<LOG_WAVE_UNIT, Grid::TENSOR, 0>(a.tab, u), c);
  }
}

}  // namespace thc
