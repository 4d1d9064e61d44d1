// Kernels between a model's tensors and the flat vectors of the path: the global norm of a list of tensors, scaling it in place,
// gathering it into a flat vector and scattering one over it.  All are bound by memory; none has more than one operation per
// element but for the norm's conversion and multiply-add in binary64.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "thc_device.hpp"
#include "thc_tensorplan.hpp"

namespace thc {

constexpr int TNT = 256;              // threads per workgroup
constexpr uint32_t NORM_PARTIALS = 2048;   // most workgroups of a norm launch: one partial each
constexpr int FINAL_NT = 1024;

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

// N consecutive elements, aligned as one of them is: one access of up to 16 bytes (the GPU takes global accesses of any alignment)
template <class T, int N>
struct __attribute__((packed, aligned(sizeof(T)))) Pack { T x[N]; };

// The tensor that a unit belongs to, and the unit's place in it.
struct Piece {
  char* ptr;
  uint64_t at;      // of the tensor's first element in the flat vector
  uint64_t numel;
  int64_t lo;       // the unit's first element, counted from the tensor's: negative where the grid starts before it
  uint32_t type;
};

// Each wave counts the tensors that start at or before the unit, 64 at a time.
template <Grid GRID, uint32_t FLAT_BYTES>
__device__ __forceinline__ Piece locate(const TensorTable& tab, uint32_t u) {
  const uint32_t lane = threadIdx.x & 63u;
  uint32_t n = 0;
#pragma unroll
  for (uint32_t k = 0; k < TABLE; k += 64) {
    const bool before = k + lane < tab.count && tab.unit[k + lane] <= u;
    n += (uint32_t)__popcll(__ballot(before));
  }
  const uint32_t i = __builtin_amdgcn_readfirstlane(n - 1u);
  Piece p;
  const uint64_t at = tab.at[i];
  p.ptr = static_cast<char*>(tab.ptr[i]);
  p.at = at & AT_MASK;
  p.type = (uint32_t)(at >> AT_BITS);
  p.numel = (tab.at[i + 1] & AT_MASK) - p.at;
  const uint32_t size = GRID == Grid::FLAT ? FLAT_BYTES : p.type == TYPE_F32 ? 4 : 2;
  const uint64_t addr = GRID == Grid::FLAT ? p.at * size : reinterpret_cast<uintptr_t>(p.ptr);
  p.lo = ((int64_t)(u - tab.unit[i]) << LOG_UNIT) - (int64_t)(addr % LINE / size);
  return p;
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

template <int KIND>
__device__ __forceinline__ double wave_join(double v) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) v = Acc<KIND>::join(v, __shfl_xor(v, m, 64));
  return v;
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

template <int KIND, class T>
__device__ __forceinline__ void norm_unit(const Piece& p, Acc<KIND>& acc) {
  constexpr int V = 16 / sizeof(T), S = UNIT / V / TNT;
  const T* const x = reinterpret_cast<const T*>(p.ptr) + p.lo;
  const uint32_t t = threadIdx.x * V;
  if (p.lo >= 0 && (uint64_t)p.lo + UNIT <= p.numel) {
    Pack<T, V> v[S];
#pragma unroll
    for (int k = 0; k < S; ++k) v[k] = *reinterpret_cast<const Pack<T, V>*>(x + (t + k * TNT * V));
#pragma unroll
    for (int k = 0; k < S; ++k)
#pragma unroll
      for (int e = 0; e < V; ++e) acc.add(widen(v[k].x[e]));
    return;
  }
#pragma unroll 1
  for (int k = 0; k < S; ++k) {
    const int64_t j = p.lo + t + k * TNT * V;
    if (j >= 0 && (uint64_t)j + V <= p.numel) {
      const Pack<T, V> v = *reinterpret_cast<const Pack<T, V>*>(x + (t + k * TNT * V));
#pragma unroll
      for (int e = 0; e < V; ++e) acc.add(widen(v.x[e]));
    } else {
#pragma unroll 1
      for (int e = 0; e < V; ++e)
        if (j + e >= 0 && (uint64_t)(j + e) < p.numel) acc.add(widen(x[t + k * TNT * V + e]));
    }
  }
}

struct NormArgs {
  double* partials;
  uint32_t units;
  uint32_t before;      // partials that an earlier launch of the call has written: these are added to
  TensorTable tab;
};
static_assert(sizeof(NormArgs) <= 4096, "kernel arguments");

template <int KIND>
__global__ __launch_bounds__(TNT) void k_norm(const NormArgs a) {
  Acc<KIND> acc;
  for (uint32_t u = blockIdx.x; u < a.units; u += gridDim.x) {
    const Piece p = locate<Grid::TENSOR, 0>(a.tab, u);
    if (p.type == TYPE_F32) norm_unit<KIND, float>(p, acc);
    else if (p.type == TYPE_BF16) norm_unit<KIND, Bf16>(p, acc);
    else norm_unit<KIND, F16>(p, acc);
  }
  const double v = group_join<KIND, TNT>(acc.get());
  if (threadIdx.x == 0) a.partials[blockIdx.x] = blockIdx.x < a.before ? Acc<KIND>::join(a.partials[blockIdx.x], v) : v;
}

// the norm and the factor that clips by it, from the partials
template <int KIND, int N>
__device__ __forceinline__ double norm_of(const double* partials, uint32_t count) {
  double v = 0.0;
  for (uint32_t i = threadIdx.x; i < count; i += N) v = Acc<KIND>::join(v, partials[i]);
  v = group_join<KIND, N>(v);
  return KIND == THC_NORM_L2 ? __builtin_sqrt(v) : v;
}
__device__ __forceinline__ float clip_factor(double norm, float max_norm) {
  return norm <= (double)max_norm ? 1.f : (float)((double)max_norm / norm);
}

struct NormOut {
  float* norm;
  float* scale;         // or null
  float max_norm;
  uint32_t count;       // partials
  const double* partials;
};

template <int KIND>
__global__ __launch_bounds__(FINAL_NT) void k_norm_final(const NormOut o) {
  const double v = norm_of<KIND, FINAL_NT>(o.partials, o.count);
  if (threadIdx.x == 0) {
    *o.norm = (float)v;
    if (o.scale) *o.scale = clip_factor(v, o.max_norm);
  }
}

// ---- moves --------------------------------------------------------------------------------------------------------
// dst[j] = round(src[j] * c) over one unit, whole 16-byte stores but at a tensor's ends
template <class S, class D>
__device__ __forceinline__ void move_unit(const S* src, D* dst, int64_t lo, uint64_t numel, float c) {
  constexpr int V = 16 / sizeof(D), K = UNIT / V / TNT;
  src += lo;
  dst += lo;
  const uint32_t t = threadIdx.x * V;
  if (lo >= 0 && (uint64_t)lo + UNIT <= numel) {
    Pack<S, V> v[K];
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = *reinterpret_cast<const Pack<S, V>*>(src + (t + k * TNT * V));
#pragma unroll
    for (int k = 0; k < K; ++k) {
      Pack<D, V> o;
#pragma unroll
      for (int e = 0; e < V; ++e) o.x[e] = narrow<D>(widen(v[k].x[e]) * c);
      *reinterpret_cast<Pack<D, V>*>(__builtin_assume_aligned(dst + (t + k * TNT * V), 16)) = o;
    }
    return;
  }
#pragma unroll 1
  for (int k = 0; k < K; ++k) {
    const uint32_t i = t + k * TNT * V;
    const int64_t j = lo + i;
#pragma unroll 1
    for (int e = 0; e < V; ++e)
      if (j + e >= 0 && (uint64_t)(j + e) < numel) dst[i + e] = narrow<D>(widen(src[i + e]) * c);
  }
}

struct ClipArgs {
  NormOut out;
  uint32_t units;
  uint32_t first;       // 1 in the launch that writes the norm
  TensorTable tab;
};
static_assert(sizeof(ClipArgs) <= 4096, "kernel arguments");

template <int KIND>
__global__ __launch_bounds__(TNT) void k_clip(const ClipArgs a) {
  const double v = norm_of<KIND, TNT>(a.out.partials, a.out.count);
  const float c = clip_factor(v, a.out.max_norm);
  if (a.first && blockIdx.x == 0 && threadIdx.x == 0) {
    *a.out.norm = (float)v;
    if (a.out.scale) *a.out.scale = c;
  }
  if (c == 1.f) return;
  for (uint32_t u = blockIdx.x; u < a.units; u += gridDim.x) {
    const Piece p = locate<Grid::TENSOR, 0>(a.tab, u);
    if (p.type == TYPE_F32) move_unit(reinterpret_cast<const float*>(p.ptr), reinterpret_cast<float*>(p.ptr), p.lo, p.numel, c);
    else if (p.type == TYPE_BF16) move_unit(reinterpret_cast<const Bf16*>(p.ptr), reinterpret_cast<Bf16*>(p.ptr), p.lo, p.numel, c);
    else move_unit(reinterpret_cast<const F16*>(p.ptr), reinterpret_cast<F16*>(p.ptr), p.lo, p.numel, c);
  }
}

struct GatherArgs {
  void* flat;
  const float* scale;   // or null
  uint32_t units;
  TensorTable tab;
};
static_assert(sizeof(GatherArgs) <= 4096, "kernel arguments");

template <class D>
__global__ __launch_bounds__(TNT) void k_gather(const GatherArgs a) {
  const float c = a.scale ? *a.scale : 1.f;
  for (uint32_t u = blockIdx.x; u < a.units; u += gridDim.x) {
    const Piece p = locate<Grid::FLAT, sizeof(D)>(a.tab, u);
    D* const dst = static_cast<D*>(a.flat) + p.at;
    if (p.type == TYPE_F32) move_unit(reinterpret_cast<const float*>(p.ptr), dst, p.lo, p.numel, c);
    else if (p.type == TYPE_BF16) move_unit(reinterpret_cast<const Bf16*>(p.ptr), dst, p.lo, p.numel, c);
    else if (p.type == TYPE_F16) move_unit(reinterpret_cast<const F16*>(p.ptr), dst, p.lo, p.numel, c);
    else
      for (uint32_t i = threadIdx.x; i < UNIT; i += TNT)
        if (p.lo + i >= 0 && (uint64_t)(p.lo + i) < p.numel) dst[p.lo + i] = narrow<D>(0.f);
  }
}

struct ScatterArgs {
  const float* flat;
  const float* scale;   // or null
  uint32_t units;
  TensorTable tab;
};
static_assert(sizeof(ScatterArgs) <= 4096, "kernel arguments");

__global__ __launch_bounds__(TNT) void k_scatter(const ScatterArgs a) {
  const float c = a.scale ? *a.scale : 1.f;
  for (uint32_t u = blockIdx.x; u < a.units; u += gridDim.x) {
    const Piece p = locate<Grid::TENSOR, 0>(a.tab, u);
    const float* const src = a.flat + p.at;
    if (p.type == TYPE_F32) move_unit(src, reinterpret_cast<float*>(p.ptr), p.lo, p.numel, c);
    else if (p.type == TYPE_BF16) move_unit(src, reinterpret_cast<Bf16*>(p.ptr), p.lo, p.numel, c);
    else move_unit(src, reinterpret_cast<F16*>(p.ptr), p.lo, p.numel, c);
  }
}

}  // namespace thc
