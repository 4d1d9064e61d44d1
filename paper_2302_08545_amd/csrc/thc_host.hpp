// What the entry points share on the host: checks of arguments and of launches.
#pragma once

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <cstdio>

#include "thc.h"

namespace thc {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline int validate(const thc_params* p) {
  if (!p) return THC_EINVAL;
  if (p->block < (1ull << 10) || p->block > (1ull << 27) || (p->block & (p->block - 1))) return THC_EINVAL;
  if (p->d == 0 || p->d % p->block || p->d >> 40) return THC_EINVAL;   // grids are 32-bit tile counts
  if (p->n < 1) return THC_EINVAL;
  if (p->n > THC_MAX_WORKERS) return THC_EUNSUPPORTED;
  if (p->b < 1 || p->b > 8) return THC_EINVAL;
  if (p->g < (1u << p->b) - 1 || p->g > 255) return THC_EINVAL;
  if (p->agg_bits < 1 || p->agg_bits > 16) return THC_EINVAL;
  if (p->in_dtype != THC_DTYPE_F32 && p->in_dtype != THC_DTYPE_BF16) return THC_EINVAL;
  if (!(p->t_p > 0.f) || !std::isfinite(p->t_p)) return THC_EINVAL;
  if (p->stage_order != THC_ORDER_ASCENDING && p->stage_order != THC_ORDER_SPLIT) return THC_EINVAL;
  if (p->group_log2 != 0 && (p->group_log2 < 10 || p->group_log2 > 40)) return THC_EINVAL;
  if (p->single_launch > 1) return THC_EINVAL;
  const uint32_t top = (1u << p->b) - 1;
  if (p->table[0] != 0 || p->table[top] != p->g) return THC_ETABLE;
  for (uint32_t z = 0; z < top; ++z)
    if (p->table[z] >= p->table[z + 1]) return THC_ETABLE;
  if ((uint64_t)p->g * p->n >= (1ull << p->agg_bits)) return THC_EOVERFLOW;
  return THC_OK;
}

inline int check_launch() {
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return THC_OK;
  std::fprintf(stderr, "libthc: kernel launch failed: %s\n", hipGetErrorString(e));
  return THC_ELAUNCH;
}

}  // namespace thc
