// C-ABI of libthc: the calls that take a model's tensors (see include/thc.h).
#include "thc.h"

#include "thc_host.hpp"
#include "thc_tensors.hpp"

namespace {

using namespace thc;

bool aligned(const void* p, uintptr_t to) { return p && reinterpret_cast<uintptr_t>(p) % to == 0; }

int check_norm(const thc_tensors* t, int kind, float max_norm, const float* norm_out, const float* scale_out, const void* ws) {
  uint64_t total = 0;
  const int rc = validate_tensors(t, &total);
  if (rc) return rc;
  if (kind != THC_NORM_L2 && kind != THC_NORM_MAX) return THC_EINVAL;
  if (!(max_norm >= 0.f) || !aligned(norm_out, 4) || !aligned(ws, 16)) return THC_EINVAL;
  if (scale_out && !aligned(scale_out, 4)) return THC_EINVAL;
  return THC_OK;
}

// the partials of all launches; returns their number
template <int KIND>
uint32_t run_partials(const thc_tensors* t, double* partials, hipStream_t s) {
  uint32_t written = 0;
  NormArgs a;
  a.partials = partials;
  for_tables(t, Grid::TENSOR, 0, 0, [&](const TensorTable& tab, uint32_t units) {
    a.tab = tab;
    a.units = units;
    a.before = written;
    const uint32_t groups = units < NORM_PARTIALS ? units : NORM_PARTIALS;
    k_norm<KIND><<<dim3(groups), dim3(TNT), 0, s>>>(a);
    written = groups > written ? groups : written;
  });
  return written;
}

template <int KIND>
int run_norm(const thc_tensors* t, NormOut o, double* partials, hipStream_t s) {
  o.count = run_partials<KIND>(t, partials, s);
  o.partials = partials;
  k_norm_final<KIND><<<dim3(1), dim3(FINAL_NT), 0, s>>>(o);
  return check_launch();
}

template <int KIND>
int run_clip(const thc_tensors* t, NormOut o, double* partials, hipStream_t s) {
  o.count = run_partials<KIND>(t, partials, s);
  o.partials = partials;
  if (!o.count) {
    k_norm_final<KIND><<<dim3(1), dim3(FINAL_NT), 0, s>>>(o);
    return check_launch();
  }
  ClipArgs a;
  a.out = o;
  a.first = 1;
  for_tables(t, Grid::TENSOR, 0, 0, [&](const TensorTable& tab, uint32_t units) {
    a.tab = tab;
    a.units = units;
    const uint32_t groups = units < NORM_PARTIALS ? units : NORM_PARTIALS;
    k_clip<KIND><<<dim3(groups), dim3(TNT), 0, s>>>(a);
    a.first = 0;
  });
  return check_launch();
}

int check_flat(const thc_params* p, const thc_tensors* t, const void* flat, uint32_t flat_bytes, const float* scale,
               bool to_tensors, uint64_t* total) {
  int rc = validate(p);
  if (rc) return rc;
  rc = validate_tensors(t, total);
  if (rc) return rc;
  if (*total > p->d || !aligned(flat, 16) || (scale && !aligned(scale, 4))) return THC_EINVAL;
  return check_overlap(t, to_tensors, flat, p->d * flat_bytes);
}

}  // namespace

extern "C" {

int thc_norm_workspace_bytes(size_t* bytes_out) {
  if (!bytes_out) return THC_EINVAL;
  *bytes_out = NORM_PARTIALS * sizeof(double);
  return THC_OK;
}

int thc_grad_norm(const thc_tensors* t, int kind, float max_norm, float* norm_out, float* scale_out, void* ws, void* stream) {
  const int rc = check_norm(t, kind, max_norm, norm_out, scale_out, ws);
  if (rc) return rc;
  const NormOut o{norm_out, scale_out, max_norm, 0, nullptr};
  double* const partials = static_cast<double*>(ws);
  hipStream_t s = static_cast<hipStream_t>(stream);
  return kind == THC_NORM_L2 ? run_norm<THC_NORM_L2>(t, o, partials, s) : run_norm<THC_NORM_MAX>(t, o, partials, s);
}

int thc_grad_clip(const thc_tensors* t, int kind, float max_norm, float* norm_out, float* scale_out, void* ws, void* stream) {
  int rc = check_norm(t, kind, max_norm, norm_out, scale_out, ws);
  if (rc) return rc;
  rc = check_overlap(t, true, nullptr, 0);
  if (rc) return rc;
  const NormOut o{norm_out, scale_out, max_norm, 0, nullptr};
  double* const partials = static_cast<double*>(ws);
  hipStream_t s = static_cast<hipStream_t>(stream);
  return kind == THC_NORM_L2 ? run_clip<THC_NORM_L2>(t, o, partials, s) : run_clip<THC_NORM_MAX>(t, o, partials, s);
}

int thc_gather(const thc_params* p, const thc_tensors* t, const float* scale, void* grad_out, void* stream) {
  uint64_t total = 0;
  const uint32_t bytes = p && p->in_dtype == THC_DTYPE_BF16 ? 2 : 4;
  const int rc = check_flat(p, t, grad_out, bytes, scale, false, &total);
  if (rc) return rc;
  hipStream_t s = static_cast<hipStream_t>(stream);
  GatherArgs a;
  a.flat = grad_out;
  a.scale = scale;
  for_tables(t, Grid::FLAT, bytes, p->d - total, [&](const TensorTable& tab, uint32_t units) {
    a.tab = tab;
    a.units = units;
    const dim3 grid(units < NORM_PARTIALS ? units : NORM_PARTIALS), blk(TNT);
    if (bytes == 2) k_gather<Bf16><<<grid, blk, 0, s>>>(a);
    else k_gather<float><<<grid, blk, 0, s>>>(a);
  });
  return check_launch();
}

int thc_scatter(const thc_params* p, const float* flat, const float* scale, const thc_tensors* t, void* stream) {
  uint64_t total = 0;
  const int rc = check_flat(p, t, flat, 4, scale, true, &total);
  if (rc) return rc;
  hipStream_t s = static_cast<hipStream_t>(stream);
  ScatterArgs a;
  a.flat = flat;
  a.scale = scale;
  for_tables(t, Grid::TENSOR, 0, 0, [&](const TensorTable& tab, uint32_t units) {
    a.tab = tab;
    a.units = units;
    k_scatter<<<dim3(units < NORM_PARTIALS ? units : NORM_PARTIALS), dim3(TNT), 0, s>>>(a);
  });
  return check_launch();
}

}  // extern "C"
