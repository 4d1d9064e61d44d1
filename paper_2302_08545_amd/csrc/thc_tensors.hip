// C-ABI of libthc: the calls that take a model's tensors (see include/thc.h).
#include "thc.h"

#include "thc_host.hpp"
#include "thc_tensors.hpp"

namespace {

using namespace thc;

bool aligned(const void* p, uintptr_t to) { return p && reinterpret_cast<uintptr_t>(p) % to == 0; }

constexpr size_t NORM_WS_BYTES = NORM_PARTIALS * sizeof(double) + 16;   // partials, and the factor where the caller keeps none

int check_norm(const thc_tensors* t, int kind, float max_norm, const float* norm_out, const float* scale_out, const void* ws,
               bool in_place, Scan* scan) {
  const int rc = scan_tensors(t, scan);
  if (rc) return rc;
  if (kind != THC_NORM_L2 && kind != THC_NORM_MAX) return THC_EINVAL;
  if (!(max_norm >= 0.f) || !aligned(norm_out, 4) || !aligned(ws, 16)) return THC_EINVAL;
  if (scale_out && !aligned(scale_out, 4)) return THC_EINVAL;
  const Range norm(norm_out, sizeof(float)), scale(scale_out, sizeof(float)), work(ws, NORM_WS_BYTES);
  if (norm.meets(scale) || norm.meets(work) || scale.meets(work)) return THC_EINVAL;
  return check_overlap(t, *scan, in_place, {norm, scale, work});
}

// launch(arguments) with the table in the smaller form that holds it
template <template <class> class Args, class Table, class Fill, class Launch>
void with_table(const Table& tab, uint32_t count, Fill&& fill, Launch&& launch) {
  if (count <= SHORT_TABLE) {
    Args<TensorTable<SHORT_TABLE>> a;
    fill(a);
    shorten(tab, count, &a.tab);
    launch(a);
  } else {
    Args<TensorTable<TABLE>> a;
    fill(a);
    a.tab = tab;
    launch(a);
  }
}

// the partials of all launches; returns their number
template <int KIND>
uint32_t run_partials(const thc_tensors* t, const Scan& scan, bool in_place, double* partials, hipStream_t s) {
  uint32_t written = 0, keep = (uint32_t)(norm_keeps(scan.bytes, in_place) >> LOG_NORM_UNIT);
  for_tables(t, scan, Grid::TENSOR, 0, 0, LOG_NORM_UNIT, [&](const TensorTable<TABLE>& tab, uint32_t count, uint32_t units) {
    const uint32_t groups = units < NORM_PARTIALS ? units : NORM_PARTIALS, kept = keep < units ? keep : units;
    with_table<NormArgs>(
        tab, count,
        [&](auto& a) {
          a.partials = partials;
          a.units = units;
          a.keep = kept;
          a.before = written;
        },
        [&](const auto& a) { k_norm<KIND><<<dim3(groups), dim3(NORM_NT), 0, s>>>(a); });
    keep -= kept;
    written = groups > written ? groups : written;
  });
  return written;
}

// whether the list goes through one launch of one workgroup; if so, that is done
template <int KIND>
bool run_one(const thc_tensors* t, const Scan& scan, bool in_place, NormOut o, hipStream_t s) {
  if (scan.bytes > ONE_MOST_UNITS << LOG_WAVE_UNIT || scan.entries > ONE_MOST_UNITS) return false;
  OneArgs a;
  a.out = o;
  a.units = 0;
  for_tables(t, scan, Grid::TENSOR, 0, 0, LOG_WAVE_UNIT, [&](const TensorTable<TABLE>& tab, uint32_t count, uint32_t units) {
    shorten(tab, count, &a.tab);
    a.units = units;
  });
  if (a.units > ONE_MOST_UNITS) return false;
  if (in_place) k_norm_one<KIND, true><<<dim3(1), dim3(ONE_NT), 0, s>>>(a);
  else k_norm_one<KIND, false><<<dim3(1), dim3(ONE_NT), 0, s>>>(a);
  return true;
}

template <class Launch>
void run_moves(const thc_tensors* t, const Scan& scan, Grid grid, uint32_t flat_bytes, uint64_t zeros, uint32_t log_unit, void* flat,
               const float* scale, Launch&& launch) {
  for_tables(t, scan, grid, flat_bytes, zeros, log_unit, [&](const TensorTable<TABLE>& tab, uint32_t count, uint32_t units) {
    with_table<MoveArgs>(
        tab, count,
        [&](auto& a) {
          a.flat = flat;
          a.scale = scale;
        },
        [&](const auto& a) { launch(a, dim3(units)); });
  });
}

template <int KIND>
void run_norm(const thc_tensors* t, const Scan& scan, NormOut o, double* partials, hipStream_t s) {
  if (run_one<KIND>(t, scan, false, o, s)) return;
  const FinalArgs f{o, partials, run_partials<KIND>(t, scan, false, partials, s)};
  k_norm_final<KIND><<<dim3(1), dim3(64), 0, s>>>(f);
}

template <int KIND>
void run_clip(const thc_tensors* t, const Scan& scan, NormOut o, double* partials, hipStream_t s) {
  if (run_one<KIND>(t, scan, true, o, s)) return;
  const uint32_t written = run_partials<KIND>(t, scan, true, partials, s);
  if (behind_norm(scan.bytes)) {
    for_tables(t, scan, Grid::TENSOR, 0, 0, LOG_NORM_UNIT, [&](const TensorTable<TABLE>& tab, uint32_t count, uint32_t units) {
      with_table<FinishArgs>(
          tab, count,
          [&](auto& a) {
            a.out = o;
            a.partials = partials;
            a.count = written;
          },
          [&](const auto& a) { k_finish_scale<KIND><<<dim3(units), dim3(TNT), 0, s>>>(a); });
    });
    return;
  }
  k_norm_final<KIND><<<dim3(1), dim3(64), 0, s>>>(FinalArgs{o, partials, written});
  const uint32_t lds = move_lds(scan.bytes);
  run_moves(t, scan, Grid::TENSOR, 0, 0, LOG_MOVE_UNIT, nullptr, o.scale, [&](const auto& a, dim3 grid) { k_scale<<<grid, dim3(TNT), lds, s>>>(a); });
}

int check_flat(const thc_params* p, const thc_tensors* t, const void* flat, uint32_t flat_bytes, const float* scale,
               bool to_tensors, Scan* scan) {
  int rc = validate(p);
  if (rc) return rc;
  rc = scan_tensors(t, scan);
  if (rc) return rc;
  if (scan->total > p->d || !aligned(flat, 16) || (scale && !aligned(scale, 4))) return THC_EINVAL;
  const Range vector(flat, p->d * flat_bytes), factor(scale, sizeof(float));
  if (!to_tensors) return factor.meets(vector) ? (int)THC_EINVAL : check_overlap(t, *scan, false, {vector});
  return check_overlap(t, *scan, true, {vector, factor});
}

}  // namespace

extern "C" {

int thc_norm_workspace_bytes(size_t* bytes_out) {
  if (!bytes_out) return THC_EINVAL;
  *bytes_out = NORM_WS_BYTES;
  return THC_OK;
}

int thc_grad_norm(const thc_tensors* t, int kind, float max_norm, float* norm_out, float* scale_out, void* ws, void* stream) {
  Scan scan;
  const int rc = check_norm(t, kind, max_norm, norm_out, scale_out, ws, false, &scan);
  if (rc) return rc;
  const NormOut o{norm_out, scale_out, max_norm};
  double* const partials = static_cast<double*>(ws);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (kind == THC_NORM_L2) run_norm<THC_NORM_L2>(t, scan, o, partials, s);
  else run_norm<THC_NORM_MAX>(t, scan, o, partials, s);
  return check_launch();
}

int thc_grad_clip(const thc_tensors* t, int kind, float max_norm, float* norm_out, float* scale_out, void* ws, void* stream) {
  Scan scan;
  const int rc = check_norm(t, kind, max_norm, norm_out, scale_out, ws, true, &scan);
  if (rc) return rc;
  hipStream_t s = static_cast<hipStream_t>(stream);
  double* const partials = static_cast<double*>(ws);
  float* const scale = scale_out ? scale_out : reinterpret_cast<float*>(partials + NORM_PARTIALS);
  const NormOut o{norm_out, scale, max_norm};
  if (kind == THC_NORM_L2) run_clip<THC_NORM_L2>(t, scan, o, partials, s);
  else run_clip<THC_NORM_MAX>(t, scan, o, partials, s);
  return check_launch();
}

int thc_gather(const thc_params* p, const thc_tensors* t, const float* scale, void* grad_out, void* stream) {
  Scan scan;
  const uint32_t bytes = p && p->in_dtype == THC_DTYPE_BF16 ? 2 : 4;
  const int rc = check_flat(p, t, grad_out, bytes, scale, false, &scan);
  if (rc) return rc;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const uint64_t zeros = p->d - scan.total;
  if (scale && gather_behind_norm(scan, bytes, zeros)) {
    run_moves(t, scan, Grid::FLAT, bytes, zeros, LOG_NORM_UNIT, grad_out, scale, [&](const auto& a, dim3 grid) {
      if (bytes == 2) k_gather<LOG_NORM_UNIT, Bf16><<<grid, dim3(TNT), BEHIND_NORM_LDS, s>>>(a);
      else k_gather<LOG_NORM_UNIT, float><<<grid, dim3(TNT), BEHIND_NORM_LDS, s>>>(a);
    });
    return check_launch();
  }
  const uint32_t lds = move_lds(scan.bytes);
  run_moves(t, scan, Grid::FLAT, bytes, zeros, LOG_MOVE_UNIT, grad_out, scale, [&](const auto& a, dim3 grid) {
    if (bytes == 2) k_gather<LOG_MOVE_UNIT, Bf16><<<grid, dim3(TNT), lds, s>>>(a);
    else k_gather<LOG_MOVE_UNIT, float><<<grid, dim3(TNT), lds, s>>>(a);
  });
  return check_launch();
}

int thc_scatter(const thc_params* p, const float* flat, const float* scale, const thc_tensors* t, void* stream) {
  Scan scan;
  const int rc = check_flat(p, t, flat, 4, scale, true, &scan);
  if (rc) return rc;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const uint32_t lds = move_lds(scan.bytes);
  run_moves(t, scan, Grid::TENSOR, 0, 0, LOG_MOVE_UNIT, const_cast<float*>(flat), scale,
            [&](const auto& a, dim3 grid) { k_scatter<<<grid, dim3(TNT), lds, s>>>(a); });
  return check_launch();
}

}  // extern "C"
