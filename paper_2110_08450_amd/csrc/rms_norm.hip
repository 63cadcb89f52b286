// libsmfg: root-mean-square norm and its gradient (include/smfg.h), host side.  Kernels: kernels_rms.h.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "smfg.h"

#include "kernels_rms.h"
#include "train_common.h"

namespace {

using namespace smfg_dev;

constexpr unsigned kRmsBlocks = 2048;
template <typename T, bool BYTES>
struct LaunchRms {
  const RmsArgs& A;
  Launches& go;
  template <int V, int NV, int LANES>
  void operator()() const {
    const unsigned blocks = blocks_for(A.max_rows, norm_threads(LANES) / LANES, kRmsBlocks);
    go(k_rms_norm<T, V, NV, LANES, BYTES>, blocks, norm_threads(LANES), A);
  }
};

template <typename T>
struct LaunchRmsGrad {
  const RmsGradArgs& A;
  int64_t& slices;
  Launches& go;
  template <int V, int NV, int LANES>
  void operator()() const {
    const int64_t blocks = ceil_div(A.max_rows, norm_threads(LANES) / LANES);
    if (blocks < slices) slices = blocks;
    go(k_rms_norm_grad<T, V, NV, LANES>, static_cast<unsigned>(slices), norm_threads(LANES), A);
  }
};

inline bool is_bytes(int32_t dtype) { return dtype == SMFG_DTYPE_I8 || dtype == SMFG_DTYPE_E4M3; }
inline bool bad_params(int32_t param_dtype, int32_t dtype, const void* a, const void* b) {
  if (param_dtype != SMFG_DTYPE_F32 && param_dtype != dtype) return true;
  const uintptr_t size = static_cast<uintptr_t>(type_bytes(param_dtype));
  return misaligned(a, size) || misaligned(b, size);
}

}  // namespace

extern "C" {

int smfg_rms_norm(const void* d_x, int64_t x_stride, int32_t dtype, const void* d_residual, int64_t residual_stride, void* d_total, int64_t total_stride,
                  const int64_t* d_num_rows, int64_t max_rows, int32_t dim, const void* d_w, int32_t param_dtype, float eps, void* d_y, int64_t y_stride,
                  int32_t y_dtype, float* d_scales, int64_t scales_stride, int32_t group, float* d_rstd, void* hip_stream) {
  const bool bytes = is_bytes(y_dtype);
  if (!d_num_rows || (max_rows > 0 && (!d_x || !d_y || (bytes && !d_scales)))) return SMFG_ERR_NULL_PTR;
  if (bad_dim(dim) || max_rows < 0 || max_rows >= kMaxRows || bad_matrix(d_x, dtype, x_stride, dim) || bad_params(param_dtype, dtype, d_w, nullptr) ||
      (d_residual && bad_matrix(d_residual, dtype, residual_stride, dim)) || (d_total && (!d_residual || bad_matrix(d_total, dtype, total_stride, dim))) ||
      !(eps >= 0.f) || misaligned(d_num_rows, 8) || misaligned(d_rstd, 4))
    return SMFG_ERR_INVALID_ARG;
  if (bytes) {
    const int64_t groups = group == 0 ? 1 : ceil_div(dim, group < 1 ? 1 : group);
    if ((group != 0 && group != 32 && group != 64 && group != 128) || y_stride < dim || y_stride >= (int64_t(1) << 40) || scales_stride < groups ||
        scales_stride >= (int64_t(1) << 40) || misaligned(d_scales, 4))
      return SMFG_ERR_INVALID_ARG;
  } else if (y_dtype != dtype || d_scales || group != 0 || bad_matrix(d_y, y_dtype, y_stride, dim)) {
    return SMFG_ERR_INVALID_ARG;
  }
  // an output in the place of an input has its stride, and its type; two outputs have places of their own
  if (max_rows > 0) {
    if (d_y == d_x && (bytes || y_stride != x_stride)) return SMFG_ERR_INVALID_ARG;
    if (d_residual && d_y == d_residual && (bytes || y_stride != residual_stride)) return SMFG_ERR_INVALID_ARG;
    if (d_total && (d_total == d_y || (d_total == d_x && total_stride != x_stride) || (d_total == d_residual && total_stride != residual_stride)))
      return SMFG_ERR_INVALID_ARG;
  }
  if (max_rows == 0) return SMFG_OK;
  Launches go(hip_stream);
  const RmsArgs A = {d_x, x_stride, d_residual, residual_stride, d_total, total_stride, d_num_rows, max_rows, dim, param_dtype == SMFG_DTYPE_F32, d_w, eps,
                     group, d_y, y_stride, d_rstd, d_scales, scales_stride, y_dtype == SMFG_DTYPE_E4M3, 0};
  with_type(dtype, [&](auto t) {
    using T = decltype(t);
    if (bytes) {
      if (!with_row_shape<T, 2048>(dim, LaunchRms<T, true>{A, go})) go.all(k_rms_norm_long<T, kVec<T>, true>, max_rows, kThreads, A);
    } else {
      if (!with_row_shape<T, 2048>(dim, LaunchRms<T, false>{A, go})) go.all(k_rms_norm_long<T, kVec<T>, false>, max_rows, kThreads, A);
    }
  });
  return go.result();
}

int64_t smfg_rms_norm_grad_scratch_bytes(int64_t max_rows, int32_t dim) {
  if (bad_dim(dim) || max_rows < 0 || max_rows >= kMaxRows) return -1;
  return up256(norm_slices(max_rows, dim) * 4 * dim);
}

int smfg_rms_norm_grad(const void* d_dy, int64_t dy_stride, const void* d_t, int64_t t_stride, int32_t dtype, const void* d_dtotal, int64_t dtotal_stride,
                       const int64_t* d_num_rows, int64_t max_rows, int32_t dim, const void* d_w, int32_t param_dtype, const float* d_rstd, void* d_dx,
                       int64_t dx_stride, void* d_dw, void* d_scratch, int64_t scratch_bytes, void* hip_stream) {
  if (!d_num_rows || (max_rows > 0 && (!d_t || !d_dy || !d_rstd || (d_dw && !d_scratch)))) return SMFG_ERR_NULL_PTR;
  if (bad_dim(dim) || max_rows < 0 || max_rows >= kMaxRows || bad_matrix(d_t, dtype, t_stride, dim) || bad_matrix(d_dy, dtype, dy_stride, dim) ||
      (d_dtotal && bad_matrix(d_dtotal, dtype, dtotal_stride, dim)) || (d_dx && bad_matrix(d_dx, dtype, dx_stride, dim)) ||
      bad_params(param_dtype, dtype, d_w, d_dw) || misaligned(d_num_rows, 8) || misaligned(d_rstd, 4) || misaligned(d_scratch, 256) ||
      (d_dx && ((d_dx == d_dy && dx_stride != dy_stride) || (d_dx == d_t && dx_stride != t_stride) || (d_dx == d_dtotal && dx_stride != dtotal_stride))))
    return SMFG_ERR_INVALID_ARG;
  int64_t slices = norm_slices(max_rows, dim);
  if (d_dw && scratch_bytes < up256(slices * 4 * dim)) return SMFG_ERR_CAPACITY;
  if (!d_dw && (max_rows == 0 || !d_dx)) return SMFG_OK;
  Launches go(hip_stream);
  float* part = d_dw ? static_cast<float*>(d_scratch) : nullptr;
  const RmsGradArgs A = {d_dy, dy_stride, d_t, t_stride, d_dtotal, dtotal_stride, d_num_rows, max_rows, dim, param_dtype == SMFG_DTYPE_F32, d_w, d_rstd, d_dx,
                         dx_stride, part, 0};
  if (max_rows > 0) {
    with_type(dtype, [&](auto t) {
      using T = decltype(t);
      constexpr int V = kVec<T>;
      if (with_row_shape<T, sizeof(T) == 4 ? 2048 : 1536>(dim, LaunchRmsGrad<T>{A, slices, go})) return;
      if (d_dw) {
        if (slices > kNormLongSlices) slices = kNormLongSlices;
        go(k_rms_grad_columns<T, V>, dim3(static_cast<unsigned>(ceil_div(ceil_div(dim, V), kThreads)), static_cast<unsigned>(slices)), kThreads, A);
      }
      if (d_dx) go.all(k_rms_norm_grad_long<T, V>, max_rows, kThreads, A);
    });
  }
  if (d_dw) {
    with_type(param_dtype, [&](auto p) {
      using P = decltype(p);
      go(k_rms_grad_join<P>, static_cast<unsigned>(ceil_div(dim, kNormJoinCols)), kNormJoinThreads, part, static_cast<int32_t>(slices), dim, static_cast<P*>(d_dw));
    });
  }
  return go.result();
}

}  // extern "C"
