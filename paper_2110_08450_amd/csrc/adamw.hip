// libsmfg: AdamW over many tensors (include/smfg.h), host side.  Kernels: kernels_adamw.h.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "smfg.h"

#include "kernels_adamw.h"
#include "train_common.h"

namespace {

using namespace smfg_dev;
static_assert(kStateBlock == SMFG_STATE_BLOCK, "blocks of the states");

bool bad_param(const smfg_param_t& p) {
  if (p.numel < 0 || p.numel >= (int64_t(1) << 48) || type_bytes(p.param_dtype) == 0 || type_bytes(p.grad_dtype) == 0) return true;
  if (p.param_dtype != SMFG_DTYPE_F32 && p.grad_dtype != SMFG_DTYPE_F32 && p.grad_dtype != p.param_dtype) return true;
  if (p.state_bits != 32 && p.state_bits != 8) return true;
  if (!std::isfinite(p.weight_decay) || p.weight_decay < 0.f) return true;
  if (p.copy && (p.param_dtype != SMFG_DTYPE_F32 || (p.copy_dtype != SMFG_DTYPE_F16 && p.copy_dtype != SMFG_DTYPE_BF16) || misaligned(p.copy, 2))) return true;
  if (p.row_elems < 0 || p.row_elems > SMFG_MAX_DIM || (p.row_elems > 0 && p.numel % p.row_elems != 0)) return true;
  if ((p.d_row_ids || p.d_rows) && p.row_elems == 0) return true;
  if (p.row_elems > 0 && p.numel / p.row_elems >= kMaxRows) return true;
  if (p.d_row_ids && (p.num_rows < 1 || p.num_rows >= kMaxRows || misaligned(p.d_row_ids, 4))) return true;
  const uintptr_t pa = static_cast<uintptr_t>(type_bytes(p.param_dtype)), ga = static_cast<uintptr_t>(type_bytes(p.grad_dtype));
  if (misaligned(p.param, pa) || misaligned(p.grad, ga) || misaligned(p.d_rows, 8)) return true;
  if (p.state_bits == 32) return misaligned(p.m, 4) || misaligned(p.v, 4);
  return misaligned(p.m_scale, 4) || misaligned(p.v_scale, 4);
}
bool bad_params(const smfg_param_t* p, int32_t n) {
  for (int i = 0; i < n; ++i)
    if (bad_param(p[i])) return true;
  return false;
}
bool has_null(const smfg_param_t& p) {
  return p.numel > 0 && (!p.param || !p.grad || !p.m || !p.v || (p.state_bits == 8 && (!p.m_scale || !p.v_scale)));
}

int64_t units_of(const smfg_param_t& p) {
  const int64_t cols = p.row_elems > 0 ? p.row_elems : p.numel;
  return cols == 0 ? 0 : p.numel / cols * ceil_div(cols, kStateBlock);
}

// Scratch: the table of more tensors than the arguments hold.  A block has so many units that there are 4096 blocks, but 16 (2 Ki elements) at least and 512 at most.
struct AdamShape {
  int64_t blocks, bytes;
  uint32_t units;
  int32_t tensors;
};
AdamShape adam_shape(const smfg_param_t* p, int32_t n) {
  AdamShape S = {0, 0, 16, 0};
  double all = 0;
  for (int i = 0; i < n; ++i) all += static_cast<double>(units_of(p[i]));
  while (S.units < 512 && all > 4096.0 * 2 * S.units) S.units *= 2;
  for (int i = 0; i < n; ++i) {
    S.tensors += p[i].numel > 0;
    S.blocks += ceil_div(units_of(p[i]), S.units);
  }
  S.bytes = S.tensors > kAdamTensors ? up256(static_cast<int64_t>(sizeof(AdamTensor)) * S.tensors) : 0;
  return S;
}

}  // namespace

extern "C" {

int64_t smfg_adamw_scratch_bytes(const smfg_param_t* params, int32_t num_params) {
  if (num_params < 0 || (num_params > 0 && !params) || bad_params(params, num_params)) return -1;
  return adam_shape(params, num_params).bytes;
}

int smfg_adamw(const smfg_param_t* params, int32_t num_params, const smfg_adamw_t* hyper, void* d_scratch, int64_t scratch_bytes, void* hip_stream) {
  if ((num_params > 0 && !params) || !hyper) return SMFG_ERR_NULL_PTR;
  const smfg_adamw_t& h = *hyper;
  if (num_params < 0 || bad_params(params, num_params) || !std::isfinite(h.lr) || !(h.beta1 >= 0.0 && h.beta1 < 1.0) || !(h.beta2 >= 0.0 && h.beta2 < 1.0) ||
      !(h.eps >= 0.0) || !std::isfinite(h.eps) || !std::isfinite(h.scale) || !(h.max_norm > 0.0) || h.step < (h.d_step ? 0 : 1) || h.step >= (int64_t(1) << 48) ||
      misaligned(h.d_step, 8) || misaligned(h.d_lr, 4) || misaligned(h.d_norm, 4) || misaligned(d_scratch, 256))
    return SMFG_ERR_INVALID_ARG;
  for (int i = 0; i < num_params; ++i)
    if (has_null(params[i])) return SMFG_ERR_NULL_PTR;
  const AdamShape S = adam_shape(params, num_params);
  if (S.blocks >= kMaxRows) return SMFG_ERR_INVALID_ARG;
  if (S.bytes > 0 && !d_scratch) return SMFG_ERR_NULL_PTR;
  if (scratch_bytes < S.bytes) return SMFG_ERR_CAPACITY;
  Launches go(hip_stream);
  const bool table = S.tensors > kAdamTensors;
  AdamArgs A;
  A.table = table ? static_cast<AdamTensor*>(d_scratch) : nullptr;
  A.tensors = S.tensors;
  A.first = A.here = 0;
  A.first_block = 0;
  A.units = S.units;
  A.lr = static_cast<float>(h.lr);
  A.b1 = static_cast<float>(h.beta1);
  A.one_b1 = static_cast<float>(1.0 - h.beta1);
  A.b2 = static_cast<float>(h.beta2);
  A.one_b2 = static_cast<float>(1.0 - h.beta2);
  A.eps = static_cast<float>(h.eps);
  A.log_b1 = std::log(h.beta1);
  A.log_b2 = std::log(h.beta2);
  A.scale = h.scale;
  A.max_norm = h.max_norm;
  A.step = h.step;
  A.d_step = h.d_step;
  A.d_lr = h.d_lr;
  A.norm = h.d_norm;
  uint32_t blocks = 0;
  for (int i = 0; i < num_params; ++i) {
    const smfg_param_t& p = params[i];
    if (p.numel == 0) continue;
    if (A.here == kAdamTensors) {
      go(k_adamw_table, 1, 64, A);
      A.first += A.here;
      A.here = 0;
    }
    const int64_t cols = p.row_elems > 0 ? p.row_elems : p.numel;
    A.t[A.here++] = {p.param, p.grad, p.m, p.v, p.m_scale, p.v_scale, p.copy, p.d_rows, p.d_row_ids, p.numel / cols, cols,
                     static_cast<int32_t>(p.d_row_ids ? p.num_rows : 0), blocks,
                     p.param_dtype | p.grad_dtype << 4 | (p.copy ? p.copy_dtype : 0) << 8 | (p.state_bits == 8) << 12, p.weight_decay};
    blocks += static_cast<uint32_t>(ceil_div(units_of(p), S.units));
  }
  if (table) go(k_adamw_table, 1, 64, A);
  if (blocks > 0) {
    if (table) go.all(k_adamw<true>, blocks, kThreads, A);
    else go.all(k_adamw<false>, blocks, kThreads, A);
  }
  return go.result();
}

int smfg_adamw_values(const void* d_codes, const float* d_scales, int64_t numel, int64_t row_elems, int32_t second, void* d_out, int32_t out_dtype,
                      void* hip_stream) {
  if (numel > 0 && (!d_codes || !d_scales || !d_out)) return SMFG_ERR_NULL_PTR;
  if (numel < 0 || numel >= (int64_t(1) << 48) || row_elems < 0 || row_elems > SMFG_MAX_DIM || (row_elems > 0 && numel % row_elems != 0) ||
      (row_elems > 0 && numel / row_elems >= kMaxRows) || (second != 0 && second != 1) || type_bytes(out_dtype) == 0 || misaligned(d_scales, 4) ||
      misaligned(d_out, static_cast<uintptr_t>(type_bytes(out_dtype))))
    return SMFG_ERR_INVALID_ARG;
  if (numel == 0) return SMFG_OK;
  Launches go(hip_stream);
  const int64_t cols = row_elems > 0 ? row_elems : numel, blocks = numel / cols * ceil_div(cols, kValueColumns);
  if (blocks >= (int64_t(1) << 32)) return SMFG_ERR_INVALID_ARG;
  const AdamValuesArgs A = {static_cast<const uint8_t*>(d_codes), d_scales, numel / cols, cols, second, d_out, 0};
  with_type(out_dtype, [&](auto t) { go.all(k_adamw_values<decltype(t)>, blocks, kThreads, A); });
  return go.result();
}

}  // extern "C"
