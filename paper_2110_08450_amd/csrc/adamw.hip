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
constexpr double kLeastNormal = 0x1p-126;  // of floats

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

inline int64_t cols_of(const smfg_param_t& p) { return p.row_elems > 0 ? p.row_elems : p.numel; }

// What a block of threads has as one: vectors of states of floats, blocks of states of 8 bits.
inline int64_t items_of(const smfg_param_t& p) {
  const int64_t cols = cols_of(p);
  if (cols == 0) return 0;
  return p.numel / cols * (p.state_bits == 8 ? ceil_div(cols, kStateBlock) : cols >= kAdamFloats ? ceil_div(cols, kAdamFloats) : cols);
}
// Blocks of threads, and how many times kStateBlock elements each has.  States of floats: 8, a vector a thread, as short-lived blocks keep the memory busiest (400 M with half
// gradients and copies 1840 us; 16 1875, 64 2140, 128 2220).  Of 8 bits, which have more to work out before they begin: 16, and with adam_bytes_wide 32 (400 M bfloat16 704 to 720 us;
// half as many 755, twice 789, four times 855; 300 M floats by half gradients 722, 786, 778 and 822).  Small calls and touched rows lean to either side: 20 M bfloat16 91 us,
// with half as many 79; 200 K rows of 100 floats 91, with half 103, with twice 87.  More, up to 512, where there would be over 2^20 blocks.
struct AdamShape {
  int64_t blocks[2];  // for states of floats, of 8 bits
  bool keep;          // parameters and copies are few enough to be kept for the next pass
  uint32_t units[2];
};
inline int64_t blocks_of(const smfg_param_t& p, const AdamShape& S) {
  const size_t pb = static_cast<size_t>(type_bytes(p.param_dtype)), gb = static_cast<size_t>(type_bytes(p.grad_dtype));
  return ceil_div(items_of(p), p.state_bits == 8 ? S.units[1] * adam_bytes_wide(pb, gb, cols_of(p)) : S.units[0] * (kStateBlock / kAdamFloats));
}
AdamShape adam_shape(const smfg_param_t* p, int32_t n) {
  AdamShape S = {{0, 0}, true, {8, 16}};
  double all[2] = {0, 0}, bytes = 0;
  for (int i = 0; i < n; ++i) {
    all[p[i].state_bits == 8] += static_cast<double>(p[i].numel) / kStateBlock;
    bytes += static_cast<double>(p[i].numel) * static_cast<double>(type_bytes(p[i].param_dtype) + (p[i].copy ? 2 : 0));
  }
  S.keep = bytes <= kKeptBytes;
  for (int k = 0; k < 2; ++k)
    while (S.units[k] < 512 && all[k] > 1048576.0 * S.units[k]) S.units[k] *= 2;
  for (int i = 0; i < n; ++i) S.blocks[p[i].state_bits == 8] += blocks_of(p[i], S);
  return S;
}

}  // namespace

extern "C" {

int smfg_adamw(const smfg_param_t* params, int32_t num_params, const smfg_adamw_t* hyper, void* hip_stream) {
  if ((num_params > 0 && !params) || !hyper) return SMFG_ERR_NULL_PTR;
  const smfg_adamw_t& h = *hyper;
  if (num_params < 0 || bad_params(params, num_params) || !std::isfinite(h.lr) || !(h.beta1 >= 0.0 && h.beta1 < 1.0) || !(h.beta2 >= 0.0 && h.beta2 < 1.0) ||
      !(h.eps >= kLeastNormal) || !std::isfinite(static_cast<float>(h.eps)) || !std::isfinite(h.scale) || !(h.max_norm > 0.0) || h.step < (h.d_step ? 0 : 1) || h.step >= (int64_t(1) << 48) ||
      misaligned(h.d_step, 8) || misaligned(h.d_lr, 4) || misaligned(h.d_norm, 4))
    return SMFG_ERR_INVALID_ARG;
  for (int i = 0; i < num_params; ++i)
    if (has_null(params[i])) return SMFG_ERR_NULL_PTR;
  const AdamShape S = adam_shape(params, num_params);
  if (S.blocks[0] >= kMaxRows || S.blocks[1] >= kMaxRows) return SMFG_ERR_INVALID_ARG;
  Launches go(hip_stream);
  AdamArgs A;
  A.first_block = 0;
  A.keep = S.keep;
  A.lr = static_cast<float>(h.lr);
  A.b1 = static_cast<float>(h.beta1);
  A.b2 = static_cast<float>(h.beta2);
  A.root_b2 = static_cast<float>(std::sqrt(h.beta2));
  A.one_b1 = 1.0 - h.beta1;
  A.root_one_b2 = std::sqrt(1.0 - h.beta2);
  A.eps = static_cast<float>(h.eps);
  A.log_b1 = std::log(h.beta1);
  A.log_b2 = std::log(h.beta2);
  const double t = static_cast<double>(h.step < 1 ? 1 : h.step);
  A.step_size = static_cast<float>(h.lr / -std::expm1(t * A.log_b1));
  A.root = static_cast<float>(1.0 / std::sqrt(-std::expm1(t * A.log_b2)));
  A.scale = h.scale;
  A.max_norm = h.max_norm;
  A.step = h.step;
  A.d_step = h.d_step;
  A.d_lr = h.d_lr;
  A.norm = h.d_norm;
  for (int bytes = 0; bytes < 2; ++bytes) {
    int64_t blocks = 0;
    A.tensors = 0;
    A.units = S.units[bytes];
    const auto launch = [&] {
      if (bytes) go.all(k_adamw<true>, blocks, kThreads, A);
      else go.all(k_adamw<false>, blocks, kThreads, A);
      A.tensors = 0;
      blocks = 0;
    };
    for (int i = 0; i < num_params; ++i) {
      const smfg_param_t& p = params[i];
      if (p.numel == 0 || (p.state_bits == 8) != (bytes == 1)) continue;
      if (A.tensors == kAdamTensors) launch();
      const int64_t cols = cols_of(p);
      A.t[A.tensors++] = {p.param, p.grad, p.m, p.v, p.m_scale, p.v_scale, p.copy, p.d_rows, p.d_row_ids, p.numel / cols, cols,
                          static_cast<int32_t>(p.d_row_ids ? p.num_rows : 0), static_cast<uint32_t>(blocks),
                          p.param_dtype | p.grad_dtype << 4 | (p.copy ? p.copy_dtype : 0) << 8, p.weight_decay};
      blocks += blocks_of(p, S);
    }
    launch();
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
  const int64_t cols = row_elems > 0 ? row_elems : numel, blocks = ceil_div(numel, kValueSpan);
  if (blocks >= (int64_t(1) << 32)) return SMFG_ERR_INVALID_ARG;
  const AdamValuesArgs A = {static_cast<const uint8_t*>(d_codes), d_scales, numel / cols, cols, d_out, 0};
  with_type(out_dtype, [&](auto t) {
    using T = decltype(t);
    if (A.rows > 1) second ? go.all(k_adamw_values<T, true, true>, blocks, kThreads, A) : go.all(k_adamw_values<T, true, false>, blocks, kThreads, A);
    else second ? go.all(k_adamw_values<T, false, true>, blocks, kThreads, A) : go.all(k_adamw_values<T, false, false>, blocks, kThreads, A);
  });
  return go.result();
}

}  // extern "C"
