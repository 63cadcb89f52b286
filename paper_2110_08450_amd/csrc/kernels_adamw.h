// libsmfg AdamW over many tensors, or over the touched rows of tables, with states of floats or of 8 bits.
//
//   g' = f g,  m = b1 m + (1 - b1) g',  v = b2 v + (1 - b2) g'^2,
//   p = p - lr decay p - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps),   f = scale min(1, max_norm / (norm + 1e-6))
//
// States of 8 bits: blocks of kStateBlock consecutive elements share two floats, A = max |m| and B = max sqrt(v), and an element has
//   m = A sgn(k) (k / 127)^2, k = rint(127 sqrt(|m| / A)) with m's sign;   sqrt(v) = B (k / 255)^2, k = rint(255 sqrt(sqrt(v) / B)), at least 1 if v > 0.
// Squares because the moments of a block spread over decades: the step from one k to the next is 2 / k of the value, 1.6 % at the top of m and 0.8 % of
// sqrt(v), and small ones have the digits that a linear scale would not leave them. v is kept by its root, which is what the update divides by; a k of 0 there would
// divide by eps alone, so that it is kept for v = 0.
#ifndef SMFG_KERNELS_ADAMW_H_
#define SMFG_KERNELS_ADAMW_H_

#include "kernels_rms.h"

namespace smfg_dev {

constexpr int kStateBlock = 128;

// Tensors are rows of `cols` elements (most of them one row), rows are units of kStateBlock columns.  A lane has V consecutive columns of a unit.
struct AdamTensor {
  void* p;
  const void* g;
  void* m;
  void* v;
  float* m_scale;
  float* v_scale;
  void* copy;
  const int64_t* num;  // rows of g in use, or null: all
  const int32_t* ids;  // the rows of p, m, v that g's are for, or null: the same
  int64_t rows, cols;  // of g
  int32_t table_rows;  // of p, with ids
  uint32_t first_block;
  int32_t type;  // of p | of g << 4 | of copy << 8 | state of 8 bits << 12
  float decay;
};
constexpr int kAdamTensors = 36;
struct AdamArgs {
  AdamTensor t[kAdamTensors];
  AdamTensor* table;
  int32_t tensors;
  int32_t first, here;
  uint32_t first_block;
  uint32_t units;  // of a block
  float lr, one_b1, b1, one_b2, b2, eps;
  double log_b1, log_b2, scale, max_norm;
  int64_t step;
  const int64_t* d_step;
  const float* d_lr;
  const float* norm;
};
static_assert(sizeof(AdamTensor) == 104 && sizeof(AdamArgs) <= 4096, "kernel arguments are limited to 4 KB");

static __global__ void __launch_bounds__(64) k_adamw_table(AdamArgs A) {
  for (int i = threadIdx.x; i < A.here; i += 64) A.table[A.first + i] = A.t[i];
}

// The last tensor that begins at the block or before it.
template <bool TABLE>
__device__ __forceinline__ AdamTensor adam_tensor(const AdamArgs& A, uint32_t block) {
  const int lane = threadIdx.x & 63;
  if constexpr (!TABLE) {
    static_assert(kAdamTensors <= 64, "one ballot");
    return A.t[__popcll(__ballot(lane < A.tensors && block >= A.t[lane < A.tensors ? lane : 0].first_block)) - 1];
  } else {
    int lo = 0, hi = A.tensors;  // it is in [lo, hi)
    while (hi - lo > 1) {
      const int step = (hi - lo + 63) / 64, at = lo + lane * step;
      const int begun = __popcll(__ballot(at < hi && block >= A.table[at < hi ? at : lo].first_block));
      lo += (begun - 1) * step;
      hi = lo + step < hi ? lo + step : hi;
    }
    return A.table[lo];
  }
}

// The numbers of a step that are the same for all elements.
struct AdamStep {
  float f;  // of the gradient
  int power;
  float lr, step, root, eps, b1, one_b1, b2, one_b2;
};
__device__ __forceinline__ AdamStep adam_step(const AdamArgs& A) {
  AdamStep S;
  int64_t t = A.step + (A.d_step ? *A.d_step : 0);
  if (t < 1) t = 1;
  S.lr = A.d_lr ? A.lr * *A.d_lr : A.lr;
  // 1 - b^t of a float b would have lost its digits
  S.step = S.lr / -expm1f(static_cast<float>(static_cast<double>(t) * A.log_b1));
  S.root = 1.f / sqrtf(-expm1f(static_cast<float>(static_cast<double>(t) * A.log_b2)));
  S.eps = A.eps;
  S.b1 = A.b1;
  S.one_b1 = A.one_b1;
  S.b2 = A.b2;
  S.one_b2 = A.one_b2;
  double f = A.scale;
  if (A.norm) {
    const double c = A.max_norm / (static_cast<double>(*A.norm) + 1e-6);
    if (c < 1.0) f *= c;
  }
  S.power = 0;
  if (fabs(f) < 0x1p-100 && f != 0.0) f = frexp(f, &S.power);  // a float has few digits left there
  S.f = static_cast<float>(f);
  return S;
}
__device__ __forceinline__ void adam_update(const AdamStep& S, float decay, float g, float& p, float& m, float& v) {
  g *= S.f;
  if (S.power != 0) g = __builtin_ldexpf(g, S.power);
  m = S.b1 * m + S.one_b1 * g;
  v = S.b2 * v + S.one_b2 * g * g;
  p = p - decay * p - S.step * m / (sqrtf(v) * S.root + S.eps);
}

__device__ __forceinline__ float state_m(float scale, uint8_t k) {
  const float x = static_cast<float>(static_cast<int8_t>(k)) * (1.f / 127.f);
  return scale * x * fabsf(x);
}
__device__ __forceinline__ float state_root(float scale, uint8_t k) {
  const float x = static_cast<float>(k) * (1.f / 255.f);
  return scale * x * x;
}

// What a block of elements has in common: the scale that is kept, and what its elements are multiplied by before their root.  Below 2^-100 all are zeros;
// an infinity or a NaN makes the block NaN.
struct StateScale {
  float kept, inverse;
};
__device__ __forceinline__ StateScale state_scale(uint32_t top, float most) {
  if (top < 0x0d800000u) return {0.f, 0.f};
  if (top >= 0x7f800000u) return {__uint_as_float(0x7fc00000u), 0.f};
  return {__uint_as_float(top), most * most / __uint_as_float(top)};
}

template <typename TP, typename TG, int V, bool BYTES>
__device__ __forceinline__ void adam_block(const AdamArgs& A, const AdamTensor& T, const AdamStep& S, uint32_t q) {
  // lanes of a unit: as many as a short row has vectors, so that none idles in short rows
  const int per_row = static_cast<int>(T.cols < kStateBlock ? (T.cols + V - 1) / V : kStateBlock / V);
  int lanes = 1;
  while (lanes < per_row) lanes <<= 1;
  const int64_t row_units = (T.cols + kStateBlock - 1) / kStateBlock;
  int64_t rows = T.rows;
  if (T.num) {
    const int64_t r = *T.num;
    rows = r < 0 ? 0 : r < rows ? r : rows;
  }
  const int64_t units = rows * row_units, first = static_cast<int64_t>(q) * A.units;
  const int64_t end = first + A.units < units ? first + A.units : units;
  const int at_once = kThreads / lanes, lane = static_cast<int>(threadIdx.x) & (lanes - 1);
  const float decay = S.lr * T.decay;
  for (int64_t base = first; base < end; base += at_once) {
    const int64_t u = base + static_cast<int>(threadIdx.x) / lanes;
    if (u >= end) continue;  // all lanes of the unit
    const int64_t row = T.rows == 1 ? 0 : u / row_units;
    int64_t to = row;
    if (T.ids) {
      to = T.ids[row];
      if (to < 0 || to >= T.table_rows) continue;
    }
    const int64_t b = u - row * row_units;
    const int64_t c = b * kStateBlock + lane * V;
    // the last vector of a row ends with it; the columns that it shares with the one before are left to that
    const int64_t start = c + V <= T.cols ? c : T.cols - V;
    const int dup = c >= T.cols || lane >= per_row ? V : static_cast<int>(c - start);
    const int64_t ig = row * T.cols + start, ip = to * T.cols + start, is = to * row_units + b;
    const Elems<TG, V> eg = *reinterpret_cast<const Elems<TG, V>*>(static_cast<const TG*>(T.g) + ig);
    const Elems<TP, V> ep = *reinterpret_cast<const Elems<TP, V>*>(static_cast<const TP*>(T.p) + ip);
    float p[V], m[V], v[V];
    if constexpr (BYTES) {
      const Elems<uint8_t, V> em = *reinterpret_cast<const Elems<uint8_t, V>*>(static_cast<const uint8_t*>(T.m) + ip);
      const Elems<uint8_t, V> ev = *reinterpret_cast<const Elems<uint8_t, V>*>(static_cast<const uint8_t*>(T.v) + ip);
      const float sm = T.m_scale[is], sv = T.v_scale[is];
#pragma unroll
      for (int j = 0; j < V; ++j) {
        m[j] = state_m(sm, em.v[j]);
        v[j] = state_root(sv, ev.v[j]);
        v[j] *= v[j];
      }
    } else {
      const Elems<float, V> em = *reinterpret_cast<const Elems<float, V>*>(static_cast<const float*>(T.m) + ip);
      const Elems<float, V> ev = *reinterpret_cast<const Elems<float, V>*>(static_cast<const float*>(T.v) + ip);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        m[j] = em.v[j];
        v[j] = ev.v[j];
      }
    }
#pragma unroll
    for (int j = 0; j < V; ++j) {
      p[j] = as_float(ep.v[j]);
      adam_update(S, decay, as_float(eg.v[j]), p[j], m[j], v[j]);
    }
    const auto store = [&](auto* dst, const auto& e) {
      if (dup == 0) {
        *reinterpret_cast<__remove_cvref(decltype(e))*>(dst) = e;
      } else {
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (j >= dup) dst[j] = e.v[j];
      }
    };
    Elems<TP, V> op;
#pragma unroll
    for (int j = 0; j < V; ++j) op.v[j] = from_float<TP>(p[j]);
    store(static_cast<TP*>(T.p) + ip, op);
    if (T.copy) {
      if ((T.type >> 8 & 15) == SMFG_DTYPE_F16) {
        Elems<_Float16, V> o;
#pragma unroll
        for (int j = 0; j < V; ++j) o.v[j] = from_float<_Float16>(p[j]);
        store(static_cast<_Float16*>(T.copy) + ip, o);
      } else {
        Elems<__bf16, V> o;
#pragma unroll
        for (int j = 0; j < V; ++j) o.v[j] = from_float<__bf16>(p[j]);
        store(static_cast<__bf16*>(T.copy) + ip, o);
      }
    }
    if constexpr (BYTES) {
      uint32_t top_m = 0, top_v = 0;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        v[j] = sqrtf(v[j]);
        if (j < dup) continue;
        top_m = max_u(top_m, magnitude(m[j]));
        top_v = max_u(top_v, magnitude(v[j]));
      }
      const StateScale sm = state_scale(wave_max(top_m, lanes), 127.f), sv = state_scale(wave_max(top_v, lanes), 255.f);
      Elems<uint8_t, V> om, ov;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float km = sm.inverse == 0.f ? 0.f : __builtin_rintf(sqrtf(fabsf(m[j]) * sm.inverse));
        float kv = sv.inverse == 0.f ? 0.f : __builtin_rintf(sqrtf(v[j] * sv.inverse));
        if (kv < 1.f && v[j] > 0.f && sv.inverse != 0.f) kv = 1.f;
        om.v[j] = static_cast<uint8_t>(static_cast<int>(copysignf(km, m[j])));
        ov.v[j] = static_cast<uint8_t>(static_cast<int>(kv));
      }
      store(static_cast<uint8_t*>(T.m) + ip, om);
      store(static_cast<uint8_t*>(T.v) + ip, ov);
      if (lane == 0) {
        T.m_scale[is] = sm.kept;
        T.v_scale[is] = sv.kept;
      }
    } else {
      Elems<float, V> om, ov;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        om.v[j] = m[j];
        ov.v[j] = v[j];
      }
      store(static_cast<float*>(T.m) + ip, om);
      store(static_cast<float*>(T.v) + ip, ov);
    }
  }
}

// Vectors of the widest type are 16 bytes; rows of fewer columns than a vector go element by element.
template <typename TP, typename TG, bool BYTES>
__device__ __forceinline__ void adam_any(const AdamArgs& A, const AdamTensor& T, const AdamStep& S, uint32_t q) {
  constexpr int V = BYTES && sizeof(TP) == 2 && sizeof(TG) == 2 ? 8 : 4;
  if (T.cols >= V) adam_block<TP, TG, V, BYTES>(A, T, S, q);
  else adam_block<TP, TG, 1, BYTES>(A, T, S, q);
}

template <bool TABLE>
__global__ void __launch_bounds__(kThreads) k_adamw(AdamArgs A) {
  if (A.norm && !(fabsf(*A.norm) < __builtin_inff())) return;  // no step with a gradient that is not finite
  const uint32_t block = A.first_block + blockIdx.x;
  const AdamTensor T = adam_tensor<TABLE>(A, block);
  const uint32_t q = block - T.first_block;
  const AdamStep S = adam_step(A);
  constexpr int F32 = SMFG_DTYPE_F32, F16 = SMFG_DTYPE_F16, BF16 = SMFG_DTYPE_BF16, BYTES = 1 << 12;
  switch (T.type & (BYTES | 255)) {
    case F32 | F32 << 4: adam_any<float, float, false>(A, T, S, q); break;
    case F32 | F16 << 4: adam_any<float, _Float16, false>(A, T, S, q); break;
    case F32 | BF16 << 4: adam_any<float, __bf16, false>(A, T, S, q); break;
    case F16 | F16 << 4: adam_any<_Float16, _Float16, false>(A, T, S, q); break;
    case F16 | F32 << 4: adam_any<_Float16, float, false>(A, T, S, q); break;
    case BF16 | BF16 << 4: adam_any<__bf16, __bf16, false>(A, T, S, q); break;
    case BF16 | F32 << 4: adam_any<__bf16, float, false>(A, T, S, q); break;
    case F32 | F32 << 4 | BYTES: adam_any<float, float, true>(A, T, S, q); break;
    case F32 | F16 << 4 | BYTES: adam_any<float, _Float16, true>(A, T, S, q); break;
    case F32 | BF16 << 4 | BYTES: adam_any<float, __bf16, true>(A, T, S, q); break;
    case F16 | F16 << 4 | BYTES: adam_any<_Float16, _Float16, true>(A, T, S, q); break;
    case F16 | F32 << 4 | BYTES: adam_any<_Float16, float, true>(A, T, S, q); break;
    case BF16 | BF16 << 4 | BYTES: adam_any<__bf16, __bf16, true>(A, T, S, q); break;
    case BF16 | F32 << 4 | BYTES: adam_any<__bf16, float, true>(A, T, S, q); break;
  }
}

// What states of 8 bits stand for.
struct AdamValuesArgs {
  const uint8_t* codes;
  const float* scales;
  int64_t rows, cols;
  int32_t second;
  void* out;
  uint32_t first_block;
};
constexpr int kValueColumns = 2048;  // of a row, by a block
template <typename T>
__global__ void __launch_bounds__(kThreads) k_adamw_values(AdamValuesArgs A) {
  const int64_t block = static_cast<int64_t>(A.first_block) + blockIdx.x, pieces = (A.cols + kValueColumns - 1) / kValueColumns;
  const int64_t row = A.rows == 1 ? 0 : block / pieces, row_units = (A.cols + kStateBlock - 1) / kStateBlock;
  for (int k = 0; k < kValueColumns / kThreads; ++k) {
    const int64_t c = (block - row * pieces) * kValueColumns + k * kThreads + static_cast<int>(threadIdx.x);
    if (c >= A.cols) break;
    const float s = A.scales[row * row_units + c / kStateBlock];
    const uint8_t code = A.codes[row * A.cols + c];
    const float root = state_root(s, code);
    static_cast<T*>(A.out)[row * A.cols + c] = from_float<T>(A.second ? root * root : state_m(s, code));
  }
}

}  // namespace smfg_dev

#endif  // SMFG_KERNELS_ADAMW_H_
