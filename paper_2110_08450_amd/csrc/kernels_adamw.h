// libsmfg AdamW over many tensors, or over the touched rows of tables, with states of floats or of 8 bits.
//
//   g' = f g,  m = b1 m + (1 - b1) g',  v = b2 v + (1 - b2) g'^2,
//   p = p - lr decay p - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps),   f = scale min(1, max_norm / (|scale| norm + 1e-6))
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

// Tensors are rows of `cols` elements (most of them one row), which blocks of threads have by items of V or kStateBlock columns.  Those with states of floats
// and those with states of 8 bits have kernels of their own.
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
  int32_t type;  // of p | of g << 4 | of copy << 8
  float decay;
};
constexpr int kAdamTensors = 36;
struct AdamArgs {
  AdamTensor t[kAdamTensors];
  int32_t tensors;
  uint32_t first_block;  // of the launch
  uint32_t units;  // a block of threads has this many times kStateBlock elements
  int32_t keep;    // parameters and copies stay in the caches
  float lr, b1, b2, root_b2, eps;
  float step_size, root;  // without a step on the device: lr / (1 - b1^t), 1 / sqrt(1 - b2^t)
  double one_b1, root_one_b2, log_b1, log_b2, scale, max_norm;
  int64_t step;
  const int64_t* d_step;
  const float* d_lr;
  const float* norm;
};
static_assert(sizeof(AdamTensor) == 104 && sizeof(AdamArgs) <= 4096, "kernel arguments are limited to 4 KB");

// The last tensor that begins at the block or before it.
__device__ __forceinline__ AdamTensor adam_tensor(const AdamArgs& A, uint32_t block) {
  static_assert(kAdamTensors <= 64, "one ballot");
  const int lane = threadIdx.x & 63;
  return A.t[__popcll(__ballot(lane < A.tensors && block >= A.t[lane < A.tensors ? lane : 0].first_block)) - 1];
}

// The numbers of a step that are the same for all elements.  The gradient's factor f is in those of the moments: m = b1 m + g1 g, v = b2 v + (g2 g)^2 with
// g1 = (1 - b1) f and g2 = sqrt(1 - b2) f.  Where f is below 2^-100, g is multiplied by 2^power first, as a float has few digits left there.
struct AdamStep {
  int power;
  float lr, step, root, eps, b1, b2, root_b2, g1, g2;
};
__device__ __forceinline__ AdamStep adam_step(const AdamArgs& A) {
  AdamStep S;
  const float rate = A.d_lr ? *A.d_lr : 1.f;
  S.lr = A.lr * rate;
  S.step = A.step_size * rate;
  S.root = A.root;
  if (A.d_step) {
    const int64_t t = A.step + *A.d_step;
    const double d = static_cast<double>(t < 1 ? 1 : t);
    // 1 - b^t of a float b would have lost its digits
    S.step = S.lr / -expm1f(static_cast<float>(d * A.log_b1));
    S.root = 1.f / sqrtf(-expm1f(static_cast<float>(d * A.log_b2)));
  }
  S.eps = A.eps;
  S.b1 = A.b1;
  S.b2 = A.b2;
  S.root_b2 = A.root_b2;
  double f = A.scale;
  if (A.norm) {
    const double c = A.max_norm / (fabs(A.scale) * static_cast<double>(*A.norm) + 1e-6);
    if (c < 1.0) f *= c;
  }
  S.power = 0;
  if (fabs(f) < 0x1p-100 && f != 0.0) f = frexp(f, &S.power);
  S.power = __builtin_amdgcn_readfirstlane(S.power);  // the same for all lanes
  S.g1 = static_cast<float>(A.one_b1 * f);
  S.g2 = static_cast<float>(A.root_one_b2 * f);
  return S;
}
// A vector's gradients, times the factor's power.
template <typename TG, int V>
__device__ __forceinline__ void adam_gradient(const AdamStep& S, const Elems<TG, V>& e, float (&g)[V]) {
#pragma unroll
  for (int j = 0; j < V; ++j) g[j] = as_float(e.v[j]);
  if (S.power != 0) {
#pragma unroll
    for (int j = 0; j < V; ++j) g[j] = __builtin_ldexpf(g[j], S.power);
  }
}
// The parameter from the moments, and the root of the second.  States of 8 bits keep the hardware busy with roots: theirs are its own, off by one in the last digit
// (a v below 2^-126 counts as 0), and the quotient is a product with its reciprocal; floats, which the memory bounds, have the exact ones.
// What is taken from the parameter is added up before: 1 - lr decay as a float has steps of 2^-24, which a decay of 1e-7 misses by 19 %, of 2e-8 altogether.  An infinite
// parameter, such as a mask's, has the largest float's decay, so that it stays what it is.
template <bool FAST>
__device__ __forceinline__ float adam_update(const AdamStep& S, float decay, float& p, float m, float v) {
  const float root = FAST ? __builtin_amdgcn_sqrtf(v) : sqrtf(v), den = root * S.root + S.eps;
  constexpr float kMost = 0x1.fffffep127f;
  p -= decay * __builtin_amdgcn_fmed3f(p, -kMost, kMost) + (FAST ? S.step * m * __builtin_amdgcn_rcpf(den) : S.step * m / den);
  return root;
}

// m = A (k / 127) |k / 127|, sqrt(v) = B (k / 255)^2: squares of whole numbers are exact.
__device__ __forceinline__ float state_m(float scale, uint8_t k) {
  const float x = static_cast<float>(static_cast<int8_t>(k));
  return x * fabsf(x) * scale;
}
__device__ __forceinline__ float state_root(float scale, uint8_t k) {
  const float x = static_cast<float>(k);
  return x * x * scale;
}
constexpr float kStateM = 127.f * 127.f, kStateV = 255.f * 255.f;

// What a block of elements has in common: the scale that is kept, and what its elements are multiplied by before their root.  Below 2^-100 all are zeros;
// an infinity or a NaN makes the block NaN.
struct StateScale {
  float kept, inverse;
};
__device__ __forceinline__ StateScale state_scale(uint32_t top, float most) {
  if (top < 0x0d800000u) return {0.f, 0.f};
  if (top >= 0x7f800000u) return {__uint_as_float(0x7fc00000u), 0.f};
  return {__uint_as_float(top), most / __uint_as_float(top)};
}

// The row and the place in it of item i of a block whose first item has the place `at` in row `first_row`, of rows of `per_row` items.
struct AdamPlace {
  int64_t row, at;
};
__device__ __forceinline__ AdamPlace place_of(int64_t rows, int64_t per_row, int64_t first_row, int64_t at, int i) {
  if (rows == 1) return {0, at + i};
  // rows of a tensor with several have at most 2^23 items
  const uint32_t b = static_cast<uint32_t>(at) + static_cast<uint32_t>(i), r = b / static_cast<uint32_t>(per_row);
  return {first_row + r, b - r * static_cast<uint32_t>(per_row)};
}
__device__ __forceinline__ int64_t rows_of(const AdamTensor& T) {
  if (!T.num) return T.rows;
  const int64_t r = *T.num;
  return r < 0 ? 0 : r < T.rows ? r : T.rows;
}
// Items of a block, of `all`.
__device__ __forceinline__ int items_of(int64_t all, int64_t first, uint32_t most) {
  const int64_t left = all - first;
  return left <= 0 ? 0 : left < most ? static_cast<int>(left) : static_cast<int>(most);
}
// Nothing of a step is read or written twice, so that it leaves the caches to others (load_once, store_once): 400 M floats with half gradients and copies (28 bytes
// each) 2430 us without the hints, 2219 with those of the stores, 2152 with both.
// Parameters and copies are what the next pass reads: `keep` says whether they stay in the caches.
template <typename T, int V>
__device__ __forceinline__ void store_next(T* dst, const float (&p)[V], int dup, bool keep) {
  Elems<T, V> e;
#pragma unroll
  for (int j = 0; j < V; ++j) e.v[j] = from_float<T>(p[j]);
  if (keep) store_own(dst, e, dup);
  else store_once(dst, e, dup);
}
template <typename TP, int V>
__device__ __forceinline__ void store_params(const AdamTensor& T, int64_t at, const float (&p)[V], int dup, bool keep) {
  store_next(static_cast<TP*>(T.p) + at, p, dup, keep);
  if (!T.copy) return;
  if ((T.type >> 8 & 15) == SMFG_DTYPE_F16) store_next(static_cast<_Float16*>(T.copy) + at, p, dup, keep);
  else store_next(static_cast<__bf16*>(T.copy) + at, p, dup, keep);
}

// States of floats: an item is a vector of V columns.  Memory bounds it: 400 M floats with half gradients and copies 1845 us, 6.1 TB/s; 240 K rows of 100 floats of a
// table 190 to 199 us for 673 MB, as rows that begin within 64 bytes cost the lines at both ends (of 96 floats the same bytes take 131).
constexpr int kAdamFloats = 4;  // columns of a vector
template <typename TP, typename TG, int V>
__device__ __forceinline__ void adam_floats(const AdamArgs& A, const AdamTensor& T, const AdamStep& S, uint32_t q) {
  const int64_t per_row = (T.cols + V - 1) / V;
  const uint32_t most = A.units * (kStateBlock / kAdamFloats);
  const int64_t first = static_cast<int64_t>(q) * most;
  const int count = items_of(rows_of(T) * per_row, first, most);
  const int64_t first_row = T.rows == 1 ? 0 : first / per_row, first_at = first - first_row * per_row;
  const float decay = S.lr * T.decay;
  for (int i = static_cast<int>(threadIdx.x); i < count; i += kThreads) {
    const AdamPlace a = place_of(T.rows, per_row, first_row, first_at, i);
    // the last vector of a row ends with it; the columns that it shares with the one before are left to that
    const int64_t c = a.at * V, start = c + V <= T.cols ? c : T.cols - V, ig = a.row * T.cols + start;
    int64_t ip = ig;
    if (T.ids) {
      const int32_t id = T.ids[a.row];
      if (static_cast<uint32_t>(id) >= static_cast<uint32_t>(T.table_rows)) continue;
      ip = id * T.cols + start;
    }
    const int dup = static_cast<int>(c - start);
    const Elems<TG, V> eg = load_once<TG, V>(static_cast<const TG*>(T.g) + ig);
    const Elems<TP, V> ep = load_once<TP, V>(static_cast<const TP*>(T.p) + ip);
    Elems<float, V> em = load_once<float, V>(static_cast<const float*>(T.m) + ip), ev = load_once<float, V>(static_cast<const float*>(T.v) + ip);
    float p[V], g[V];
    adam_gradient(S, eg, g);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      p[j] = as_float(ep.v[j]);
      em.v[j] = S.b1 * em.v[j] + S.g1 * g[j];
      ev.v[j] = S.b2 * ev.v[j] + (S.g2 * g[j]) * (S.g2 * g[j]);
      adam_update<false>(S, decay, p[j], em.v[j], ev.v[j]);
    }
    store_params<TP, V>(T, ip, p, dup, A.keep != 0);
    store_once(static_cast<float*>(T.m) + ip, em, dup);
    store_once(static_cast<float*>(T.v) + ip, ev, dup);
  }
}

// Columns of a vector where states are of 8 bits, so that the widest of its types is 16 bytes, and how many times A.units a block has of them then.
__host__ __device__ constexpr int adam_bytes_vector(size_t param, size_t grad) { return param == 2 && grad == 2 ? 8 : 4; }
__host__ __device__ constexpr uint32_t adam_bytes_wide(size_t param, size_t grad, int64_t cols) {
  return adam_bytes_vector(param, grad) == 8 && cols >= 8 ? 2 : 1;
}
// States of 8 bits: an item is a block of kStateBlock columns, whose largest values its lanes tell each other.  400 M bfloat16, 10 bytes each, 718 us (5.6 TB/s) with some
// 57 vector instructions an element (counted).
// Rows are read through the caches: those of few bytes share their lines with their neighbours, and a row has four bytes of a line of each scale.  200 K rows of 100 floats
// of a table of 2 M by half gradients 91 us (110 past the caches) for 284 MB; of 96 81 (80), of 128 80 (76).
template <typename T, int V, bool ROWS>
__device__ __forceinline__ Elems<T, V> load_bytes(const T* src) {
  if constexpr (ROWS) return *reinterpret_cast<const Elems<T, V>*>(src);
  else return load_once<T, V>(src);
}
template <typename TP, typename TG, int V, bool ROWS>
__device__ __forceinline__ void adam_bytes(const AdamArgs& A, const AdamTensor& T, const AdamStep& S, uint32_t q) {
  // lanes of a block: as many as a short row has vectors, so that none idles in short rows
  const int vectors = static_cast<int>(T.cols < kStateBlock ? (T.cols + V - 1) / V : kStateBlock / V);
  int lanes = 1;
  while (lanes < vectors) lanes <<= 1;
  const uint32_t most = A.units * adam_bytes_wide(sizeof(TP), sizeof(TG), T.cols);
  const int64_t per_row = (T.cols + kStateBlock - 1) / kStateBlock, first = static_cast<int64_t>(q) * most;
  const int count = items_of(rows_of(T) * per_row, first, most);
  const int64_t first_row = T.rows == 1 ? 0 : first / per_row, first_at = first - first_row * per_row;
  const bool ragged = T.cols % V != 0;
  const int lane = static_cast<int>(threadIdx.x) & (lanes - 1), mine = static_cast<int>(threadIdx.x) / lanes, at_once = kThreads / lanes;
  const float decay = S.lr * T.decay;
  for (int base = 0; base < count; base += at_once) {
    const int i = base + mine;
    const AdamPlace a = place_of(T.rows, per_row, first_row, first_at, i < count ? i : 0);
    const int64_t c = a.at * kStateBlock + lane * V, start = c + V <= T.cols ? c : T.cols - V;
    int dup = i >= count || c >= T.cols || lane >= vectors ? V : static_cast<int>(c - start);
    int64_t to = a.row;
    if (T.ids) {
      const int32_t id = T.ids[a.row];
      const bool inside = static_cast<uint32_t>(id) < static_cast<uint32_t>(T.table_rows);
      if (!inside) dup = V;
      to = inside ? id : 0;
    }
    const int64_t ig = a.row * T.cols + start, ip = to * T.cols + start, is = to * per_row + a.at;
    const Elems<TG, V> eg = load_once<TG, V>(static_cast<const TG*>(T.g) + ig);
    const Elems<TP, V> ep = load_bytes<TP, V, ROWS>(static_cast<const TP*>(T.p) + ip);
    Elems<uint8_t, V> em = load_bytes<uint8_t, V, ROWS>(static_cast<const uint8_t*>(T.m) + ip);
    Elems<uint8_t, V> ev = load_bytes<uint8_t, V, ROWS>(static_cast<const uint8_t*>(T.v) + ip);
    const float xm = T.m_scale[is] * (1.f / kStateM), xv = T.v_scale[is] * (1.f / kStateV);
    float p[V], m[V], root[V], g[V];
    adam_gradient(S, eg, g);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      p[j] = as_float(ep.v[j]);
      const float r = state_root(xv * S.root_b2, ev.v[j]);
      m[j] = state_m(xm * S.b1, em.v[j]) + S.g1 * g[j];
      root[j] = adam_update<true>(S, decay, p[j], m[j], r * r + (S.g2 * g[j]) * (S.g2 * g[j]));
    }
    store_params<TP, V>(T, ip, p, dup, A.keep != 0);
    if (ragged) {  // columns of the block before
#pragma unroll
      for (int j = 0; j < V; ++j) {
        m[j] = j < dup ? 0.f : m[j];
        root[j] = j < dup ? 0.f : root[j];
      }
    }
    float top_m = 0.f;
    uint32_t top_v = 0;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      top_m = fmaxf(top_m, fabsf(m[j]));
      top_v = max_u(top_v, __float_as_uint(root[j]));
    }
    // no maximum of floats lets a NaN through: it is in the root as well, but for one that a kept scale brought
    if (!(fabsf(xm) < __builtin_inff())) top_v = 0x7fc00000u;
    if (dup == V) {
      top_m = 0.f;
      top_v = 0;
    }
    top_v = lanes_max(top_v, lanes);
    const StateScale av = state_scale(top_v, kStateV), am = state_scale(max_u(lanes_max(__float_as_uint(top_m), lanes), top_v < 0x7f800000u ? 0 : top_v), kStateM);
    uint32_t wm[(V + 3) / 4], wv[(V + 3) / 4];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      if (j % 4 == 0) wm[j / 4] = wv[j / 4] = 0;
      // The instruction rounds to nearest even, holds what is beyond to 0 or 255, and puts the byte in its place.  128 makes the signed ones positive.
      const float km = copysignf(__builtin_amdgcn_sqrtf(fabsf(m[j]) * am.inverse), m[j]) + 128.f;
      wm[j / 4] = __builtin_amdgcn_cvt_pk_u8_f32(km, j % 4, wm[j / 4]);
      // at least 1 where the root, which is 2^-75 at least, is not 0
      const float kv = __builtin_amdgcn_fmed3f(__builtin_amdgcn_sqrtf(root[j] * av.inverse), 1.f, root[j] * 0x1p100f);
      wv[j / 4] = __builtin_amdgcn_cvt_pk_u8_f32(kv, j % 4, wv[j / 4]);
    }
#pragma unroll
    for (int j = 0; j < V; ++j) {
      em.v[j] = static_cast<uint8_t>((wm[j / 4] ^ 0x80808080u) >> 8 * (j % 4));
      ev.v[j] = static_cast<uint8_t>(wv[j / 4] >> 8 * (j % 4));
    }
    store_once(static_cast<uint8_t*>(T.m) + ip, em, dup);
    store_once(static_cast<uint8_t*>(T.v) + ip, ev, dup);
    if (lane == 0 && dup < V) {
      T.m_scale[is] = am.kept;
      T.v_scale[is] = av.kept;
    }
  }
}

// Vectors of the widest type are 16 bytes; rows of fewer columns than a vector go element by element.
template <typename TP, typename TG, bool BYTES>
__device__ __forceinline__ void adam_any(const AdamArgs& A, const AdamTensor& T, const AdamStep& S, uint32_t q) {
  if constexpr (BYTES) {
    constexpr int V = adam_bytes_vector(sizeof(TP), sizeof(TG));
    if (T.cols < V) adam_bytes<TP, TG, 1, true>(A, T, S, q);
    else if (T.rows > 1) adam_bytes<TP, TG, V, true>(A, T, S, q);
    else adam_bytes<TP, TG, V, false>(A, T, S, q);
  } else {
    if (T.cols >= kAdamFloats) adam_floats<TP, TG, kAdamFloats>(A, T, S, q);
    else adam_floats<TP, TG, 1>(A, T, S, q);
  }
}

template <bool BYTES>
__global__ void __launch_bounds__(kThreads) k_adamw(AdamArgs A) {
  if (A.norm && !(fabsf(*A.norm) < __builtin_inff())) return;  // no step with a gradient that is not finite
  const uint32_t block = A.first_block + blockIdx.x;
  const AdamTensor T = adam_tensor(A, block);
  const uint32_t q = block - T.first_block;
  const AdamStep S = adam_step(A);
  constexpr int F32 = SMFG_DTYPE_F32, F16 = SMFG_DTYPE_F16, BF16 = SMFG_DTYPE_BF16;
  switch (T.type & 255) {
    case F32 | F32 << 4: adam_any<float, float, BYTES>(A, T, S, q); break;
    case F32 | F16 << 4: adam_any<float, _Float16, BYTES>(A, T, S, q); break;
    case F32 | BF16 << 4: adam_any<float, __bf16, BYTES>(A, T, S, q); break;
    case F16 | F16 << 4: adam_any<_Float16, _Float16, BYTES>(A, T, S, q); break;
    case F16 | F32 << 4: adam_any<_Float16, float, BYTES>(A, T, S, q); break;
    case BF16 | BF16 << 4: adam_any<__bf16, __bf16, BYTES>(A, T, S, q); break;
    default: adam_any<__bf16, float, BYTES>(A, T, S, q); break;
  }
}

// What states of 8 bits stand for.
struct AdamValuesArgs {
  const uint8_t* codes;
  const float* scales;
  int64_t rows, cols;
  void* out;
  uint32_t first_block;
};
// All values as one sequence, a vector of them a thread and turn; a block of kValueSpan begins anywhere in a row, the rest by 32-bit arithmetic.  400 M to bfloat16
// 200 us, 6.1 TB/s.
constexpr int kValueSpan = 8192;
// A vector of a single row lies within one block, as it begins at a multiple of V.
template <typename T, bool ROWS, bool SECOND>
__global__ void __launch_bounds__(kThreads) k_adamw_values(AdamValuesArgs A) {
  constexpr int V = 8, kTurns = kValueSpan / kThreads / V;
  const int64_t block = static_cast<int64_t>(A.first_block) + blockIdx.x, first = block * kValueSpan, all = A.rows * A.cols;
  const int64_t row_units = (A.cols + kStateBlock - 1) / kStateBlock;
  const int64_t first_row = A.rows == 1 ? 0 : first / A.cols, first_col = first - first_row * A.cols;
  constexpr float most = 1.f / (SECOND ? kStateV : kStateM);
  const auto value = [&](float scale, uint8_t k) {
    if constexpr (!SECOND) return state_m(scale, k);
    const float root = state_root(scale, k);
    return root * root;
  };
  Elems<uint8_t, V> e[kTurns];
  float scale[kTurns][2];  // of the vector's first elements, and of those from `cut` on
  int cut[kTurns];         // V: there are none; negative: element by element
  if (all >= V) {          // loads without conditions, all on their way before one is used
#pragma unroll
    for (int t = 0; t < kTurns; ++t) {
      const int here = (t * kThreads + static_cast<int>(threadIdx.x)) * V, i = first + here + V <= all ? here : 0;
      const AdamPlace at = ROWS ? place_of(A.rows, A.cols, first_row, first_col, i) : AdamPlace{0, first + i};
      const int64_t unit = at.row * row_units + at.at / kStateBlock;
      e[t] = *reinterpret_cast<const Elems<uint8_t, V>*>(A.codes + (first + V <= all ? first + i : 0));
      scale[t][0] = A.scales[unit];
      cut[t] = i == here && first + here + V <= all ? V : -1;
      if constexpr (ROWS) {
        const int64_t left = A.cols - at.at, room = kStateBlock - at.at % kStateBlock, end = left < room ? left : room;  // of the block
        const int64_t next = left > room ? left - room : A.cols;
        if (cut[t] == V && end < V) cut[t] = next < V - end ? -1 : static_cast<int>(end);  // not across a third block
        scale[t][1] = A.scales[cut[t] > 0 && cut[t] < V ? unit + 1 : unit];  // the next one of the row, or the first of the next row
      }
    }
  }
#pragma unroll
  for (int t = 0; t < kTurns; ++t) {
    const int here = (t * kThreads + static_cast<int>(threadIdx.x)) * V;
    T* out = static_cast<T*>(A.out) + first + here;
    if (all >= V && cut[t] >= 0) {
      Elems<T, V> o;
#pragma unroll
      for (int j = 0; j < V; ++j) o.v[j] = from_float<T>(value((ROWS && j >= cut[t] ? scale[t][1] : scale[t][0]) * most, e[t].v[j]));
      *reinterpret_cast<Elems<T, V>*>(out) = o;
    } else {
      for (int j = 0; j < V && first + here + j < all; ++j) {
        const AdamPlace at = place_of(A.rows, A.cols, first_row, first_col, here + j);
        out[j] = from_float<T>(value(A.scales[at.row * row_units + at.at / kStateBlock] * most, A.codes[first + here + j]));
      }
      asm volatile("" ::: "memory");  // as in store_own
    }
  }
}

}  // namespace smfg_dev

#endif  // SMFG_KERNELS_ADAMW_H_
