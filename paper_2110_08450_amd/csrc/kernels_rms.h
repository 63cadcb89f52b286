// libsmfg root-mean-square norm over rows, with the addition of a residual before it and an output in 8 bits with scales, and its gradient.
//
//   t = x + residual, rounded to their type (without a residual t = x),  r_i = 1 / sqrt(mean(t_i^2) + eps),  y_ij = t_ij r_i w_j
//   n = t r, g = dy w:  dx = r (g - n mean(g n)) + dt,  dw_j = sum_i dy_ij n_ij
//
// The norm is of the sum as it is kept, not of the one before its rounding: the gradient reads the kept one, so it is that of what was computed.
#ifndef SMFG_KERNELS_RMS_H_
#define SMFG_KERNELS_RMS_H_

#include "kernels_norm.h"

namespace smfg_dev {

struct RmsArgs {
  const void* x;
  int64_t x_stride;
  const void* residual;  // or null
  int64_t residual_stride;
  void* total;  // or null
  int64_t total_stride;
  const int64_t* num;
  int64_t max_rows;
  int32_t dim;
  int32_t float_params;
  const void* w;
  float eps;
  int32_t group;  // columns of a scale; 0: all
  void* y;
  int64_t y_stride;
  float* rstd;
  float* scales;
  int64_t scales_stride;
  int32_t e4m3;  // of 8-bit outputs: e4m3, else whole numbers
  uint32_t first_block;  // of the launch, where a row is a block's
};

// Bits of a magnitude: as whole numbers they are in the order of the magnitudes, infinity and then NaN the largest, so that a maximum lets a NaN through.
__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// Largest of groups of `lanes` lanes (1 to 32, a power of two).
__device__ __forceinline__ uint32_t lanes_max(uint32_t x, int lanes) {
  switch (lanes) {  // the same for all lanes
    case 1: return x;
    case 2: return lanes_all<2>(x, max_u);
    case 4: return lanes_all<4>(x, max_u);
    case 8: return lanes_all<8>(x, max_u);
    case 16: return lanes_all<16>(x, max_u);
    default: return lanes_all<32>(x, max_u);
  }
}
template <int LANES>
__device__ __forceinline__ uint32_t group_max(uint32_t x, uint32_t* lds) {
  x = lanes_all<(LANES < 64 ? LANES : 64)>(x, max_u);
  if constexpr (LANES > 64) {
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < LANES / 64; ++w) x = max_u(x, lds[w]);
  }
  return x;
}

// Rows of 128 vectors and more are read past the caches, and the sum, which the next layer reads much later, is written past them; what the next operator reads is
// not (16 K rows of 4096 halfs with the sum 100 -> 80 us, with a product of y behind it 145 -> 118; y past the caches as well 80, and 152).  Both ways of reading, halfs
// with the sum, alone / with a pass over y behind: 16 K x 4096 through 102 / 149 us, past 83 / 140; 50 K x 2048 156 / 227 and 157 / 216; 100 K x 1024 (128 vectors) 153 / 224
// and 157 / 215; 20 K x 1024 26 / 41 and 28 / 39.  Below the limit, where they are read through, 200 K x 512 158 / 228 and 160 / 218; 154 K x 256 60 / 88 and 52 / 75: narrower
// rows would gain as well, down to 16 vectors (400 K x 128 78 / 114 and 65 / 102).  The gradient likewise: 94 / 142 past for 104 / 153 at 4096, 65 / 94 through for 57 / 81 at 256.
template <typename T, int V, int VECTORS>
__device__ __forceinline__ Elems<T, V> load_row(const T* src) {
  if constexpr (VECTORS >= 128) return load_once<T, V>(src);
  else return *reinterpret_cast<const Elems<T, V>*>(src);
}

// The scale of values up to a largest magnitude, and what they are multiplied by.  The largest becomes 127, or 448, the largest e4m3.  Below 2^-120 (e4m3: 2^-119) the
// factor would leave a float's range, of which 127 * 2^120 and 448 * 2^119 are the last: all are zeros then, and the scale as well.  With an infinity or a NaN
// among them the scale is NaN.
struct ByteScale {
  float scale, inverse;
};
__device__ __forceinline__ ByteScale byte_scale(uint32_t top, bool e4m3) {
  const float most = e4m3 ? 448.f : 127.f;
  if (top < (e4m3 ? 0x04000000u : 0x03800000u)) return {0.f, 0.f};
  if (top >= 0x7f800000u) return {__uint_as_float(0x7fc00000u), 0.f};
  return {__uint_as_float(top) / most, most / __uint_as_float(top)};
}
// Rounded to nearest even.  With an inverse of 0 all are zeros, NaN among them.
template <int V>
__device__ __forceinline__ Elems<uint8_t, V> to_bytes(const float (&y)[V], float inverse, bool e4m3) {
  Elems<uint8_t, V> o;
  float q[V];
#pragma unroll
  for (int j = 0; j < V; ++j) q[j] = inverse == 0.f ? 0.f : y[j] * inverse;
  if (e4m3) {
#pragma unroll
    for (int j = 0; j < V; j += 2) {
      const int two = __builtin_amdgcn_cvt_pk_fp8_f32(q[j], V > 1 ? q[j + (V > 1)] : 0.f, 0, false);
      o.v[j] = static_cast<uint8_t>(two);
      if constexpr (V > 1) o.v[j + 1] = static_cast<uint8_t>(two >> 8);
    }
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j) o.v[j] = static_cast<uint8_t>(static_cast<int>(__builtin_rintf(q[j])));
  }
  return o;
}

// The sum that is normed, as it is kept.
template <typename T>
__device__ __forceinline__ float kept_sum(T x, T residual) {
  return as_float(from_float<T>(as_float(x) + as_float(residual)));
}

// One vector of a row in 8 bits, and the group's scale by the first lane of those that have one.  Columns that the last vector shares with the one before
// belong to another group there: they are left to it.
template <int V>
__device__ __forceinline__ void store_bytes(const RmsArgs& A, int64_t row, const Columns<V>& c, int index, const float (&y)[V], ByteScale s, int group_lanes) {
  if (c.dup == V) return;
  const Elems<uint8_t, V> o = to_bytes<V>(y, s.inverse, A.e4m3 != 0);
  store_own(static_cast<uint8_t*>(A.y) + row * A.y_stride + c.start, o, c.dup);
  if (index % group_lanes == 0) A.scales[row * A.scales_stride + index / group_lanes] = s.scale;
}

// As k_layer_norm: a group of LANES lanes has a row in its registers, NV vectors of V columns a lane, and asks for its next one while it works on it.  Memory
// bounds it: 154 K rows of 256 halfs with the sum 61 us, 5.2 TB/s; 16 K rows of 4096 bfloat16 with the sum to e4m3, a scale for 128 columns, 78 us, 6.0 TB/s.
template <typename T, int V, int NV, int LANES, bool BYTES>
__global__ void __launch_bounds__(norm_threads(LANES)) k_rms_norm(RmsArgs A) {
  __shared__ float lds[2][norm_threads(LANES) / 64];
  __shared__ uint32_t tops[BYTES ? norm_threads(LANES) / 64 : 1];
  constexpr int kGroups = norm_threads(LANES) / LANES;
  const int lane = threadIdx.x % LANES;
  const int64_t step = static_cast<int64_t>(gridDim.x) * kGroups;
  int64_t row = static_cast<int64_t>(blockIdx.x) * kGroups + threadIdx.x / LANES;
  const bool ragged = A.dim % V != 0;
  const T* const x = static_cast<const T*>(A.x);
  const T* const res = static_cast<const T*>(A.residual);
  Elems<T, V> e[NV], q[NV];
  float w[NV][V];
  const auto load = [&](int64_t i) {
#pragma unroll
    for (int k = 0; k < NV; ++k) e[k] = load_row<T, V, NV * LANES>(x + i * A.x_stride + columns_of<V, NV, LANES>(k, lane, A.dim).start);
    if (res) {
#pragma unroll
      for (int k = 0; k < NV; ++k) q[k] = load_row<T, V, NV * LANES>(res + i * A.residual_stride + columns_of<V, NV, LANES>(k, lane, A.dim).start);
    }
  };
  load(row < A.max_rows ? row : A.max_rows - 1);
#pragma unroll
  for (int k = 0; k < NV; ++k) load_params<T, V>(A.w, A.float_params != 0, columns_of<V, NV, LANES>(k, lane, A.dim).start, 1.f, w[k]);
  const int64_t n = count_of(A.num, A.max_rows);
  for (int turn = 0; row < n; row += step, turn ^= 1) {
    float v[NV][V];
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const Columns<V> c = columns_of<V, NV, LANES>(k, lane, A.dim);
      float part = 0.f;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        v[k][j] = res ? kept_sum(e[k].v[j], q[k].v[j]) : as_float(e[k].v[j]);
        if (ragged && j < c.dup) continue;
        part += v[k][j] * v[k][j];
      }
      s += c.dup < V ? part : 0.f;
    }
    if (row + step < n) load(row + step);
    const float r = 1.f / sqrtf(row_sum<LANES>(s, lds[turn]) / static_cast<float>(A.dim) + A.eps);
    if (lane == 0 && A.rstd) A.rstd[row] = r;
    // the sum: behind the barrier, as it may take the place of x or of the residual, which other lanes read as well
    if (A.total) {
      T* t = static_cast<T*>(A.total) + row * A.total_stride;
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const Columns<V> c = columns_of<V, NV, LANES>(k, lane, A.dim);
        if (c.dup == V) continue;
        Elems<T, V> o;
#pragma unroll
        for (int j = 0; j < V; ++j) o.v[j] = from_float<T>(v[k][j]);
        store_once(t + c.start, o, 0);
      }
    }
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int j = 0; j < V; ++j) v[k][j] = v[k][j] * r * w[k][j];
    if constexpr (BYTES) {
      uint32_t top[NV];
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const Columns<V> c = columns_of<V, NV, LANES>(k, lane, A.dim);
        top[k] = 0;
#pragma unroll
        for (int j = 0; j < V; ++j) top[k] = j >= c.dup ? max_u(top[k], magnitude(v[k][j])) : top[k];
      }
      int lanes = A.group / V;  // of a scale
      if (A.group == 0) {
        lanes = NV * LANES;
#pragma unroll
        for (int k = 1; k < NV; ++k) top[0] = max_u(top[0], top[k]);
        top[0] = group_max<LANES>(top[0], tops);
#pragma unroll
        for (int k = 1; k < NV; ++k) top[k] = top[0];
      } else {
#pragma unroll
        for (int k = 0; k < NV; ++k) top[k] = lanes_max(top[k], lanes < LANES ? lanes : LANES);
      }
#pragma unroll
      for (int k = 0; k < NV; ++k)
        store_bytes<V>(A, row, columns_of<V, NV, LANES>(k, lane, A.dim), k * LANES + lane, v[k], byte_scale(top[k], A.e4m3 != 0), lanes);
    } else {
      T* y = static_cast<T*>(A.y) + row * A.y_stride;
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const Columns<V> c = columns_of<V, NV, LANES>(k, lane, A.dim);
        if (c.dup == V) continue;
        Elems<T, V> o;
#pragma unroll
        for (int j = 0; j < V; ++j) o.v[j] = from_float<T>(v[k][j]);
        *reinterpret_cast<Elems<T, V>*>(y + c.start) = o;
      }
    }
  }
}

// Rows that outgrow the registers of a block: one to a block, read again for each sum, which is in double as in k_layer_norm_long.  A thread has the same
// columns in every round and touches no others, so that outputs may take the place of inputs.  3000 rows of 20 000 floats with the sum 234 us (4.1 TB/s).
template <typename T, int V, bool BYTES>
__global__ void __launch_bounds__(kThreads) k_rms_norm_long(RmsArgs A) {
  __shared__ double lds[kThreads / 64];
  __shared__ uint32_t tops[kThreads / 64];
  const int64_t row = static_cast<int64_t>(A.first_block) + blockIdx.x;
  if (row >= count_of(A.num, A.max_rows)) return;
  const T* x = static_cast<const T*>(A.x) + row * A.x_stride;
  const T* res = A.residual ? static_cast<const T*>(A.residual) + row * A.residual_stride : nullptr;
  T* total = A.total ? static_cast<T*>(A.total) + row * A.total_stride : nullptr;
  const int vectors = (A.dim + V - 1) / V;
  // the sum of a vector's columns; from the kept one where there is one, which may be in the place of x
  const auto values = [&](const Columns<V>& c, bool kept, float(&v)[V]) {
    const Elems<T, V> e = *reinterpret_cast<const Elems<T, V>*>((kept && total ? total : x) + c.start);
    if (res && !(kept && total)) {
      const Elems<T, V> q = *reinterpret_cast<const Elems<T, V>*>(res + c.start);
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] = kept_sum(e.v[j], q.v[j]);
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] = as_float(e.v[j]);
    }
  };
  double s = 0.0;
  for (int i = threadIdx.x; i < vectors; i += kThreads) {
    const Columns<V> c(i, A.dim);
    float v[V];
    values(c, false, v);
    Elems<T, V> o;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      s += j >= c.dup ? static_cast<double>(v[j]) * v[j] : 0.0;
      o.v[j] = from_float<T>(v[j]);
    }
    if (total) store_own(total + c.start, o, c.dup);
  }
  const float r = 1.f / sqrtf(static_cast<float>(group_sum<kThreads>(s, lds) / A.dim) + A.eps);
  if (threadIdx.x == 0 && A.rstd) A.rstd[row] = r;
  const auto outputs = [&](const Columns<V>& c, float(&v)[V]) {
    float w[V];
    values(c, true, v);
    load_params<T, V>(A.w, A.float_params != 0, c.start, 1.f, w);
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = v[j] * r * w[j];
  };
  const auto top_of = [](const Columns<V>& c, const float(&v)[V]) {
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < V; ++j) top = j >= c.dup ? max_u(top, magnitude(v[j])) : top;
    return top;
  };
  ByteScale scale = {0.f, 0.f};
  if (BYTES && A.group == 0) {
    uint32_t top = 0;
    for (int i = threadIdx.x; i < vectors; i += kThreads) {
      const Columns<V> c(i, A.dim);
      float v[V];
      outputs(c, v);
      top = max_u(top, top_of(c, v));
    }
    scale = byte_scale(group_max<kThreads>(top, tops), A.e4m3 != 0);
  }
  for (int base = 0; base < vectors; base += kThreads) {  // all lanes together, as they ask each other for their maxima
    const int i = base + static_cast<int>(threadIdx.x);
    const Columns<V> c(i, A.dim);
    float v[V];
    outputs(c, v);
    if constexpr (BYTES) {
      if (A.group != 0) scale = byte_scale(lanes_max(top_of(c, v), A.group / V), A.e4m3 != 0);
      store_bytes<V>(A, row, c, i, v, scale, A.group == 0 ? 1 << 30 : A.group / V);
    } else {
      T* y = static_cast<T*>(A.y) + row * A.y_stride;
      Elems<T, V> o;
#pragma unroll
      for (int j = 0; j < V; ++j) o.v[j] = from_float<T>(v[j]);
      store_own(y + c.start, o, c.dup);
    }
  }
}

struct RmsGradArgs {
  const void* dy;
  int64_t dy_stride;
  const void* t;  // the sum, or x
  int64_t t_stride;
  const void* dt;  // its gradient from elsewhere, or null
  int64_t dt_stride;
  const int64_t* num;
  int64_t max_rows;
  int32_t dim;
  int32_t float_params;
  const void* w;
  const float* rstd;
  void* dx;  // or null
  int64_t dx_stride;
  float* part;  // [slices][dim]: sums of dy n over the rows of a slice, or null
  uint32_t first_block;  // of the launch, where a row is a block's
};

// As k_layer_norm_grad.  16 K rows of 4096 bfloat16 with the sum's gradient 96 us, 5.6 TB/s; 47 K of 301 floats 30 us, 5.7 TB/s.
template <typename T, int V, int NV, int LANES>
__global__ void __launch_bounds__(norm_threads(LANES)) k_rms_norm_grad(RmsGradArgs A) {
  __shared__ float lds[2][norm_threads(LANES) / 64];
  constexpr int kGroups = norm_threads(LANES) / LANES;
  const int lane = threadIdx.x % LANES;
  const int64_t n = count_of(A.num, A.max_rows), step = static_cast<int64_t>(gridDim.x) * kGroups;
  const float inv = 1.f / static_cast<float>(A.dim);
  const bool ragged = A.dim % V != 0;
  float w[NV][V], dw[NV][V];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    load_params<T, V>(A.w, A.float_params != 0, columns_of<V, NV, LANES>(k, lane, A.dim).start, 1.f, w[k]);
#pragma unroll
    for (int j = 0; j < V; ++j) dw[k][j] = 0.f;
  }
  const T* const t = static_cast<const T*>(A.t);
  const T* const dy = static_cast<const T*>(A.dy);
  const T* const dt = static_cast<const T*>(A.dt);
  Elems<T, V> et[NV], ey[NV], ed[NV];
  float r = 0.f;
  const auto load = [&](int64_t row) {
    r = A.rstd[row];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const Columns<V> c = columns_of<V, NV, LANES>(k, lane, A.dim);
      et[k] = load_row<T, V, NV * LANES>(t + row * A.t_stride + c.start);
      ey[k] = load_row<T, V, NV * LANES>(dy + row * A.dy_stride + c.start);
    }
    if (dt) {
#pragma unroll
      for (int k = 0; k < NV; ++k) ed[k] = load_row<T, V, NV * LANES>(dt + row * A.dt_stride + columns_of<V, NV, LANES>(k, lane, A.dim).start);
    }
  };
  int64_t row = static_cast<int64_t>(blockIdx.x) * kGroups + threadIdx.x / LANES;
  if (row < n) load(row);
  for (int turn = 0; row < n; row += step, turn ^= 1) {
    float h[NV][V], g[NV][V], d[NV][V];
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const Columns<V> c = columns_of<V, NV, LANES>(k, lane, A.dim);
      float part = 0.f;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        h[k][j] = as_float(et[k].v[j]) * r;
        const float y = as_float(ey[k].v[j]);
        dw[k][j] += y * h[k][j];
        g[k][j] = y * w[k][j];
        d[k][j] = dt ? as_float(ed[k].v[j]) : 0.f;
        // the row has been read before the barrier, as dx may take the place of dt
        asm volatile("" : "+v"(d[k][j]));
        if (ragged && j < c.dup) continue;
        part += g[k][j] * h[k][j];
      }
      s += c.dup < V ? part : 0.f;
    }
    const float scale = r;
    if (row + step < n) load(row + step);
    if (!A.dx) continue;
    const float c2 = row_sum<LANES>(s, lds[turn]) * inv;
    T* dx = static_cast<T*>(A.dx) + row * A.dx_stride;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const Columns<V> c = columns_of<V, NV, LANES>(k, lane, A.dim);
      if (c.dup == V) continue;
      Elems<T, V> e;
#pragma unroll
      for (int j = 0; j < V; ++j) e.v[j] = from_float<T>(scale * (g[k][j] - h[k][j] * c2) + d[k][j]);
      *reinterpret_cast<Elems<T, V>*>(dx + c.start) = e;
    }
  }
  if (!A.part) return;
  // groups of a wave, then waves, always in the same order
  constexpr int kWidth = LANES * NV * V;
  __shared__ float sums[LANES <= 64 ? kThreads / 64 * kWidth : 1];
  float* out = A.part + static_cast<int64_t>(blockIdx.x) * A.dim;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
#pragma unroll
    for (int j = 0; j < V; ++j)
#pragma unroll
      for (int o = LANES; o < 64; o <<= 1) dw[k][j] += __shfl_xor(dw[k][j], o, 64);
  }
  if constexpr (LANES > 64) {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const Columns<V> c = columns_of<V, NV, LANES>(k, lane, A.dim);
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (j >= c.dup) out[c.start + j] = dw[k][j];
    }
  } else {
    if ((threadIdx.x & 63) < LANES) {
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int j = 0; j < V; ++j) sums[(threadIdx.x >> 6) * kWidth + (k * V + j) * LANES + lane] = dw[k][j];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < kWidth; i += kThreads) {
      const int kj = i / LANES;
      const Columns<V> c(kj / V * LANES + i % LANES, A.dim);
      const int j = kj % V;
      if (j < c.dup) continue;
      float s = 0.f;
#pragma unroll
      for (int q = 0; q < kThreads / 64; ++q) s += sums[q * kWidth + i];
      out[c.start + j] = s;
    }
  }
}

// Rows that outgrow the registers of a block: dx by a block per row, which reads it twice and adds in double; the weight's sums by k_rms_grad_columns.  3000
// rows of 20 000 floats, all of it, 351 us (2.7 TB/s).
template <typename T, int V>
__global__ void __launch_bounds__(kThreads) k_rms_norm_grad_long(RmsGradArgs A) {
  __shared__ double lds[kThreads / 64];
  const int64_t row = static_cast<int64_t>(A.first_block) + blockIdx.x;
  if (row >= count_of(A.num, A.max_rows)) return;
  const T* t = static_cast<const T*>(A.t) + row * A.t_stride;
  const T* dy = static_cast<const T*>(A.dy) + row * A.dy_stride;
  const T* dt = A.dt ? static_cast<const T*>(A.dt) + row * A.dt_stride : nullptr;
  T* dx = static_cast<T*>(A.dx) + row * A.dx_stride;
  const float r = A.rstd[row];
  const int vectors = (A.dim + V - 1) / V;
  double s = 0.0;
  for (int i = threadIdx.x; i < vectors; i += kThreads) {
    const Columns<V> c(i, A.dim);
    const Elems<T, V> et = *reinterpret_cast<const Elems<T, V>*>(t + c.start);
    const Elems<T, V> ey = *reinterpret_cast<const Elems<T, V>*>(dy + c.start);
    float w[V];
    load_params<T, V>(A.w, A.float_params != 0, c.start, 1.f, w);
#pragma unroll
    for (int j = 0; j < V; ++j) s += j >= c.dup ? (as_float(ey.v[j]) * w[j]) * (as_float(et.v[j]) * r) : 0.f;
  }
  const float c2 = static_cast<float>(group_sum<kThreads>(s, lds) / A.dim);
  for (int i = threadIdx.x; i < vectors; i += kThreads) {
    const Columns<V> c(i, A.dim);
    const Elems<T, V> et = *reinterpret_cast<const Elems<T, V>*>(t + c.start);
    const Elems<T, V> ey = *reinterpret_cast<const Elems<T, V>*>(dy + c.start);
    Elems<T, V> ed = {};
    if (dt) ed = *reinterpret_cast<const Elems<T, V>*>(dt + c.start);
    float w[V];
    load_params<T, V>(A.w, A.float_params != 0, c.start, 1.f, w);
    Elems<T, V> o;
#pragma unroll
    for (int j = 0; j < V; ++j) o.v[j] = from_float<T>(r * (as_float(ey.v[j]) * w[j] - as_float(et.v[j]) * r * c2) + (dt ? as_float(ed.v[j]) : 0.f));
    store_own(dx + c.start, o, c.dup);
  }
}

// Slice blockIdx.y of the rows, V columns a thread.  Where dx takes the place of dy or of the sum it has to run before it.
template <typename T, int V>
__global__ void __launch_bounds__(kThreads) k_rms_grad_columns(RmsGradArgs A) {
  const int64_t n = count_of(A.num, A.max_rows);
  const Columns<V> c(static_cast<int>(blockIdx.x * kThreads + threadIdx.x), A.dim);
  if (c.dup == V) return;
  float dw[V] = {};
  for (int64_t row = blockIdx.y; row < n; row += gridDim.y) {
    const Elems<T, V> et = *reinterpret_cast<const Elems<T, V>*>(static_cast<const T*>(A.t) + row * A.t_stride + c.start);
    const Elems<T, V> ey = *reinterpret_cast<const Elems<T, V>*>(static_cast<const T*>(A.dy) + row * A.dy_stride + c.start);
    const float r = A.rstd[row];
#pragma unroll
    for (int j = 0; j < V; ++j) dw[j] += as_float(ey.v[j]) * (as_float(et.v[j]) * r);
  }
  float* out = A.part + static_cast<int64_t>(blockIdx.y) * A.dim;
#pragma unroll
  for (int j = 0; j < V; ++j)
    if (j >= c.dup) out[c.start + j] = dw[j];
}

// dw from the slices' sums, as k_norm_grad_join.
template <typename P>
__global__ void __launch_bounds__(kNormJoinThreads) k_rms_grad_join(const float* __restrict__ part, int32_t slices, int32_t dim, P* dw) {
  __shared__ float lds[kNormJoinThreads];
  const int64_t i = static_cast<int64_t>(blockIdx.x) * kNormJoinCols + threadIdx.x % kNormJoinCols;
  const float s = join_slices(part, slices, dim, i, lds);
  if (threadIdx.x < kNormJoinCols && i < dim) dw[i] = from_float<P>(s);
}

}  // namespace smfg_dev

#endif  // SMFG_KERNELS_RMS_H_
