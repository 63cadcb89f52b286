// libsmfg layer norm over rows, and its gradient.
//
//   m = mean(x_i), r = 1 / sqrt(mean((x_i - m)^2) + eps), y_ij = (x_ij - m) r w_j + b_j
//   h = (x - m) r, g = dy w:  dx = r (g - mean(g) - h mean(g h)),  dw_j = sum_i dy_ij h_ij,  db_j = sum_i dy_ij
#ifndef SMFG_KERNELS_NORM_H_
#define SMFG_KERNELS_NORM_H_

#include "elements.h"

namespace smfg_dev {

struct NormArgs {
  const void* x;
  int64_t x_stride;
  const int64_t* num;
  int64_t max_rows;
  int32_t dim;
  int32_t float_params;
  const void* w;
  const void* b;
  float eps;
  void* y;
  int64_t y_stride;
  float* mean;
  float* rstd;
  uint32_t first_block;  // of the launch, where a row is a block's
};

// Threads of a block whose groups of LANES lanes have a row each.
constexpr int norm_threads(int lanes) { return lanes > kThreads ? lanes : kThreads; }

// A group of LANES lanes has a row in its registers, NV vectors of V columns a lane: read once, centred before it is squared.  A block
// strides over rows, so that the parameters stay in registers, and asks for a row while the one before is worked on; the first is on its
// way together with the number of rows, as a launch has no more groups than the arrays have rows.  Memory bounds it: 154 K rows of 256 halfs
// 33 us, 4.8 TB/s, the rate of a copy.
template <typename T, int V, int NV, int LANES>
__global__ void __launch_bounds__(norm_threads(LANES)) k_layer_norm(NormArgs A) {
  __shared__ float lds[2][norm_threads(LANES) / 64];
  constexpr int kGroups = norm_threads(LANES) / LANES;
  const int lane = threadIdx.x % LANES;
  const int64_t step = static_cast<int64_t>(gridDim.x) * kGroups;
  int64_t row = static_cast<int64_t>(blockIdx.x) * kGroups + threadIdx.x / LANES;
  const bool ragged = A.dim % V != 0;
  const T* const x = static_cast<const T*>(A.x);
  Elems<T, V> e[NV];
  float w[NV][V], b[NV][V];
  const auto load = [&](int64_t i) {
#pragma unroll
    for (int k = 0; k < NV; ++k) e[k] = *reinterpret_cast<const Elems<T, V>*>(x + i * A.x_stride + Columns<V>(k * LANES + lane, A.dim).start);
  };
  load(row < A.max_rows ? row : A.max_rows - 1);
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const Columns<V> c(k * LANES + lane, A.dim);
    load_params<T, V>(A.w, A.float_params != 0, c.start, 1.f, w[k]);
    load_params<T, V>(A.b, A.float_params != 0, c.start, 0.f, b[k]);
  }
  const int64_t n = count_of(A.num, A.max_rows);
  for (; row < n; row += step) {
    float v[NV][V];
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const Columns<V> c(k * LANES + lane, A.dim);
      float part = 0.f;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        v[k][j] = as_float(e[k].v[j]);
        if (ragged && j < c.dup) continue;
        part += v[k][j];
      }
      s += c.dup < V ? part : 0.f;
    }
    if (row + step < n) load(row + step);
    const float m = group_sum<LANES>(s, lds[0]) / static_cast<float>(A.dim);
    s = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const Columns<V> c(k * LANES + lane, A.dim);
      float part = 0.f;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        v[k][j] -= m;
        if (ragged && j < c.dup) continue;
        part += v[k][j] * v[k][j];
      }
      s += c.dup < V ? part : 0.f;
    }
    const float r = 1.f / sqrtf(group_sum<LANES>(s, lds[1]) / static_cast<float>(A.dim) + A.eps);
    if (lane == 0) {
      if (A.mean) A.mean[row] = m;
      if (A.rstd) A.rstd[row] = r;
    }
    T* y = static_cast<T*>(A.y) + row * A.y_stride;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const Columns<V> c(k * LANES + lane, A.dim);
      if (c.dup == V) continue;
      Elems<T, V> o;
#pragma unroll
      for (int j = 0; j < V; ++j) o.v[j] = from_float<T>(v[k][j] * r * w[k][j] + b[k][j]);
      *reinterpret_cast<Elems<T, V>*>(y + c.start) = o;
    }
  }
}

// Rows that outgrow the registers of a block: one to a block, read three times.  The columns that the last vector shares with the
// one before are written once, as y may be x.  A thread adds dim / 256 columns, one after the other: in double, as a chain of floats rounds to one
// side where all columns are alike (the mean of 2^20 columns of 100.1 was off by 0.0025, which the factor r makes 0.8); it costs 2 % at most.
// 4096 rows of 20 000 floats 255 us (2.6 TB/s), of 32 768 halfs 292, 64 of 2^20 floats 2165: with few rows most of the chip has none.
template <typename T, int V>
__global__ void __launch_bounds__(kThreads) k_layer_norm_long(NormArgs A) {
  __shared__ double lds[2][kThreads / 64];
  const int64_t row = static_cast<int64_t>(A.first_block) + blockIdx.x;
  if (row >= count_of(A.num, A.max_rows)) return;
  const T* x = static_cast<const T*>(A.x) + row * A.x_stride;
  const int vectors = (A.dim + V - 1) / V;
  double s = 0.0;
  for (int i = threadIdx.x; i < vectors; i += kThreads) {
    const Columns<V> c(i, A.dim);
    const Elems<T, V> e = *reinterpret_cast<const Elems<T, V>*>(x + c.start);
#pragma unroll
    for (int j = 0; j < V; ++j) s += j >= c.dup ? as_float(e.v[j]) : 0.f;
  }
  const float m = static_cast<float>(group_sum<kThreads>(s, lds[0]) / A.dim);
  s = 0.0;
  for (int i = threadIdx.x; i < vectors; i += kThreads) {
    const Columns<V> c(i, A.dim);
    const Elems<T, V> e = *reinterpret_cast<const Elems<T, V>*>(x + c.start);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const double d = as_float(e.v[j]) - m;
      s += j >= c.dup ? d * d : 0.0;
    }
  }
  const float r = 1.f / sqrtf(static_cast<float>(group_sum<kThreads>(s, lds[1]) / A.dim) + A.eps);
  if (threadIdx.x == 0) {
    if (A.mean) A.mean[row] = m;
    if (A.rstd) A.rstd[row] = r;
  }
  T* y = static_cast<T*>(A.y) + row * A.y_stride;
  for (int i = threadIdx.x; i < vectors; i += kThreads) {
    const Columns<V> c(i, A.dim);
    const Elems<T, V> e = *reinterpret_cast<const Elems<T, V>*>(x + c.start);
    float w[V], b[V];
    load_params<T, V>(A.w, A.float_params != 0, c.start, 1.f, w);
    load_params<T, V>(A.b, A.float_params != 0, c.start, 0.f, b);
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (j >= c.dup) y[c.start + j] = from_float<T>((as_float(e.v[j]) - m) * r * w[j] + b[j]);
  }
}

struct NormGradArgs {
  const void* dy;
  int64_t dy_stride;
  const void* x;
  int64_t x_stride;
  const int64_t* num;
  int64_t max_rows;
  int32_t dim;
  int32_t float_params;
  const void* w;
  const float* mean;
  const float* rstd;
  void* dx;  // or null
  int64_t dx_stride;
  float* part;  // [slices][2][dim]: sums of dy h and of dy over the rows of a slice, or null
  uint32_t first_block;  // of the launch, where a row is a block's
};

// As k_layer_norm, a block striding over rows: a lane's columns are the same in each of them, so the sums for dw and db stay in
// its registers until the block is done, and leave it once, as a slice of `part`.  A row is asked for while the one before is worked on.
// 16 K rows of 4096 bfloat16 80 us (5.0 TB/s), 47 K of 301 floats 35 us (4.8 TB/s); waiting for each row took 131 us for the first.
template <typename T, int V, int NV, int LANES>
__global__ void __launch_bounds__(norm_threads(LANES)) k_layer_norm_grad(NormGradArgs A) {
  __shared__ float lds[2][2][norm_threads(LANES) / 64];
  constexpr int kGroups = norm_threads(LANES) / LANES;
  const int lane = threadIdx.x % LANES;
  const int64_t n = count_of(A.num, A.max_rows), step = static_cast<int64_t>(gridDim.x) * kGroups;
  const float inv = 1.f / static_cast<float>(A.dim);
  const bool ragged = A.dim % V != 0;
  float w[NV][V], dw[NV][V], db[NV][V];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const Columns<V> c(k * LANES + lane, A.dim);
    load_params<T, V>(A.w, A.float_params != 0, c.start, 1.f, w[k]);
#pragma unroll
    for (int j = 0; j < V; ++j) dw[k][j] = db[k][j] = 0.f;
  }
  const T* const x = static_cast<const T*>(A.x);
  const T* const dy = static_cast<const T*>(A.dy);
  Elems<T, V> ex[NV], ey[NV];
  float m = 0.f, r = 0.f;
  const auto load = [&](int64_t row) {
    m = A.mean[row];
    r = A.rstd[row];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const Columns<V> c(k * LANES + lane, A.dim);
      ex[k] = *reinterpret_cast<const Elems<T, V>*>(x + row * A.x_stride + c.start);
      ey[k] = *reinterpret_cast<const Elems<T, V>*>(dy + row * A.dy_stride + c.start);
    }
  };
  int64_t row = static_cast<int64_t>(blockIdx.x) * kGroups + threadIdx.x / LANES;
  if (row < n) load(row);
  for (int turn = 0; row < n; row += step, turn ^= 1) {
    float h[NV][V], g[NV][V];
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const Columns<V> c(k * LANES + lane, A.dim);
      float s1 = 0.f, s2 = 0.f;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        h[k][j] = (as_float(ex[k].v[j]) - m) * r;
        const float d = as_float(ey[k].v[j]);
        dw[k][j] += d * h[k][j];
        db[k][j] += d;
        g[k][j] = d * w[k][j];
        if (ragged && j < c.dup) continue;
        s1 += g[k][j];
        s2 += g[k][j] * h[k][j];
      }
      s[0] += c.dup < V ? s1 : 0.f;
      s[1] += c.dup < V ? s2 : 0.f;
    }
    const float scale = r;
    if (row + step < n) load(row + step);
    if (!A.dx) continue;
    // both sums at once; the array of the turn before is still being read
#pragma unroll
    for (int o = 1; o < (LANES < 64 ? LANES : 64); o <<= 1) {
      s[0] += __shfl_xor(s[0], o, 64);
      s[1] += __shfl_xor(s[1], o, 64);
    }
    if constexpr (LANES > 64) {
      if ((threadIdx.x & 63) == 0) {
        lds[turn][0][threadIdx.x >> 6] = s[0];
        lds[turn][1][threadIdx.x >> 6] = s[1];
      }
      __syncthreads();
      s[0] = s[1] = 0.f;
#pragma unroll
      for (int q = 0; q < LANES / 64; ++q) {
        s[0] += lds[turn][0][q];
        s[1] += lds[turn][1][q];
      }
    }
    const float c1 = s[0] * inv, c2 = s[1] * inv;
    T* dx = static_cast<T*>(A.dx) + row * A.dx_stride;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const Columns<V> c(k * LANES + lane, A.dim);
      if (c.dup == V) continue;
      Elems<T, V> e;
#pragma unroll
      for (int j = 0; j < V; ++j) e.v[j] = from_float<T>(scale * (g[k][j] - c1 - h[k][j] * c2));
      *reinterpret_cast<Elems<T, V>*>(dx + c.start) = e;
    }
  }
  if (!A.part) return;
  // groups of a wave, then waves, always in the same order
  constexpr int kWidth = LANES * NV * V;
  __shared__ float sums[LANES <= 64 ? kThreads / 64 * kWidth : 1];
  float* out = A.part + static_cast<int64_t>(blockIdx.x) * 2 * A.dim;
#pragma unroll
  for (int what = 0; what < 2; ++what) {
    float(&acc)[NV][V] = what == 0 ? dw : db;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
#pragma unroll
      for (int j = 0; j < V; ++j)
#pragma unroll
        for (int o = LANES; o < 64; o <<= 1) acc[k][j] += __shfl_xor(acc[k][j], o, 64);
    }
    if constexpr (LANES > 64) {
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const Columns<V> c(k * LANES + lane, A.dim);
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (j >= c.dup) out[what * static_cast<int64_t>(A.dim) + c.start + j] = acc[k][j];
      }
    } else {
      __syncthreads();
      if ((threadIdx.x & 63) < LANES) {
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
          for (int j = 0; j < V; ++j) sums[(threadIdx.x >> 6) * kWidth + (k * V + j) * LANES + lane] = acc[k][j];
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
        out[what * static_cast<int64_t>(A.dim) + c.start + j] = s;
      }
    }
  }
}

// Rows that outgrow the registers of a block: dx by a block per row, which reads it twice and adds in
// double, as k_layer_norm_long; the sums by k_norm_grad_columns.  4096 rows of 20 000 floats 371 us (2.7 TB/s), with dw and db 496; of 32 768 halfs 351 and 464.
template <typename T, int V>
__global__ void __launch_bounds__(kThreads) k_layer_norm_grad_long(NormGradArgs A) {
  __shared__ double lds[2][kThreads / 64];
  const int64_t row = static_cast<int64_t>(A.first_block) + blockIdx.x;
  if (row >= count_of(A.num, A.max_rows)) return;
  const T* x = static_cast<const T*>(A.x) + row * A.x_stride;
  const T* dy = static_cast<const T*>(A.dy) + row * A.dy_stride;
  T* dx = static_cast<T*>(A.dx) + row * A.dx_stride;
  const float m = A.mean[row], r = A.rstd[row];
  const int vectors = (A.dim + V - 1) / V;
  double s1 = 0.0, s2 = 0.0;
  for (int i = threadIdx.x; i < vectors; i += kThreads) {
    const Columns<V> c(i, A.dim);
    const Elems<T, V> ex = *reinterpret_cast<const Elems<T, V>*>(x + c.start);
    const Elems<T, V> ey = *reinterpret_cast<const Elems<T, V>*>(dy + c.start);
    float w[V];
    load_params<T, V>(A.w, A.float_params != 0, c.start, 1.f, w);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float g = as_float(ey.v[j]) * w[j], h = (as_float(ex.v[j]) - m) * r;
      s1 += j >= c.dup ? g : 0.f;
      s2 += j >= c.dup ? g * h : 0.f;
    }
  }
  const float c1 = static_cast<float>(group_sum<kThreads>(s1, lds[0]) / A.dim), c2 = static_cast<float>(group_sum<kThreads>(s2, lds[1]) / A.dim);
  for (int i = threadIdx.x; i < vectors; i += kThreads) {
    const Columns<V> c(i, A.dim);
    const Elems<T, V> ex = *reinterpret_cast<const Elems<T, V>*>(x + c.start);
    const Elems<T, V> ey = *reinterpret_cast<const Elems<T, V>*>(dy + c.start);
    float w[V];
    load_params<T, V>(A.w, A.float_params != 0, c.start, 1.f, w);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float g = as_float(ey.v[j]) * w[j], h = (as_float(ex.v[j]) - m) * r;
      if (j >= c.dup) dx[c.start + j] = from_float<T>(r * (g - c1 - h * c2));
    }
  }
}

// Slice blockIdx.y of the rows, V columns a thread.  Where dx takes the place of dy or x it has to run before it.
template <typename T, int V>
__global__ void __launch_bounds__(kThreads) k_norm_grad_columns(NormGradArgs A) {
  const int64_t n = count_of(A.num, A.max_rows);
  const Columns<V> c(static_cast<int>(blockIdx.x * kThreads + threadIdx.x), A.dim);
  if (c.dup == V) return;
  float dw[V] = {}, db[V] = {};
  for (int64_t row = blockIdx.y; row < n; row += gridDim.y) {
    const Elems<T, V> ex = *reinterpret_cast<const Elems<T, V>*>(static_cast<const T*>(A.x) + row * A.x_stride + c.start);
    const Elems<T, V> ey = *reinterpret_cast<const Elems<T, V>*>(static_cast<const T*>(A.dy) + row * A.dy_stride + c.start);
    const float m = A.mean[row], r = A.rstd[row];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float d = as_float(ey.v[j]);
      dw[j] += d * ((as_float(ex.v[j]) - m) * r);
      db[j] += d;
    }
  }
  float* out = A.part + static_cast<int64_t>(blockIdx.y) * 2 * A.dim;
#pragma unroll
  for (int j = 0; j < V; ++j)
    if (j >= c.dup) {
      out[c.start + j] = dw[j];
      out[static_cast<int64_t>(A.dim) + c.start + j] = db[j];
    }
}

// dw and db (either may be null) from the slices' sums: 16 columns to a block, the slices dealt to its 64 rows of threads (with 8 rows of
// threads 1024 slices of 602 sums took 35 us, the 128 loads of a thread one after the other).
constexpr int kNormJoinCols = 16;
constexpr int kNormJoinThreads = 1024;
constexpr int kNormJoinRows = kNormJoinThreads / kNormJoinCols;
// The sum of column i over the slices' sums, in the first kNormJoinCols threads of the block.
__device__ __forceinline__ float join_slices(const float* __restrict__ part, int32_t slices, int64_t width, int64_t i, float* lds) {
  const float* p = part + (i < width ? i : width - 1);
  float s = 0.f;
#pragma unroll 8
  for (int q = threadIdx.x / kNormJoinCols; q < slices; q += kNormJoinRows) s += p[q * width];
  lds[threadIdx.x] = s;
  __syncthreads();
  if (threadIdx.x < 128) {
    s = 0.f;
#pragma unroll
    for (int q = 0; q < 8; ++q) s += lds[(threadIdx.x / kNormJoinCols + 8 * q) * kNormJoinCols + threadIdx.x % kNormJoinCols];
  }
  __syncthreads();
  if (threadIdx.x < 128) lds[threadIdx.x] = s;
  __syncthreads();
  s = 0.f;
  if (threadIdx.x < kNormJoinCols) {
#pragma unroll
    for (int q = 0; q < 8; ++q) s += lds[q * kNormJoinCols + threadIdx.x];
  }
  return s;
}
template <typename P>
__global__ void __launch_bounds__(kNormJoinThreads) k_norm_grad_join(const float* __restrict__ part, int32_t slices, int32_t dim, P* dw, P* db) {
  __shared__ float lds[kNormJoinThreads];
  const int64_t width = 2 * static_cast<int64_t>(dim), i = static_cast<int64_t>(blockIdx.x) * kNormJoinCols + threadIdx.x % kNormJoinCols;
  const float s = join_slices(part, slices, width, i, lds);
  if (threadIdx.x >= kNormJoinCols || i >= width) return;
  P* out = i < dim ? dw : db;
  if (out) out[i < dim ? i : i - dim] = from_float<P>(s);
}

}  // namespace smfg_dev

#endif  // SMFG_KERNELS_NORM_H_
