// libsmfg softmax cross entropy over rows of logits, with the logits' gradient in the same pass.
//
//   M_i = max_j x_ij, S_i = sum_j exp(x_ij - M_i),  loss_i = log S_i - (x_iy - M_i),  p_ij = exp(x_ij - M_i) / S_i
//   dx_ij = c (p_ij - [j = y_i]),  c = scale, or scale divided by the number of rows with a label
#ifndef SMFG_KERNELS_LOSS_H_
#define SMFG_KERNELS_LOSS_H_

#include "elements.h"

namespace smfg_dev {

// What a block leaves of its rows.
struct LossPart {
  double sum;
  int64_t rows;  // with a label
};
struct LossArgs {
  const void* x;
  int64_t x_stride;
  const void* labels;
  int32_t label_bytes;
  int32_t classes;
  const int64_t* num;
  int64_t max_rows;
  int32_t mean;
  float scale;
  void* dx;  // or null
  int64_t dx_stride;
  float* row_loss;  // or null
  float* loss;
  LossPart* part;
  int32_t parts;
  int64_t* counts;  // rows with a label among each kCountRows of them
  int32_t num_counts;  // 0: every block counts them itself
};

constexpr int kCountRows = 8192;
constexpr float kLog2E = 1.44269504088896340736f;

__device__ __forceinline__ int64_t label_of(const LossArgs& A, int64_t row) {
  return A.label_bytes == 8 ? static_cast<const int64_t*>(A.labels)[row] : static_cast<const int32_t*>(A.labels)[row];
}
__device__ __forceinline__ bool is_class(int64_t label, int32_t classes) { return static_cast<uint64_t>(label) < static_cast<uint64_t>(classes); }

// Rows with a label in [from, to), in every thread of the block.
template <int THREADS>
__device__ __forceinline__ int64_t count_labels(const LossArgs& A, int64_t from, int64_t to, int64_t* lds) {
  int s = 0;
  for (int64_t i = from + threadIdx.x; i < to; i += THREADS) s += is_class(label_of(A, i), A.classes);
  return group_sum<THREADS>(static_cast<int64_t>(s), lds);
}
static __global__ void __launch_bounds__(1024) k_loss_count(LossArgs A) {
  __shared__ int64_t lds[16];
  const int64_t n = count_of(A.num, A.max_rows), from = static_cast<int64_t>(blockIdx.x) * kCountRows, to = from + kCountRows;
  const int64_t s = count_labels<1024>(A, from, to < n ? to : n, lds);
  if (threadIdx.x == 0) A.counts[blockIdx.x] = s;
}

// c for all rows.
template <int THREADS>
__device__ __forceinline__ float gradient_scale(const LossArgs& A, int64_t n, int64_t* lds) {
  if (!A.mean || !A.dx) return A.scale;
  int64_t rows;
  if (A.num_counts == 0) {
    rows = count_labels<THREADS>(A, 0, n, lds);
  } else {
    int64_t s = 0;
    for (int i = threadIdx.x; i < A.num_counts; i += THREADS) s += A.counts[i];
    rows = group_sum<THREADS>(s, lds);
  }
  return rows > 0 ? A.scale / static_cast<float>(rows) : 0.f;
}

// exp(x) by the hardware's power of two: a result below 2^-126 is zero.
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2E); }

// Maximum, and sum of exponentials relative to it, of several lanes: each lane brings its own maximum (-inf: none) and its sum relative to that.
struct SoftSum {
  float m, s;
};
// A maximum of -inf is taken for 0: the exponentials are zeros then, not NaN.
__device__ __forceinline__ float base_of(float m) { return m == -__builtin_inff() ? 0.f : m; }
template <int LANES>
__device__ __forceinline__ SoftSum wave_soft_sum(SoftSum a) {
  float m = a.m;
#pragma unroll
  for (int o = 1; o < LANES; o <<= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
  float s = a.s * exp_of(a.m - base_of(m));
#pragma unroll
  for (int o = 1; o < LANES; o <<= 1) s += __shfl_xor(s, o, 64);
  return {m, s};
}
template <int LANES>
__device__ __forceinline__ SoftSum group_soft_sum(SoftSum a, SoftSum* lds) {
  a = wave_soft_sum<(LANES < 64 ? LANES : 64)>(a);
  if constexpr (LANES > 64) {
    constexpr int kWaves = LANES / 64;
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = a;
    __syncthreads();
    a = wave_soft_sum<kWaves>(lds[threadIdx.x & (kWaves - 1)]);
  }
  return a;
}

// The block's sums of its threads' losses.
template <int THREADS>
__device__ __forceinline__ void leave_part(const LossArgs& A, double sum, int rows) {
  __shared__ double sums[THREADS / 64];
  __shared__ int64_t counts[THREADS / 64];
  __syncthreads();
  sum = group_sum<THREADS>(sum, sums);
  const int64_t all = group_sum<THREADS>(static_cast<int64_t>(rows), counts);
  if (threadIdx.x == 0) A.part[blockIdx.x] = {sum, all};
}

constexpr int loss_threads(int lanes) { return lanes > kThreads ? lanes : kThreads; }

// A group of LANES lanes has a row in its registers, NV vectors of V columns a lane: read once, its exponentials kept until their sum is known, and asks for
// its next row while it works on it.  The lane that has the label's column works out the loss.
template <typename T, int V, int NV, int LANES>
__global__ void __launch_bounds__(loss_threads(LANES)) k_cross_entropy(LossArgs A) {
  constexpr int kBlock = loss_threads(LANES), kGroups = kBlock / LANES;
  __shared__ SoftSum lds[2][kBlock / 64];
  __shared__ int64_t count_lds[kBlock / 64];
  const int lane = threadIdx.x % LANES;
  const int64_t step = static_cast<int64_t>(gridDim.x) * kGroups;
  int64_t row = static_cast<int64_t>(blockIdx.x) * kGroups + threadIdx.x / LANES;
  const bool ragged = A.classes % V != 0;
  const T* const x = static_cast<const T*>(A.x);
  Elems<T, V> e[NV];
  int64_t label = 0;
  const auto load = [&](int64_t i) {
    label = label_of(A, i);
#pragma unroll
    for (int k = 0; k < NV; ++k) e[k] = *reinterpret_cast<const Elems<T, V>*>(x + i * A.x_stride + Columns<V>(k * LANES + lane, A.classes).start);
  };
  load(row < A.max_rows ? row : A.max_rows - 1);
  const int64_t n = count_of(A.num, A.max_rows);
  const float c = gradient_scale<kBlock>(A, n, count_lds);
  double sum = 0.0;
  int rows = 0;
  for (int turn = 0; row < n; row += step, turn ^= 1) {
    float v[NV][V];
    SoftSum a = {-__builtin_inff(), 0.f};
#pragma unroll
    for (int k = 0; k < NV; ++k) {
#pragma unroll
      for (int j = 0; j < V; ++j) v[k][j] = as_float(e[k].v[j]);
      // columns that two vectors share do no harm to the maximum
#pragma unroll
      for (int j = 0; j < V; ++j) a.m = fmaxf(a.m, v[k][j]);
    }
    const bool live = is_class(label, A.classes);
    const int y = live ? static_cast<int>(label) : -1;
    if (row + step < n) load(row + step);
    const float base = base_of(a.m);
    float xy = 0.f;
    bool owner = false;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const Columns<V> col(k * LANES + lane, A.classes);
      const int at = y - col.start;
      if (static_cast<unsigned>(at) < static_cast<unsigned>(V) && at >= col.dup) {
        owner = true;
#pragma unroll
        for (int j = 0; j < V; ++j) xy = at == j ? v[k][j] : xy;
      }
      float part = 0.f;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        v[k][j] = exp_of(v[k][j] - base);
        if (ragged && j < col.dup) continue;
        part += v[k][j];
      }
      a.s += col.dup < V ? part : 0.f;
    }
    const SoftSum all = group_soft_sum<LANES>(a, lds[turn]);
    if (owner || (!live && lane == 0)) {
      const float loss = live ? logf(all.s) - (xy - base_of(all.m)) : 0.f;
      if (A.row_loss) A.row_loss[row] = loss;
      sum += loss;
      rows += live;
    }
    if (!A.dx) continue;
    const float f = exp_of(base - base_of(all.m)) * (c / all.s);
    T* dx = static_cast<T*>(A.dx) + row * A.dx_stride;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const Columns<V> col(k * LANES + lane, A.classes);
      if (col.dup == V) continue;
      const int at = y - col.start;
#pragma unroll
      for (int j = 0; j < V; ++j) v[k][j] = live ? v[k][j] * f : 0.f;
      if (static_cast<unsigned>(at) < static_cast<unsigned>(V)) {
#pragma unroll
        for (int j = 0; j < V; ++j) v[k][j] -= at == j ? c : 0.f;
      }
      Elems<T, V> o;
#pragma unroll
      for (int j = 0; j < V; ++j) o.v[j] = from_float<T>(v[k][j]);
      // columns that two vectors share have other roundings in each, as the lanes' maxima differ: the first writes them
      store_own(dx + col.start, o, ragged ? col.dup : 0);
    }
  }
  leave_part<kBlock>(A, sum, rows);
}

// Rows that outgrow the registers of a block: one to a block at a time, read twice.  A thread has the same columns both times and writes no others, so
// that the gradient may take the place of the logits.
constexpr int kLongLossThreads = 1024;
template <typename T, int V>
__global__ void __launch_bounds__(kLongLossThreads) k_cross_entropy_long(LossArgs A) {
  __shared__ SoftSum lds[2][kLongLossThreads / 64];
  __shared__ int64_t count_lds[kLongLossThreads / 64];
  const int64_t n = count_of(A.num, A.max_rows);
  const float c = gradient_scale<kLongLossThreads>(A, n, count_lds);
  const int vectors = (A.classes + V - 1) / V;
  double sum = 0.0;
  int rows = 0, turn = 0;
  for (int64_t row = blockIdx.x; row < n; row += gridDim.x, turn ^= 1) {
    const T* x = static_cast<const T*>(A.x) + row * A.x_stride;
    const int64_t label = label_of(A, row);
    const bool live = is_class(label, A.classes);
    const int y = live ? static_cast<int>(label) : -1;
    SoftSum a = {-__builtin_inff(), 0.f};
    float xy = 0.f;
    bool owner = false;
#pragma unroll 4
    for (int i = threadIdx.x; i < vectors; i += kLongLossThreads) {
      const Columns<V> col(i, A.classes);
      const Elems<T, V> e = *reinterpret_cast<const Elems<T, V>*>(x + col.start);
      float m = a.m;
#pragma unroll
      for (int j = 0; j < V; ++j) m = j >= col.dup ? fmaxf(m, as_float(e.v[j])) : m;
      const float base = base_of(m);
      a.s *= exp_of(a.m - base);
      a.m = m;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        if (j < col.dup) continue;
        a.s += exp_of(as_float(e.v[j]) - base);
        if (col.start + j == y) {
          owner = true;
          xy = as_float(e.v[j]);
        }
      }
    }
    const SoftSum all = group_soft_sum<kLongLossThreads>(a, lds[turn]);
    if (owner || (!live && threadIdx.x == 0)) {
      const float loss = live ? logf(all.s) - (xy - base_of(all.m)) : 0.f;
      if (A.row_loss) A.row_loss[row] = loss;
      sum += loss;
      rows += live;
    }
    if (!A.dx) continue;
    const float base = base_of(all.m), f = c / all.s;
    T* dx = static_cast<T*>(A.dx) + row * A.dx_stride;
#pragma unroll 4
    for (int i = threadIdx.x; i < vectors; i += kLongLossThreads) {
      const Columns<V> col(i, A.classes);
      const Elems<T, V> e = *reinterpret_cast<const Elems<T, V>*>(x + col.start);
      Elems<T, V> o;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float p = live ? exp_of(as_float(e.v[j]) - base) * f : 0.f;
        o.v[j] = from_float<T>(p - (col.start + j == y ? c : 0.f));
      }
      store_own(dx + col.start, o, col.dup);
    }
  }
  leave_part<kLongLossThreads>(A, sum, rows);
}

// The loss from the blocks' sums; of no rows with a label 0.
static __global__ void __launch_bounds__(kThreads) k_loss_join(LossArgs A) {
  __shared__ double sums[kThreads / 64];
  __shared__ int64_t counts[kThreads / 64];
  double s = 0.0;
  int64_t rows = 0;
  for (int i = threadIdx.x; i < A.parts; i += kThreads) {
    s += A.part[i].sum;
    rows += A.part[i].rows;
  }
  s = group_sum<kThreads>(s, sums);
  rows = group_sum<kThreads>(rows, counts);
  if (threadIdx.x == 0) *A.loss = static_cast<float>(A.mean && rows > 0 ? s / static_cast<double>(rows) : s);
}

}  // namespace smfg_dev

#endif  // SMFG_KERNELS_LOSS_H_
