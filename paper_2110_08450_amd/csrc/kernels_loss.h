// libsmfg softmax cross entropy over rows of logits, with the logits' gradient in the same pass.
//
//   M_i = max_j x_ij, S_i = sum_j exp(x_ij - M_i),  loss_i = log S_i - (x_iy - M_i),  p_ij = exp(x_ij - M_i) / S_i
//   dx_ij = c (p_ij - [j = y_i]),  c = scale, or scale divided by the number of rows with a label
#ifndef SMFG_KERNELS_LOSS_H_
#define SMFG_KERNELS_LOSS_H_

#include <type_traits>

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
  int64_t* counts;  // rows with a label among each count_rows of them
  int32_t num_counts;  // 0: every block counts them itself
  int64_t count_rows;
  int32_t keep;  // the gradient stays in the caches
};

constexpr int kCountAll = 8192;  // up to so many rows every block counts all labels itself
constexpr float kLog2E = 1.44269504088896340736f;

__device__ __forceinline__ int64_t label_of(const LossArgs& A, int64_t row) {
  return A.label_bytes == 8 ? static_cast<const int64_t*>(A.labels)[row] : static_cast<const int32_t*>(A.labels)[row];
}
__device__ __forceinline__ bool is_class(int64_t label, int32_t classes) { return static_cast<uint64_t>(label) < static_cast<uint64_t>(classes); }

// Rows with a label in [from, to), in every thread of the block.
template <int THREADS>
__device__ __forceinline__ int64_t count_labels(const LossArgs& A, int64_t from, int64_t to, int64_t* lds) {
  int s = 0;
#pragma unroll 4
  for (int64_t i = from + threadIdx.x; i < to; i += THREADS) s += is_class(label_of(A, i), A.classes);
  return group_sum<THREADS>(static_cast<int64_t>(s), lds);
}
static __global__ void __launch_bounds__(kThreads) k_loss_count(LossArgs A) {
  __shared__ int64_t lds[kThreads / 64];
  const int64_t n = count_of(A.num, A.max_rows), from = static_cast<int64_t>(blockIdx.x) * A.count_rows, to = from + A.count_rows;
  const int64_t s = count_labels<kThreads>(A, from, to < n ? to : n, lds);
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

// exp(x), x <= 0, by the hardware's power of two: a result below 2^-126 is zero.  The exponent is a product of two rounded numbers, rounded: with the rounding of x
// itself a result is off by up to 3 * 2^-24 |x| of itself.
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2E); }

// Maximum, and sum of exponentials relative to it, of several lanes: each lane brings its own maximum (-inf: none) and its sum relative to that.
struct SoftSum {
  float m, s;
};
// A maximum of -inf is taken for 0: the exponentials are zeros then, not NaN.
__device__ __forceinline__ float base_of(float m) { return m == -__builtin_inff() ? 0.f : m; }
template <int LANES>
__device__ __forceinline__ SoftSum wave_soft_sum(SoftSum a) {
  const float m = lanes_all<LANES>(a.m, max_f);
  return {m, lanes_all<LANES>(a.s * exp_of(a.m - base_of(m)), sum_f)};
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

// The loss from the sum of the rows'; of no rows with a label 0.
__device__ __forceinline__ float loss_of(const LossArgs& A, double sum, int64_t rows) {
  return static_cast<float>(A.mean && rows > 0 ? sum / static_cast<double>(rows) : sum);
}
// The block's sums of its threads' losses, or the loss if there is no other block.
template <int THREADS>
__device__ __forceinline__ void leave_part(const LossArgs& A, double sum, int rows) {
  __shared__ double sums[THREADS / 64];
  __shared__ int64_t counts[THREADS / 64];
  __syncthreads();
  sum = group_sum<THREADS>(sum, sums);
  const int64_t all = group_sum<THREADS>(static_cast<int64_t>(rows), counts);
  if (threadIdx.x != 0) return;
  if (gridDim.x == 1) *A.loss = loss_of(A, sum, all);
  else A.part[blockIdx.x] = {sum, all};
}

constexpr int loss_threads(int lanes) { return lanes > kThreads ? lanes : kThreads; }

// A group of LANES lanes has a row in its registers, NV vectors of V columns a lane: it reads it once, keeps the exponentials until their sum is known, and has its
// next row on its way meanwhile.  The lane that has the label's column works out the loss.
// Logits of rows of 1024 lanes are read past the caches: of 1000 rows of 50 K bfloat16, 100 MB, 50.6 us instead of 57.0 (with a pass over the gradient behind 80 and 88); of
// 8192, where nothing stays in them, 321 and 314 (587 and 582), of 32 000 columns 200 either way.  Fewer lanes read through them: 10 K rows of 8192 70 us (past them 67.5), 8192 of
// 12 000 83.5 (84), 16 K of 4096 60 (54.7), 80 K of 1000 70.6 (68), 150 K of 172 halfs 37.2 (39.8), 50 K of 700 floats 61.5 (52.9).  Memory bounds it: 8192 rows of 50 K bfloat16
// 322 us, 5.1 TB/s; 33 K rows of 1013 floats 52 us, 5.2 TB/s.  All vectors but a lane's last are known to be whole: with places of their own they took the registers that the next
// row lies in (572 us for the first).
template <typename T, int V, int NV, int LANES>
__global__ void __launch_bounds__(loss_threads(LANES)) k_cross_entropy(LossArgs A) {
  constexpr int kBlock = loss_threads(LANES), kGroups = kBlock / LANES;
  __shared__ SoftSum lds[2][kBlock / 64];
  __shared__ int64_t count_lds[kBlock / 64];
  const int lane = threadIdx.x % LANES;
  const int64_t step = static_cast<int64_t>(gridDim.x) * kGroups;
  // rows of a wave or more are the same for its lanes: addresses of scalars then
  const int group = static_cast<int>(threadIdx.x) / LANES;
  int64_t row = static_cast<int64_t>(blockIdx.x) * kGroups + (LANES >= 64 ? __builtin_amdgcn_readfirstlane(group) : group);
  const bool ragged = A.classes % V != 0;
  const T* const x = static_cast<const T*>(A.x);
  Words<T, V> e[NV];
  int64_t label = 0;
  const auto columns = [&](int k) { return columns_of<V, NV, LANES>(k, lane, A.classes); };
  const auto load = [&](int64_t i) {
    label = label_of(A, i);
#pragma unroll
    for (int k = 0; k < NV; ++k) e[k] = load_words<T, V, LANES == 1024>(x + i * A.x_stride + static_cast<unsigned>(columns(k).start));
  };
  load(row < A.max_rows ? row : A.max_rows - 1);
  const int64_t n = count_of(A.num, A.max_rows);
  const float c = gradient_scale<kBlock>(A, n, count_lds);
  // Up to a wave the row's maximum is known to all lanes before the first exponential; beyond it each lane takes its own, so that one barrier does.
  constexpr bool kCommon = LANES <= 64;
  double sum = 0.0;
  int rows = 0;
  for (int turn = 0; row < n; row += step, turn ^= 1) {
    float v[NV][V];
    SoftSum a = {-__builtin_inff(), 0.f};
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      // columns that two vectors share do no harm to the maximum
#pragma unroll
      for (int j = 0; j < V; ++j) {
        v[k][j] = e[k][j];
        a.m = fmaxf(a.m, v[k][j]);
      }
    }
    const bool live = is_class(label, A.classes);
    const int y = live ? static_cast<int>(label) : -1;
    if (row + step < n) load(row + step);
    if constexpr (kCommon) a.m = lanes_all<LANES>(a.m, max_f);
    const float base = base_of(a.m);
    float xy = 0.f;
    bool owner = false;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      float(&u)[V] = v[k];
      const Columns<V> col = columns(k);
      const int at = y - col.start;
      if (static_cast<unsigned>(at) < static_cast<unsigned>(V) && at >= col.dup) {
        owner = true;
#pragma unroll
        for (int j = 0; j < V; ++j) xy = at == j ? u[j] : xy;
      }
      float part = 0.f;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        u[j] = exp_of(u[j] - base);
        if (ragged && j < col.dup) continue;
        part += u[j];
      }
      a.s += col.dup < V ? part : 0.f;
    }
    SoftSum all = {a.m, 0.f};
    if constexpr (kCommon) all.s = lanes_all<LANES>(a.s, sum_f);
    else all = group_soft_sum<LANES>(a, lds[turn]);
    if (owner || (!live && lane == 0)) {
      const float loss = live ? logf(all.s) - (xy - base_of(all.m)) : 0.f;
      if (A.row_loss) A.row_loss[row] = loss;
      sum += loss;
      rows += live;
    }
    if (!A.dx) continue;
    // A lane whose columns are all -infinity has a factor of 0 beside its zeros: from its base of 0 the factor would be infinite where the row's largest logit is below -88.
    const float f = (kCommon ? 1.f : exp_of(a.m - base_of(all.m))) * (c / all.s);
    T* dx = static_cast<T*>(A.dx) + row * A.dx_stride;
    const auto leave = [&](auto keep) {
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        float(&u)[V] = v[k];
        const Columns<V> col = columns(k);
        const int at = y - col.start;
#pragma unroll
        for (int j = 0; j < V; ++j) u[j] = live ? u[j] * f : 0.f;
        if (static_cast<unsigned>(at) < static_cast<unsigned>(V)) {
#pragma unroll
          for (int j = 0; j < V; ++j) u[j] -= at == j ? c : 0.f;
        }
        Elems<T, V> o;
#pragma unroll
        for (int j = 0; j < V; ++j) o.v[j] = from_float<T>(u[j]);
        // columns that two vectors share have the same bits in both but where the lanes' maxima differ: there the first writes them
        const int shared = kCommon && col.dup < V ? 0 : col.dup;
        if constexpr (decltype(keep)::value) store_own(dx + static_cast<unsigned>(col.start), o, shared);
        else store_once(dx + static_cast<unsigned>(col.start), o, shared);
      }
    };
    if (A.keep) leave(std::true_type{});
    else leave(std::false_type{});
  }
  leave_part<kBlock>(A, sum, rows);
}

// Rows that outgrow the registers of a block: one to a block at a time, read twice, four vectors of a thread at once (3000 rows of 128 K bfloat16 330 us, one at
// a time 475).  A thread has the same columns both times and
// writes no others, so that the gradient may take the place of the logits.
constexpr int kLongLossThreads = 1024;
template <typename T, int V>
__global__ void __launch_bounds__(kLongLossThreads) k_cross_entropy_long(LossArgs A) {
  constexpr int kTurns = 4;
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
    for (int first = threadIdx.x; first < vectors; first += kTurns * kLongLossThreads) {
      Words<T, V> e[kTurns];
#pragma unroll
      for (int k = 0; k < kTurns; ++k) e[k] = load_words<T, V, false>(x + static_cast<unsigned>(Columns<V>(first + k * kLongLossThreads, A.classes).start));
      float m = a.m;
#pragma unroll
      for (int k = 0; k < kTurns; ++k)
#pragma unroll
        for (int j = 0; j < V; ++j) m = fmaxf(m, e[k][j]);  // of columns of other threads as well, which does no harm
      const float base = base_of(m);
      a.s *= exp_of(a.m - base);
      a.m = m;
#pragma unroll
      for (int k = 0; k < kTurns; ++k) {
        const Columns<V> col(first + k * kLongLossThreads, A.classes);
        float part = 0.f;
#pragma unroll
        for (int j = 0; j < V; ++j) part += j >= col.dup ? exp_of(e[k][j] - base) : 0.f;
        a.s += part;
        const int at = y - col.start;
        if (static_cast<unsigned>(at) < static_cast<unsigned>(V) && at >= col.dup) {
          owner = true;
#pragma unroll
          for (int j = 0; j < V; ++j) xy = at == j ? e[k][j] : xy;
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
    for (int first = threadIdx.x; first < vectors; first += kTurns * kLongLossThreads) {
      Words<T, V> e[kTurns];
#pragma unroll
      for (int k = 0; k < kTurns; ++k) e[k] = load_words<T, V, true>(x + static_cast<unsigned>(Columns<V>(first + k * kLongLossThreads, A.classes).start));
#pragma unroll
      for (int k = 0; k < kTurns; ++k) {
        const Columns<V> col(first + k * kLongLossThreads, A.classes);
        const int at = y - col.start;
        float u[V];
#pragma unroll
        for (int j = 0; j < V; ++j) u[j] = live ? exp_of(e[k][j] - base) * f : 0.f;
        if (static_cast<unsigned>(at) < static_cast<unsigned>(V)) {
#pragma unroll
          for (int j = 0; j < V; ++j) u[j] -= at == j ? c : 0.f;
        }
        Elems<T, V> o;
#pragma unroll
        for (int j = 0; j < V; ++j) o.v[j] = from_float<T>(u[j]);
        if (A.keep) store_own(dx + static_cast<unsigned>(col.start), o, col.dup);
        else store_once(dx + static_cast<unsigned>(col.start), o, col.dup);
      }
    }
  }
  leave_part<kLongLossThreads>(A, sum, rows);
}

// The loss from the blocks' sums.
constexpr int kLossJoinThreads = 1024;
static __global__ void __launch_bounds__(kLossJoinThreads) k_loss_join(LossArgs A) {
  __shared__ double sums[kLossJoinThreads / 64];
  __shared__ int64_t counts[kLossJoinThreads / 64];
  double s = 0.0;
  int64_t rows = 0;
#pragma unroll 2
  for (int i = threadIdx.x; i < A.parts; i += kLossJoinThreads) {
    s += A.part[i].sum;
    rows += A.part[i].rows;
  }
  s = group_sum<kLossJoinThreads>(s, sums);
  rows = group_sum<kLossJoinThreads>(rows, counts);
  if (threadIdx.x == 0) *A.loss = loss_of(A, s, rows);
}

}  // namespace smfg_dev

#endif  // SMFG_KERNELS_LOSS_H_
