// libsmfg gradient clipping by the global norm over many tensors.
//
//   N = sqrt(sum over all elements of (scale g)^2),  c = min(1, max_norm / (N + 1e-6)),  out = scale c g
#ifndef SMFG_KERNELS_CLIP_H_
#define SMFG_KERNELS_CLIP_H_

#include "elements.h"

namespace smfg_dev {

// Up to kClipTensors tensors are in the arguments of the launches themselves.  More are written to a table in the scratch first, kClipTensors a
// launch, so that squares and scaling are one launch each: 290 tensors of 400 M halfs in four launches each took 743 us, one each 698: most of the
// difference is at their ends, where a launch no longer fills the chip.
// The table is indexed by a scalar register, and the compiler may split such an address between two of them; scalar loads drop
// the lowest two bits of each, so every index step has to be whole words (a table of bytes made pointers beside it garbage).
constexpr int kClipTensors = 80;
constexpr int64_t kClipLeast = 2048, kClipMost = 65536;  // elements of a block
struct ClipTensor {
  const void* src;
  void* dst;
  int64_t numel;
  const int64_t* rows;  // or null: the tensor counts up to *rows * row_elems elements
  int64_t row_elems;
  uint32_t first_block;  // block first_block + q has elements [q * chunk, (q + 1) * chunk)
  int32_t type;          // of src | of dst << 4
};
// scale * c = digits * 2^power.  The power is 0 but where the product is below 2^-100, as with a norm of 1e38 or a limit as small: a float has few
// digits left for it there, or none, while the gradients that it makes small are large.
struct ClipFactor {
  float digits;
  int power;
};
struct ClipArgs {
  ClipTensor t[kClipTensors];
  ClipTensor* table;    // of all tensors, or null: t has them all
  int32_t tensors;      // of the table, or of t
  int32_t first, here;  // tensors of the table that t has, for k_clip_table
  uint32_t blocks;
  uint32_t first_block;  // of the launch
  int64_t chunk;
  double* part;         // a block's sum of squares
  ClipFactor* factor;
  float* norm;
  float scale, max_norm;
};
static_assert(sizeof(ClipTensor) == 48 && sizeof(ClipArgs) <= 4096, "kernel arguments are limited to 4 KB");

static __global__ void __launch_bounds__(64) k_clip_table(ClipArgs A) {
  for (int i = threadIdx.x; i < A.here; i += 64) A.table[A.first + i] = A.t[i];
}

// The last tensor that begins at the block or before it.
template <bool TABLE>
__device__ __forceinline__ ClipTensor tensor_of_block(const ClipArgs& A, uint32_t block) {
  const int lane = threadIdx.x & 63;
  if constexpr (!TABLE) {
    int t = -1;
#pragma unroll
    for (int i = 0; i < kClipTensors; i += 64)
      t += __popcll(__ballot(i + lane < A.tensors && block >= A.t[i + lane < A.tensors ? i + lane : 0].first_block));
    return A.t[t];
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
__device__ __forceinline__ int64_t elements_of(const ClipTensor& T) {
  int64_t n = T.numel;
  if (T.rows) {
    const int64_t r = *T.rows, most = n / T.row_elems;
    n = (r < 0 ? 0 : r > most ? most : r) * T.row_elems;
  }
  return n;
}

// The elements of a block: those of its chunk, shifted back to where `base` is a multiple of 16 bytes, so that all vectors but the first chunk's
// single elements are aligned and rounds are whole (400 M halfs in 60 tensors at any address: 651 -> 645 us; with a few single elements at every chunk instead 665).
struct ClipRange {
  int64_t from, to;
  int ahead;  // single elements before the first vector
};
template <typename T>
__device__ __forceinline__ ClipRange range_of(const T* base, uint32_t q, int64_t chunk, int64_t numel, int64_t n) {
  const int past = static_cast<int>(reinterpret_cast<uintptr_t>(base) & 15) / static_cast<int>(sizeof(T));
  const int64_t from = q == 0 ? 0 : q * chunk - past;
  const bool last = (q + 1) * chunk >= numel;
  const int64_t to = last ? numel : (q + 1) * chunk - past;
  const int ahead = q == 0 && past > 0 ? 16 / static_cast<int>(sizeof(T)) - past : 0;
  return {from, to < n ? to : n, ahead};
}

// A chunk by a block: rounds of TURNS vectors a thread, vector(i, k) for all of them and then done(i, k), i the vector's first element; the
// rest vector by vector, and single(i) for what is no whole one.
template <int V, int TURNS, typename Vector, typename Done, typename Single>
__device__ __forceinline__ void for_chunk(const ClipRange& R, Vector vector, Done done, Single single) {
  constexpr int kRound = kThreads * V * TURNS;
  int64_t at = R.from + R.ahead < R.to ? R.from + R.ahead : R.to;
  if (static_cast<int>(threadIdx.x) < at - R.from) single(R.from + static_cast<int>(threadIdx.x));
  for (; at + kRound <= R.to; at += kRound) {
#pragma unroll
    for (int k = 0; k < TURNS; ++k) vector(at + (k * kThreads + static_cast<int>(threadIdx.x)) * V, k);
#pragma unroll
    for (int k = 0; k < TURNS; ++k) done(at + (k * kThreads + static_cast<int>(threadIdx.x)) * V, k);
  }
  for (; at < R.to; at += kThreads * V) {
    const int64_t i = at + static_cast<int>(threadIdx.x) * V;
    if (i + V <= R.to) {
      vector(i, 0);
      done(i, 0);
    } else {
      for (int64_t q = i; q < R.to; ++q) single(q);
    }
  }
}
constexpr int kClipTurns = 4;

// 400 M halfs in 290 tensors: 182 us, 4.4 TB/s.  Squares are added in 64 bits: those of floats from 1e19 on are beyond a float's range, and a sum over 10^9 elements keeps its digits.
template <typename T>
__device__ __forceinline__ double sum_of_squares(const T* src, uint32_t q, int64_t chunk, int64_t numel, int64_t n) {
  constexpr int V = 16 / sizeof(T);
  double s = 0.0;
  Elems<T, V> e[kClipTurns];
  const auto add = [&](T x) {
    const double d = as_float(x);
    s += d * d;
  };
  for_chunk<V, kClipTurns>(
      range_of(src, q, chunk, numel, n), [&](int64_t i, int k) { e[k] = *reinterpret_cast<const Elems<T, V>*>(src + i); },
      [&](int64_t, int k) {
#pragma unroll
        for (int j = 0; j < V; ++j) add(e[k].v[j]);
      },
      [&](int64_t i) { add(src[i]); });
  return s;
}

template <bool TABLE>
__global__ void __launch_bounds__(kThreads) k_clip_squares(ClipArgs A) {
  __shared__ double lds[kThreads / 64];
  const uint32_t block = A.first_block + blockIdx.x;
  const ClipTensor T = tensor_of_block<TABLE>(A, block);
  const int64_t n = elements_of(T);
  const uint32_t q = block - T.first_block;
  double s;
  switch (T.type & 15) {
    case SMFG_DTYPE_F32: s = sum_of_squares(static_cast<const float*>(T.src), q, A.chunk, T.numel, n); break;
    case SMFG_DTYPE_F16: s = sum_of_squares(static_cast<const _Float16*>(T.src), q, A.chunk, T.numel, n); break;
    default: s = sum_of_squares(static_cast<const __bf16*>(T.src), q, A.chunk, T.numel, n); break;
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) s += __shfl_xor(s, o, 64);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int w = 1; w < kThreads / 64; ++w) s += lds[w];
    A.part[block] = s;
  }
}

// The norm from the blocks' sums, by a block of THREADS; scale times the factor.
template <int THREADS>
__device__ __forceinline__ ClipFactor factor_of(const double* part, int64_t parts, float scale, float max_norm, double* lds, float& norm) {
  double s = 0.0;
#pragma unroll 8
  for (int64_t i = threadIdx.x; i < parts; i += THREADS) s += part[i];
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) s += __shfl_xor(s, o, 64);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
  __syncthreads();
  s = 0.0;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) s += lds[w];
  const double n = fabs(static_cast<double>(scale)) * sqrt(s), c = max_norm / (n + 1e-6);
  norm = static_cast<float>(n);
  const double f = scale * (c >= 1.0 || (__builtin_isinf(max_norm) && n == n) ? 1.0 : c);  // of a NaN among the gradients NaN
  if (!(fabs(f) < 0x1p-100) || f == 0.0) return {static_cast<float>(f), 0};
  int power;
  const double digits = frexp(f, &power);
  return {static_cast<float>(digits), power};
}

// Up to kClipJoin blocks every one of k_clip_scale adds up all sums itself; of more a launch of one block does (nine tensors of 281 K floats in all, 142
// blocks: two launches instead of three, 2 us less).
constexpr int64_t kClipJoin = 1024;
constexpr int kClipNormThreads = 1024;
static __global__ void __launch_bounds__(kClipNormThreads) k_clip_norm(ClipArgs A) {
  __shared__ double lds[kClipNormThreads / 64];
  float norm;
  const ClipFactor f = factor_of<kClipNormThreads>(A.part, A.blocks, A.scale, A.max_norm, lds, norm);
  if (threadIdx.x != 0) return;
  *A.norm = norm;
  *A.factor = f;
}

// Vectors of 16 bytes of the wider type, so that the lanes of an instruction read and write bytes without a gap.
// The power of a factor is looked at once a vector: with an instruction for every element 400 M halfs took 4 % more.
template <typename TD, typename TS, int V>
__device__ __forceinline__ Elems<TD, V> scaled(const Elems<TS, V>& x, const ClipFactor& f) {
  float y[V];
#pragma unroll
  for (int j = 0; j < V; ++j) y[j] = f.digits * as_float(x.v[j]);
  if (f.power != 0) {
#pragma unroll
    for (int j = 0; j < V; ++j) y[j] = __builtin_ldexpf(y[j], f.power);
  }
  Elems<TD, V> o;
#pragma unroll
  for (int j = 0; j < V; ++j) o.v[j] = from_float<TD>(y[j]);
  return o;
}
template <typename TS, typename TD>
__device__ __forceinline__ void scaled_copy(const TS* src, TD* dst, uint32_t q, int64_t chunk, int64_t numel, int64_t n, ClipFactor f) {
  constexpr int V = 16 / (sizeof(TS) > sizeof(TD) ? sizeof(TS) : sizeof(TD));
  Elems<TS, V> e[kClipTurns];
  for_chunk<V, kClipTurns>(
      range_of(dst, q, chunk, numel, n), [&](int64_t i, int k) { e[k] = *reinterpret_cast<const Elems<TS, V>*>(src + i); },
      [&](int64_t i, int k) { *reinterpret_cast<Elems<TD, V>*>(dst + i) = scaled<TD>(e[k], f); },
      [&](int64_t i) { dst[i] = scaled<TD>(Elems<TS, 1>{{src[i]}}, f).v[0]; });
}

// The last elements first: they are what the sum of squares has left in the caches (1 % of 670 us).  400 M halfs to floats 480 us, 5.0 TB/s.
template <bool TABLE>
__global__ void __launch_bounds__(kThreads) k_clip_scale(ClipArgs A) {
  const uint32_t block = A.blocks - 1 - (A.first_block + blockIdx.x);
  const ClipTensor T = tensor_of_block<TABLE>(A, block);
  ClipFactor f;
  if (A.blocks <= kClipJoin) {
    __shared__ double lds[kThreads / 64];
    float norm;
    f = factor_of<kThreads>(A.part, A.blocks, A.scale, A.max_norm, lds, norm);
    if (blockIdx.x == 0 && threadIdx.x == 0) *A.norm = norm;
  } else {
    f = *A.factor;
  }
  f.power = __builtin_amdgcn_readfirstlane(f.power);  // the same for all lanes
  if (f.digits == 1.f && f.power == 0 && T.src == T.dst) return;  // in place, nothing to clip
  const int64_t n = elements_of(T);
  const uint32_t q = block - T.first_block;
  constexpr int F32 = SMFG_DTYPE_F32, F16 = SMFG_DTYPE_F16, BF16 = SMFG_DTYPE_BF16;
  switch (T.type) {
    case F32 | F32 << 4: scaled_copy(static_cast<const float*>(T.src), static_cast<float*>(T.dst), q, A.chunk, T.numel, n, f); break;
    case F16 | F16 << 4: scaled_copy(static_cast<const _Float16*>(T.src), static_cast<_Float16*>(T.dst), q, A.chunk, T.numel, n, f); break;
    case F16 | F32 << 4: scaled_copy(static_cast<const _Float16*>(T.src), static_cast<float*>(T.dst), q, A.chunk, T.numel, n, f); break;
    case BF16 | BF16 << 4: scaled_copy(static_cast<const __bf16*>(T.src), static_cast<__bf16*>(T.dst), q, A.chunk, T.numel, n, f); break;
    default: scaled_copy(static_cast<const __bf16*>(T.src), static_cast<float*>(T.dst), q, A.chunk, T.numel, n, f); break;
  }
}

}  // namespace smfg_dev

#endif  // SMFG_KERNELS_CLIP_H_
