// libsmfg gradient clipping by the global norm over many tensors.
//
//   N = sqrt(sum over all elements of (scale g)^2),  c = min(1, max_norm / (N + 1e-6)),  out = scale c g
#ifndef SMFG_KERNELS_CLIP_H_
#define SMFG_KERNELS_CLIP_H_

#include "elements.h"

namespace smfg_dev {

// The tensors of a launch, in its arguments.  Block first_block + q of a tensor has its elements [q * chunk, (q + 1) * chunk).
// The table is indexed by a scalar register, and the compiler may split such an address between two of them; scalar loads drop
// the lowest two bits of each, so every index step has to be whole words (a table of bytes made pointers beside it garbage).
constexpr int kClipTensors = 84;
constexpr int64_t kClipLeast = 2048, kClipMost = 65536;  // elements of a block
struct ClipTensor {
  const void* src;
  void* dst;
  int64_t numel;
  const int64_t* rows;  // or null: the tensor counts up to *rows * row_elems elements
  int64_t row_elems;
  uint32_t first_block;
  int32_t type;         // of src | of dst << 4
};
struct ClipArgs {
  ClipTensor t[kClipTensors];
  int32_t tensors;
  uint32_t blocks;
  int64_t chunk;
  double* part;         // a block's sum of squares
  const float* factor;  // scale * c
};
static_assert(sizeof(ClipTensor) == 48 && sizeof(ClipArgs) <= 4096, "kernel arguments are limited to 4 KB");

__device__ __forceinline__ int tensor_of_block(const ClipArgs& A) {
  const int lane = threadIdx.x & 63;
  int t = -1;  // the last tensor that begins at this block or before
#pragma unroll
  for (int i = 0; i < kClipTensors; i += 64)
    t += __popcll(__ballot(i + lane < A.tensors && blockIdx.x >= A.t[i + lane < A.tensors ? i + lane : 0].first_block));
  return t;
}
__device__ __forceinline__ int64_t elements_of(const ClipTensor& T) {
  int64_t n = T.numel;
  if (T.rows) {
    const int64_t r = *T.rows, most = n / T.row_elems;
    n = (r < 0 ? 0 : r > most ? most : r) * T.row_elems;
  }
  return n;
}

// A chunk by a block: rounds of TURNS vectors a thread, vector(i, k) for all of them and then done(i, k), i the vector's first element; the
// rest vector by vector, and single(i) for what is no whole one.
template <int V, int TURNS, typename Vector, typename Done, typename Single>
__device__ __forceinline__ void for_chunk(int64_t from, int64_t to, Vector vector, Done done, Single single) {
  constexpr int kRound = kThreads * V * TURNS;
  int64_t at = from;
  for (; at + kRound <= to; at += kRound) {
#pragma unroll
    for (int k = 0; k < TURNS; ++k) vector(at + (k * kThreads + static_cast<int>(threadIdx.x)) * V, k);
#pragma unroll
    for (int k = 0; k < TURNS; ++k) done(at + (k * kThreads + static_cast<int>(threadIdx.x)) * V, k);
  }
  for (; at < to; at += kThreads * V) {
    const int64_t i = at + static_cast<int>(threadIdx.x) * V;
    if (i + V <= to) {
      vector(i, 0);
      done(i, 0);
    } else {
      for (int64_t q = i; q < to; ++q) single(q);
    }
  }
}
constexpr int kClipTurns = 4;

// Squares are added in 64 bits: those of floats from 1e19 on are beyond a float's range, and a sum over 10^9 elements keeps its digits.
template <typename T>
__device__ __forceinline__ double sum_of_squares(const T* src, int64_t from, int64_t to) {
  constexpr int V = 16 / sizeof(T);
  double s = 0.0;
  Elems<T, V> e[kClipTurns];
  const auto add = [&](T x) {
    const double d = as_float(x);
    s += d * d;
  };
  for_chunk<V, kClipTurns>(
      from, to, [&](int64_t i, int k) { e[k] = *reinterpret_cast<const Elems<T, V>*>(src + i); },
      [&](int64_t, int k) {
#pragma unroll
        for (int j = 0; j < V; ++j) add(e[k].v[j]);
      },
      [&](int64_t i) { add(src[i]); });
  return s;
}

static __global__ void __launch_bounds__(kThreads) k_clip_squares(ClipArgs A) {
  __shared__ double lds[kThreads / 64];
  const ClipTensor T = A.t[tensor_of_block(A)];
  const int64_t n = elements_of(T), from = static_cast<int64_t>(blockIdx.x - T.first_block) * A.chunk;
  const int64_t to = from + A.chunk < n ? from + A.chunk : n;
  double s;
  switch (T.type & 15) {
    case SMFG_DTYPE_F32: s = sum_of_squares(static_cast<const float*>(T.src), from, to); break;
    case SMFG_DTYPE_F16: s = sum_of_squares(static_cast<const _Float16*>(T.src), from, to); break;
    default: s = sum_of_squares(static_cast<const __bf16*>(T.src), from, to); break;
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) s += __shfl_xor(s, o, 64);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int w = 1; w < kThreads / 64; ++w) s += lds[w];
    A.part[blockIdx.x] = s;
  }
}

// The norm and the factor, by one block.
constexpr int kClipNormThreads = 1024;
static __global__ void __launch_bounds__(kClipNormThreads) k_clip_norm(const double* part, int64_t parts, float scale, float max_norm, float* norm,
                                                                float* factor) {
  __shared__ double lds[kClipNormThreads / 64];
  double s = 0.0;
#pragma unroll 8
  for (int64_t i = threadIdx.x; i < parts; i += kClipNormThreads) s += part[i];
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) s += __shfl_xor(s, o, 64);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x != 0) return;
#pragma unroll
  for (int w = 1; w < kClipNormThreads / 64; ++w) s += lds[w];
  const double n = fabs(static_cast<double>(scale)) * sqrt(s), c = max_norm / (n + 1e-6);
  *norm = static_cast<float>(n);
  *factor = static_cast<float>(scale * (__builtin_isinf(max_norm) || c >= 1.0 ? 1.0 : c));  // NaN stays NaN
}

// Vectors of 16 bytes of the wider type, so that the lanes of an instruction read and write bytes without a gap.
template <typename TS, typename TD>
__device__ __forceinline__ void scaled_copy(const TS* src, TD* dst, int64_t from, int64_t to, float f) {
  constexpr int V = 16 / (sizeof(TS) > sizeof(TD) ? sizeof(TS) : sizeof(TD));
  Elems<TS, V> e[kClipTurns];
  for_chunk<V, kClipTurns>(
      from, to, [&](int64_t i, int k) { e[k] = *reinterpret_cast<const Elems<TS, V>*>(src + i); },
      [&](int64_t i, int k) {
        Elems<TD, V> o;
#pragma unroll
        for (int j = 0; j < V; ++j) o.v[j] = from_float<TD>(f * as_float(e[k].v[j]));
        *reinterpret_cast<Elems<TD, V>*>(dst + i) = o;
      },
      [&](int64_t i) { dst[i] = from_float<TD>(f * as_float(src[i])); });
}

static __global__ void __launch_bounds__(kThreads) k_clip_scale(ClipArgs A) {
  const ClipTensor T = A.t[tensor_of_block(A)];
  const float f = *A.factor;
  if (f == 1.f && T.src == T.dst) return;  // in place, nothing to clip
  const int64_t n = elements_of(T), from = static_cast<int64_t>(blockIdx.x - T.first_block) * A.chunk;
  const int64_t to = from + A.chunk < n ? from + A.chunk : n;
  constexpr int F32 = SMFG_DTYPE_F32, F16 = SMFG_DTYPE_F16, BF16 = SMFG_DTYPE_BF16;
  switch (T.type) {
    case F32 | F32 << 4: scaled_copy(static_cast<const float*>(T.src), static_cast<float*>(T.dst), from, to, f); break;
    case F16 | F16 << 4: scaled_copy(static_cast<const _Float16*>(T.src), static_cast<_Float16*>(T.dst), from, to, f); break;
    case F16 | F32 << 4: scaled_copy(static_cast<const _Float16*>(T.src), static_cast<float*>(T.dst), from, to, f); break;
    case BF16 | BF16 << 4: scaled_copy(static_cast<const __bf16*>(T.src), static_cast<__bf16*>(T.dst), from, to, f); break;
    default: scaled_copy(static_cast<const __bf16*>(T.src), static_cast<float*>(T.dst), from, to, f); break;
  }
}

}  // namespace smfg_dev

#endif  // SMFG_KERNELS_CLIP_H_
