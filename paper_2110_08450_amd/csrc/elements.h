// Element types of the training operators: vectors of them at any element address, conversion to and from float.
#ifndef SMFG_ELEMENTS_H_
#define SMFG_ELEMENTS_H_

#include "device_common.h"

namespace smfg_dev {

// V consecutive elements at a multiple of the element's size; the target reads and writes vectors at any address.
template <typename T, int V>
struct alignas(sizeof(T)) Elems {
  T v[V];
};

// Sums and products run in float; a result is rounded to its type once, to nearest even.
template <typename T>
__device__ __forceinline__ float as_float(T x) {
  return static_cast<float>(x);
}
// For half the value is kept apart from the product it comes from: the compiler merges the two into v_fma_mixlo_f16, which
// rounded two of 38 400 products to the wrong side (of a tie in float, or just beside one).
template <typename T>
__device__ __forceinline__ T from_float(float x) {
  if constexpr (__is_same(T, _Float16)) asm("" : "+v"(x));
  return static_cast<T>(x);
}

// V values, the first `dup` of which are left alone.  Without the asm the compiler joins the last of the single stores with the vector's, which becomes three
// stores then (400 M values of two bytes 315 us instead of 205).
template <typename T, int V>
__device__ __forceinline__ void store_own(T* dst, const Elems<T, V>& e, int dup) {
  if (dup == 0) {
    *reinterpret_cast<Elems<T, V>*>(dst) = e;
  } else if (dup < V) {
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (j >= dup) dst[j] = e.v[j];
    asm volatile("" ::: "memory");
  }
}

// A count that lives on the device, within what the launch was sized for.
__device__ __forceinline__ int64_t count_of(const int64_t* num, int64_t max) {
  const int64_t n = *num;
  return n < 0 ? 0 : n > max ? max : n;
}

// The vector of V columns that a lane has of a row of dim (>= V) columns, by the vector's index: it begins at column
// index * V, or ends with the row, its first `dup` columns those of the vector before.  dup == V: there is none, and `start` is the
// last vector's, so that a load needs no condition.
template <int V>
struct Columns {
  int start, dup;
  __device__ __forceinline__ Columns(int index, int dim) {
    const int c = index * V;
    start = c + V <= dim ? c : dim - V;
    dup = c >= dim ? V : c - start;
  }
};

// V parameters from column c on, of float or of T; all of them `none` without an array.
template <typename T, int V>
__device__ __forceinline__ void load_params(const void* p, bool is_float, int c, float none, float (&out)[V]) {
  if (!p) {
#pragma unroll
    for (int j = 0; j < V; ++j) out[j] = none;
  } else if (is_float) {
    const Elems<float, V> x = *reinterpret_cast<const Elems<float, V>*>(static_cast<const float*>(p) + c);
#pragma unroll
    for (int j = 0; j < V; ++j) out[j] = x.v[j];
  } else {
    const Elems<T, V> x = *reinterpret_cast<const Elems<T, V>*>(static_cast<const T*>(p) + c);
#pragma unroll
    for (int j = 0; j < V; ++j) out[j] = as_float(x.v[j]);
  }
}

// Sum over groups of LANES lanes, in every lane; LANES of a whole block go through `lds`, a number per wave.  Between two sums through the
// same array has to be one through another: its barrier tells that the first has been read.
template <int LANES, typename S>
__device__ __forceinline__ S group_sum(S x, S* lds) {
#pragma unroll
  for (int o = 1; o < (LANES < 64 ? LANES : 64); o <<= 1) x += __shfl_xor(x, o, 64);
  if constexpr (LANES > 64) {
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    x = 0;
#pragma unroll
    for (int w = 0; w < LANES / 64; ++w) x += lds[w];
  }
  return x;
}

}  // namespace smfg_dev

#endif  // SMFG_ELEMENTS_H_
