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

// V values at any element's address that are not read or written again soon: they leave the caches to others.
template <typename T, int V>
using Raw = T __attribute__((ext_vector_type(V), aligned(sizeof(T))));
template <typename T, int V>
__device__ __forceinline__ Elems<T, V> load_once(const T* src) {
  if constexpr (V == 1) {
    return *reinterpret_cast<const Elems<T, V>*>(src);
  } else {
    using Vector = Elems<T, V>;
    return __builtin_bit_cast(Vector, __builtin_nontemporal_load(reinterpret_cast<const Raw<T, V>*>(src)));
  }
}
template <typename T, int V>
__device__ __forceinline__ void store_once(T* dst, const Elems<T, V>& e, int dup) {
  if (V > 1 && dup == 0) {
    if constexpr (V > 1) __builtin_nontemporal_store(__builtin_bit_cast(Raw<T, V>, e), reinterpret_cast<Raw<T, V>*>(dst));
  } else {
    store_own(dst, e, dup);
  }
}

// V elements in as few registers as hold them, for what is kept from a load to its use: as elements of their own the compiler gives each a register.
template <typename T, int V>
struct Words {
  static constexpr int kWords = (V * static_cast<int>(sizeof(T)) + 3) / 4;
  uint32_t w[kWords];
  __device__ __forceinline__ float operator[](int j) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[j]);
    else return as_float(__builtin_bit_cast(T, static_cast<uint16_t>(w[j / 2] >> 16 * (j % 2))));
  }
};
template <typename T, int V, bool ONCE>
__device__ __forceinline__ Words<T, V> load_words(const T* src) {
  using Out = Words<T, V>;
  if constexpr (V == 1 && sizeof(T) == 2) {
    return {{__builtin_bit_cast(uint16_t, *src)}};
  } else if constexpr (V == 1) {
    return {{__builtin_bit_cast(uint32_t, *src)}};
  } else {
    using Raw32 = uint32_t __attribute__((ext_vector_type(Out::kWords), aligned(sizeof(T)), may_alias));
    const Raw32* p = reinterpret_cast<const Raw32*>(src);
    Out o;
    Raw32 x;
    if constexpr (ONCE) x = __builtin_nontemporal_load(p);
    else x = *p;
#pragma unroll
    for (int i = 0; i < Out::kWords; ++i) o.w[i] = x[i];
    return o;
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
  __device__ __forceinline__ Columns(int whole) : start(whole), dup(0) {}
};
// Vector k of a lane's NV in a row that LANES lanes have; the row has more than (NV - 1) * LANES vectors, so that all but the last are whole.
template <int V, int NV, int LANES>
__device__ __forceinline__ Columns<V> columns_of(int k, int lane, int dim) {
  return k < NV - 1 ? Columns<V>((k * LANES + lane) * V) : Columns<V>(k * LANES + lane, dim);
}

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

// What `op` makes of the values of groups of LANES lanes of a wave, in each of them: by moves between registers, which need no memory's pipeline as shuffles do.  In
// every step the lanes that are joined hold the same, so that all lanes get the same bits.
template <int CONTROL>
__device__ __forceinline__ uint32_t moved(uint32_t x) {
  return static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(x), CONTROL, 15, 15, true));
}
template <int LANES, typename T, typename Op>
__device__ __forceinline__ T lanes_all(T x, Op op) {
  static_assert(sizeof(T) == 4, "a register");
  const auto bits = [](T y) { return __builtin_bit_cast(uint32_t, y); };
  const auto value = [](uint32_t y) { return __builtin_bit_cast(T, y); };
  if constexpr (LANES > 1) x = op(x, value(moved<0xb1>(bits(x))));   // the neighbour
  if constexpr (LANES > 2) x = op(x, value(moved<0x4e>(bits(x))));   // the other pair of four
  if constexpr (LANES > 4) x = op(x, value(moved<0x141>(bits(x))));  // the other four of eight, mirrored
  if constexpr (LANES > 8) x = op(x, value(moved<0x140>(bits(x))));  // the other eight of sixteen, mirrored
  if constexpr (LANES > 16) {
    const auto rows = __builtin_amdgcn_permlane16_swap(bits(x), bits(x), false, false);
    x = op(value(rows[0]), value(rows[1]));
  }
  if constexpr (LANES > 32) {
    const auto halves = __builtin_amdgcn_permlane32_swap(bits(x), bits(x), false, false);
    x = op(value(halves[0]), value(halves[1]));
  }
  return x;
}
__device__ __forceinline__ float sum_f(float a, float b) { return a + b; }
__device__ __forceinline__ float max_f(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ uint32_t max_u(uint32_t a, uint32_t b) { return a > b ? a : b; }

// group_sum by them.
template <int LANES>
__device__ __forceinline__ float row_sum(float x, float* lds) {
  x = lanes_all<(LANES < 64 ? LANES : 64)>(x, sum_f);
  if constexpr (LANES > 64) {
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    x = 0.f;
#pragma unroll
    for (int w = 0; w < LANES / 64; ++w) x += lds[w];
  }
  return x;
}

}  // namespace smfg_dev

#endif  // SMFG_ELEMENTS_H_
