// Host helpers of the training operators: checks of arguments, element types, launches, the shapes of rows that lie in registers.
#ifndef SMFG_TRAIN_COMMON_H_
#define SMFG_TRAIN_COMMON_H_

#include <hip/hip_runtime.h>

#include <cstdint>

#include "smfg.h"

#include "host_common.h"

namespace {

constexpr int64_t kMaxRows = int64_t(1) << 31;

inline int64_t type_bytes(int32_t t) { return t == SMFG_DTYPE_F32 ? 4 : t == SMFG_DTYPE_F16 || t == SMFG_DTYPE_BF16 ? 2 : 0; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int64_t up256(int64_t a) { return (a + 255) & ~int64_t(255); }

// A matrix argument: type, stride, alignment.
inline bool bad_matrix(const void* p, int32_t type, int64_t stride, int64_t dim) {
  return type_bytes(type) == 0 || stride < dim || stride >= (int64_t(1) << 40) || misaligned(p, static_cast<uintptr_t>(type_bytes(type)));
}
inline bool bad_dim(int32_t dim) { return dim < 1 || dim > SMFG_MAX_DIM; }

// Calls f(T{}) with the element type.
template <typename F>
void with_type(int32_t type, F f) {
  if (type == SMFG_DTYPE_F32) f(float{});
  else if (type == SMFG_DTYPE_F16) f(_Float16{});
  else f(__bf16{});
}
// The launches of a call, one behind the other.  Behind one that failed there are no more: they would work on scratch that it should have
// written, places of the output among it.
class Launches {
  static constexpr int64_t kLaunchItems = int64_t(1) << 31;
  template <typename T>
  struct Just {
    using type = T;
  };

 public:
  explicit Launches(void* stream) : stream_(static_cast<hipStream_t>(stream)) {}
  template <typename... P>
  void operator()(void (*kernel)(P...), dim3 blocks, int threads, const typename Just<P>::type&... args) {
    if (error_ != hipSuccess) return;
    void* list[] = {const_cast<void*>(static_cast<const void*>(&args))...};
    error_ = hipLaunchKernel(reinterpret_cast<const void*>(kernel), blocks, dim3(static_cast<unsigned>(threads)), list, 0, stream_);
  }
  // One block after the other of a number that a launch may not hold, as it has fewer than 2^32 work items: as many launches as it takes, each
  // of which finds its first block in the arguments.
  template <typename A>
  void all(void (*kernel)(A), int64_t blocks, int threads, A args) {
    const int64_t most = kLaunchItems / threads;
    for (int64_t first = 0; first < blocks; first += most) {
      args.first_block = static_cast<uint32_t>(first);
      (*this)(kernel, static_cast<unsigned>(blocks - first < most ? blocks - first : most), threads, args);
    }
  }
  int result() const {
    if (error_ != hipSuccess) (void)hipGetLastError();  // told here, and not once more by who asks next
    return hip_err(error_);
  }

 private:
  hipStream_t stream_;
  hipError_t error_ = hipSuccess;
};

template <typename T>
constexpr int kVec = 16 / static_cast<int>(sizeof(T));  // columns of a 16-byte vector

// What the next operator reads stays in the caches if it is no more than this, twice the 256 MB that the memory side's has; more of it goes past them.  Measured with a product of
// it behind the operator: gradients of 30 K rows of 4096 logits, 246 MB, 186 us kept and 194 past the caches; 40 K rows 246 and 256; 8192 rows of 50 K, 819 MB,
// 615 and 590.  Parameters: 50 M floats and their half copies, 300 MB, 255 us kept and 271 past; 400 M with copies, the step alone, 1985 and 1832.  It goes by the
// size of the arrays, as how many of their rows are in use is not known on the host.  The norm's outputs always stay.
constexpr double kKeptBytes = 512.0 * (1 << 20);

// ---- rows in registers --------------------------------------------------------------------------

// How rows of `vectors` vectors are dealt: LANES lanes and NV vectors a lane; f.template operator()<V, NV, LANES>.
// most: the largest LANES * NV that the registers hold.  As few lanes as have a row in one vector each, so that a wave has up to 16 rows (200 K rows of
// 32 halfs 9.5 us, their gradient 14.6; with 16 lanes for each 16.8 and 21.4), 64 up to two vectors, then a block: a wave of four would hold twice the registers.
template <typename T, int most, typename F>
bool with_row_shape(int32_t dim, F f) {
  constexpr int V = kVec<T>;
  if (dim < V) return f.template operator()<1, 1, 16>(), true;
  const int64_t vectors = ceil_div(dim, V);
  if (vectors <= 4) f.template operator()<V, 1, 4>();
  else if (vectors <= 8) f.template operator()<V, 1, 8>();
  else if (vectors <= 16) f.template operator()<V, 1, 16>();
  else if (vectors <= 32) f.template operator()<V, 1, 32>();
  else if (vectors <= 64) f.template operator()<V, 1, 64>();
  else if (vectors <= 128) f.template operator()<V, 2, 64>();
  else if (vectors <= 256) f.template operator()<V, 1, 256>();
  else if (vectors <= 512) f.template operator()<V, 2, 256>();
  else if (vectors <= 768) f.template operator()<V, 3, 256>();
  else if (vectors <= 1024) f.template operator()<V, 2, 512>();
  else if (vectors <= 1536) f.template operator()<V, 3, 512>();
  else if (most >= 2048 && vectors <= 2048) f.template operator()<V, most >= 2048 ? 4 : 3, 512>();
  else return false;
  return true;
}

// Slices of the weight's gradient.  Rows in registers: the blocks of the launch, 16 MiB of sums, but 256 to 1024 (16 K rows of 4096 in 128 blocks
// 169 us, 256 131, 512 with the next row on its way 80).  Longer rows: 64 at most, as the columns alone are many threads.
constexpr int kNormSlices = 1024, kNormLongSlices = 64, kNormLongDim = 16384;
inline int64_t norm_slices(int64_t max_rows, int32_t dim) {
  int64_t s = (int64_t(16) << 20) / (8 * static_cast<int64_t>(dim));
  const int64_t least = dim <= kNormLongDim ? 256 : 1, most = dim <= kNormLongDim ? kNormSlices : kNormLongSlices;
  if (s < least) s = least;
  if (s > most) s = most;
  return s < max_rows ? s : max_rows;
}

}  // namespace

#endif  // SMFG_TRAIN_COMMON_H_
