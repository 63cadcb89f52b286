// Host helpers shared by the entry points.
#ifndef SMFG_HOST_COMMON_H_
#define SMFG_HOST_COMMON_H_

#include <hip/hip_runtime.h>

#include <cstdint>

#include "smfg.h"

namespace {

inline int hip_err(hipError_t e) { return e == hipSuccess ? SMFG_OK : SMFG_ERR_HIP_BASE - static_cast<int>(e); }

// Typed device pointers must be multiples of their element size (atomics and vector accesses on a
// misaligned address are undefined).
inline bool misaligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

inline unsigned blocks_for(int64_t work_items, int64_t per_block, unsigned cap) {
  int64_t b = (work_items + per_block - 1) / per_block;
  if (b < 1) b = 1;
  if (b > cap) b = cap;
  return static_cast<unsigned>(b);
}

}  // namespace

#endif  // SMFG_HOST_COMMON_H_
