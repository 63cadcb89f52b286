// libsmfg: softmax cross entropy and its gradient (include/smfg.h), host side.  Kernels: kernels_loss.h.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "smfg.h"

#include "kernels_loss.h"
#include "train_common.h"

namespace {

using namespace smfg_dev;

constexpr unsigned kLossBlocks = 2048, kWideLossBlocks = 512, kLongLossBlocks = 256;  // at most
constexpr int64_t kCounts = 512;

// The blocks' sums, then the counts of labels.
struct LossScratch {
  int64_t counts, count_rows, bytes;
};
LossScratch loss_scratch(int64_t max_rows) {
  LossScratch S;
  S.counts = up256(kLossBlocks * static_cast<int64_t>(sizeof(LossPart)));
  S.count_rows = up256(ceil_div(max_rows, kCounts));
  if (S.count_rows < 1024) S.count_rows = 1024;
  S.bytes = S.counts + up256(8 * kCounts);
  return S;
}

template <typename T>
struct LaunchLoss {
  LossArgs& A;
  Launches& go;
  template <int V, int NV, int LANES>
  void operator()() const {
    constexpr int threads = loss_threads(LANES);
    constexpr int rows = threads / LANES;  // of a block
    // Up to four turns of a block take less than the launch that joins several: 30 rows of 172 halfs 9.6 -> 6.9 us.  Rows of more than a wave have one (two of 50 K
    // 14.5 instead of 12.1).
    A.parts = A.max_rows <= (LANES <= 64 ? 4 : 1) * rows ? 1 : static_cast<int32_t>(blocks_for(A.max_rows, rows, LANES == 1024 ? kWideLossBlocks : kLossBlocks));
    go(k_cross_entropy<T, V, NV, LANES>, static_cast<unsigned>(A.parts), threads, A);
  }
};

// How rows of `vectors` vectors are dealt.  Where a row is a wave's or less, up to four vectors a lane, as what a row takes besides its elements is shared by the rows
// of a wave then, and no barrier is met (100 K rows of 512 halfs 41 us, with a vector a lane 51; 50 K of 700 floats 55, in blocks of 256 lanes 73); up to 16 vectors one a lane, whose
// loads are next to each other (190 K rows of 47 floats 20.6, four lanes 41).
template <typename T>
bool launch_loss(LossArgs& A, Launches& go) {
  constexpr int V = kVec<T>;
  const LaunchLoss<T> f{A, go};
  const int64_t vectors = ceil_div(A.classes, V);
  if (A.classes < V) f.template operator()<1, 1, V>();
  else if (vectors <= 2) f.template operator()<V, 1, 2>();
  else if (vectors <= 4) f.template operator()<V, 1, 4>();
  else if (vectors <= 8) f.template operator()<V, 1, 8>();
  else if (vectors <= 16) f.template operator()<V, 1, 16>();
  else if (vectors <= 32) f.template operator()<V, 1, 32>();
  else if (vectors <= 48) f.template operator()<V, 3, 16>();
  else if (vectors <= 64) f.template operator()<V, 4, 16>();
  else if (vectors <= 96) f.template operator()<V, 3, 32>();
  else if (vectors <= 128) f.template operator()<V, 4, 32>();
  else if (vectors <= 192) f.template operator()<V, 3, 64>();
  else if (vectors <= 256) f.template operator()<V, 4, 64>();
  else if (vectors <= 512) f.template operator()<V, 2, 256>();
  else if (vectors <= 768) f.template operator()<V, 3, 256>();
  else if (vectors <= 1024) f.template operator()<V, 2, 512>();
  else if (vectors <= 1536) f.template operator()<V, 3, 512>();
  else {
    switch (ceil_div(vectors, 1024)) {  // a block of the largest size: as few vectors a lane as hold the row
      case 2: f.template operator()<V, 2, 1024>(); break;
      case 3: f.template operator()<V, 3, 1024>(); break;
      case 4: f.template operator()<V, 4, 1024>(); break;
      case 5: f.template operator()<V, 5, 1024>(); break;
      case 6: f.template operator()<V, 6, 1024>(); break;
      case 7: f.template operator()<V, 7, 1024>(); break;
      default: return false;
    }
  }
  return true;
}

}  // namespace

extern "C" {

int64_t smfg_cross_entropy_scratch_bytes(int64_t max_rows, int32_t classes) {
  if (bad_dim(classes) || max_rows < 0 || max_rows >= kMaxRows) return -1;
  return loss_scratch(max_rows).bytes;
}

int smfg_cross_entropy(const void* d_logits, int64_t logits_stride, int32_t dtype, const void* d_labels, int32_t label_bytes, const int64_t* d_num_rows,
                       int64_t max_rows, int32_t classes, int32_t reduction, float scale, float* d_loss, float* d_row_loss, void* d_dlogits,
                       int64_t dlogits_stride, void* d_scratch, int64_t scratch_bytes, void* hip_stream) {
  if (!d_num_rows || !d_loss || !d_scratch || (max_rows > 0 && (!d_logits || !d_labels))) return SMFG_ERR_NULL_PTR;
  if (bad_dim(classes) || max_rows < 0 || max_rows >= kMaxRows || bad_matrix(d_logits, dtype, logits_stride, classes) ||
      (label_bytes != 4 && label_bytes != 8) || misaligned(d_labels, static_cast<uintptr_t>(label_bytes)) ||
      (reduction != SMFG_LOSS_MEAN && reduction != SMFG_LOSS_SUM) || !std::isfinite(scale) || misaligned(d_num_rows, 8) || misaligned(d_loss, 4) ||
      misaligned(d_row_loss, 4) || misaligned(d_scratch, 256) ||
      (d_dlogits && (bad_matrix(d_dlogits, dtype, dlogits_stride, classes) || (d_dlogits == d_logits && dlogits_stride != logits_stride))))
    return SMFG_ERR_INVALID_ARG;
  const LossScratch S = loss_scratch(max_rows);
  if (scratch_bytes < S.bytes) return SMFG_ERR_CAPACITY;
  Launches go(hip_stream);
  uint8_t* scratch = static_cast<uint8_t*>(d_scratch);
  LossArgs A = {d_logits, logits_stride, d_labels, label_bytes, classes, d_num_rows, max_rows, reduction == SMFG_LOSS_MEAN, scale, d_dlogits, dlogits_stride,
                d_row_loss, d_loss, reinterpret_cast<LossPart*>(scratch), 0, reinterpret_cast<int64_t*>(scratch + S.counts), 0, S.count_rows,
                static_cast<double>(max_rows) * classes * static_cast<double>(type_bytes(dtype)) <= kKeptBytes};
  if (max_rows > 0) {
    if (A.mean && d_dlogits && max_rows > kCountAll) {
      A.num_counts = static_cast<int32_t>(ceil_div(max_rows, S.count_rows));
      go(k_loss_count, static_cast<unsigned>(A.num_counts), kThreads, A);
    }
    with_type(dtype, [&](auto t) {
      using T = decltype(t);
      if (launch_loss<T>(A, go)) return;
      A.parts = static_cast<int32_t>(blocks_for(max_rows, 1, kLongLossBlocks));
      go(k_cross_entropy_long<T, kVec<T>>, static_cast<unsigned>(A.parts), kLongLossThreads, A);
    });
  }
  if (A.parts != 1) go(k_loss_join, 1, kLossJoinThreads, A);
  return go.result();
}

}  // extern "C"
