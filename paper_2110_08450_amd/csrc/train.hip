// libsmfg: operators of a training step (include/smfg.h), host side.  Kernels: kernels_embed.h, kernels_norm.h,
// kernels_clip.h.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "smfg.h"

#include "elements.h"
#include "host_common.h"
#include "kernels_clip.h"
#include "kernels_embed.h"
#include "kernels_norm.h"

namespace {

using namespace smfg_dev;

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

// ---- embedding ----------------------------------------------------------------------------------

template <typename TI, typename TO>
void launch_embedding(const EmbedArgs& A, int64_t blocks, bool vectors, Launches& go) {
  if (vectors) go.all(k_embedding<TI, TO, kVec<TO>>, blocks, kThreads, A);
  else go.all(k_embedding<TI, TO, 1>, blocks, kThreads, A);
}

// Blocks of k_embed_sums for the tokens, tiles of 64 * V columns, and floats of a row of partial sums.
struct GradShape {
  int64_t blocks, tiles, width;
};
GradShape grad_shape(int64_t max_ids, int32_t dim) {
  const int V = grad_columns(dim);
  const int64_t vectors = ceil_div(dim, V);
  return {ceil_div(max_ids, kBlockTokens), ceil_div(vectors, 64), vectors * V};
}

// Blocks have numbers of 32 bits: fewer than 2^31 that add up (as many are for 2^45 values), and those that clear, at most num_rows, behind them.
bool too_many_blocks(int64_t max_ids, int32_t dim) {
  const GradShape G = grad_shape(max_ids, dim);
  return G.blocks * G.tiles >= kMaxRows;
}

struct EmbedScratch {
  int64_t rec[2], hist, starts, totals, part, tile_runs, block_runs, tail_rank, bytes;
  int64_t tiles, run_tiles;
  int turns;
};
EmbedScratch embed_scratch(int64_t max_ids, int32_t dim) {
  EmbedScratch S;
  S.turns = max_ids <= 2 * kSortThreads * kSortColumns ? 2 : 4;
  S.tiles = ceil_div(max_ids, S.turns * kSortThreads);
  S.run_tiles = ceil_div(max_ids, kRunTile);
  const GradShape G = grad_shape(max_ids, dim);
  int64_t at = 0;
  const auto take = [&at](int64_t bytes) {
    const int64_t here = at;
    at += up256(bytes);
    return here;
  };
  S.rec[0] = take(8 * max_ids);
  S.rec[1] = take(8 * max_ids);
  // as much for many ids as for the most that have smaller tiles: scratch for max_ids has room for calls of fewer
  const int64_t small_tiles = ceil_div(max_ids, 2 * kSortThreads);
  S.hist = take(max_ids > kSmallSort ? 2 * kSortBins * (S.turns == 2 || S.tiles > kSortColumns ? S.tiles : small_tiles < kSortColumns ? small_tiles : kSortColumns) : 0);
  S.starts = take(S.tiles > kSortColumns ? 4 * kSortBins * S.tiles : 0);
  S.totals = take(4 * kSortBins);
  S.part = take(4 * 2 * G.blocks * G.width);
  S.tile_runs = take(4 * S.run_tiles);
  S.block_runs = take(4 * G.blocks);
  S.tail_rank = take(4 * G.blocks);
  S.bytes = at;
  return S;
}

// A matrix to be cleared beside the sort, base null: none.
struct Clear {
  void* base;
  int64_t rows, dim, stride, elem_bytes;
};

// Blocks of a launch of the sort, with those that clear its share (part of parts) of the matrix: about 64 KiB each.
unsigned sort_blocks(SortArgs& A, int64_t own, const Clear& c, int part, int parts) {
  A.own_blocks = static_cast<uint32_t>(own);
  A.clear = nullptr;
  if (!c.base) return A.own_blocks;
  const int64_t units = c.elem_bytes / 2, from = c.rows * part / parts, to = c.rows * (part + 1) / parts;
  A.clear = static_cast<uint16_t*>(c.base) + from * c.stride * units;
  A.clear_rows = to - from;
  A.clear_width = c.dim * units;
  A.clear_stride = c.stride * units;
  if (to == from) return A.own_blocks;
  return A.own_blocks + blocks_for(A.clear_rows * A.clear_width, 32 << 10, 1u << 20);
}

// (row, token) of the call's ids, sorted by row.  num_rows itself, which stands for no row, is a key as well.
const uint2* launch_sort(const EmbedScratch& S, uint8_t* scratch, const void* ids, int32_t id_bytes, const int64_t* num, int64_t max_ids,
                         int64_t num_rows, const Clear& clear, Launches& go) {
  SortArgs A = {};
  A.ids = ids;
  A.id_bytes = id_bytes;
  A.num_rows = num_rows;
  A.num = num;
  A.max_ids = max_ids;
  A.hist = reinterpret_cast<uint16_t*>(scratch + S.hist);
  A.tiles = static_cast<int32_t>(S.tiles);
  if (S.tiles > kSortColumns) A.starts = reinterpret_cast<uint32_t*>(scratch + S.starts);
  A.totals = reinterpret_cast<uint32_t*>(scratch + S.totals);
  A.out = reinterpret_cast<uint2*>(scratch + S.rec[0]);
  if (max_ids <= kSmallSort) {
    const unsigned blocks = sort_blocks(A, ceil_div(max_ids, kSmallTokens), clear, 0, 1);
    go(k_sort_small, blocks, kSmallThreads, A);
    return A.out;
  }
  int key_bits = 0;
  while (num_rows >> key_bits != 0) ++key_bits;
  const int passes = (key_bits + kSortBits - 1) / kSortBits;
  A.bits = (key_bits + passes - 1) / passes;
  for (int p = 0; p < passes; ++p, A.shift += A.bits) {
    A.out = reinterpret_cast<uint2*>(scratch + S.rec[p & 1]);
    unsigned blocks = sort_blocks(A, S.tiles, clear, 2 * p, 2 * passes);
    if (S.turns == 2) go(k_sort_count<2>, blocks, kSortThreads, A);
    else go(k_sort_count<4>, blocks, kSortThreads, A);
    if (A.starts) go(k_sort_scan, static_cast<unsigned>(ceil_div(1 << A.bits, 2 * kScanPairs)), kSortThreads, A);
    blocks = sort_blocks(A, S.tiles, clear, 2 * p + 1, 2 * passes);
    if (S.turns == 2) go(k_sort_scatter<2>, blocks, kSortThreads, A);
    else go(k_sort_scatter<4>, blocks, kSortThreads, A);
    A.in = A.out;
  }
  return A.in;
}

template <typename TD, typename TG, int V>
void launch_embed_sums(EmbedGradArgs A, const GradShape& G, bool clear, Launches& go) {
  A.sum_blocks = G.blocks > 0 ? static_cast<uint32_t>(G.blocks) : 1u;  // without tokens there is one, which has no tile
  A.tiles = G.blocks > 0 ? static_cast<uint32_t>(G.tiles) : 0u;
  // a block clears about 32 KiB, of at most a row a thread
  const int64_t rows = (32 << 10) / (A.dim * static_cast<int64_t>(sizeof(TG)));
  A.clear_rows = static_cast<int32_t>(rows < 1 ? 1 : rows > kGradThreads ? kGradThreads : rows);
  const bool tiny = A.max_ids <= kTinyIds;
  if (tiny) A.sum_blocks = 1;
  const int64_t blocks = static_cast<int64_t>(A.sum_blocks) * A.tiles + (clear ? ceil_div(A.num_rows, A.clear_rows) : 0);
  if (blocks == 0) return;
  if (tiny) {
    if (A.accumulate) go.all(k_embed_sums<TD, TG, V, true, true>, blocks, kTinyThreads, A);
    else go.all(k_embed_sums<TD, TG, V, true, false>, blocks, kTinyThreads, A);
    return;
  }
  if (A.accumulate) go.all(k_embed_sums<TD, TG, V, false, true>, blocks, kGradThreads, A);
  else go.all(k_embed_sums<TD, TG, V, false, false>, blocks, kGradThreads, A);
  if (G.blocks < 2) return;
  const uint32_t joins = static_cast<uint32_t>(ceil_div(G.blocks, kJoinWaves));
  const unsigned longs = static_cast<unsigned>((G.blocks - 1) / kJoinShort);
  go(k_embed_join<TG, V>, dim3(joins + longs, static_cast<unsigned>(G.tiles)), kJoinThreads, A, joins);
}

template <typename TD, typename TG>
void launch_embed_grad(const EmbedGradArgs& A, const GradShape& G, bool clear, Launches& go) {
  const int V = grad_columns(A.dim);
  if (V == 1) launch_embed_sums<TD, TG, 1>(A, G, clear, go);
  else if (V == 2) launch_embed_sums<TD, TG, 2>(A, G, clear, go);
  else launch_embed_sums<TD, TG, 4>(A, G, clear, go);
}

// Is the whole gradient cleared beside the sort, and the touched rows written over?  Else only the untouched ones are, beside the sums.  At most half
// of the rows are written twice.
bool early_clear(int64_t max_ids, int64_t num_rows) { return num_rows >= 2 * max_ids; }

int embedding_grad(const void* d_ids, int32_t id_bytes, const int64_t* d_num_ids, int64_t max_ids, const void* d_dy, int64_t dy_stride,
                   int32_t dy_dtype, int32_t dim, float scale, void* d_grad, int64_t num_rows, int64_t grad_stride, int32_t grad_dtype,
                   int32_t accumulate, bool rows_only, int32_t* d_row_ids, int64_t* d_num_unique, void* d_scratch, int64_t scratch_bytes,
                   void* hip_stream) {
  if (!d_num_ids || !d_grad || (max_ids > 0 && (!d_ids || !d_dy || !d_scratch))) return SMFG_ERR_NULL_PTR;
  if (rows_only && (!d_num_unique || (max_ids > 0 && !d_row_ids))) return SMFG_ERR_NULL_PTR;
  if (bad_dim(dim) || (id_bytes != 4 && id_bytes != 8) || max_ids < 0 || max_ids >= kMaxRows || num_rows < 1 || num_rows >= kMaxRows ||
      bad_matrix(d_dy, dy_dtype, dy_stride, dim) || bad_matrix(d_grad, grad_dtype, grad_stride, dim) ||
      (grad_dtype != SMFG_DTYPE_F32 && grad_dtype != dy_dtype) || misaligned(d_ids, static_cast<uintptr_t>(id_bytes)) ||
      misaligned(d_num_ids, 8) || misaligned(d_row_ids, 4) || misaligned(d_num_unique, 8) || misaligned(d_scratch, 256))
    return SMFG_ERR_INVALID_ARG;
  if (too_many_blocks(max_ids, dim)) return SMFG_ERR_INVALID_ARG;
  if (max_ids == 0 && !rows_only && accumulate) return SMFG_OK;
  Launches go(hip_stream);
  const EmbedScratch S = embed_scratch(max_ids, dim);
  if (max_ids > 0 && scratch_bytes < S.bytes) return SMFG_ERR_CAPACITY;
  const GradShape G = grad_shape(max_ids, dim);
  uint8_t* scratch = static_cast<uint8_t*>(d_scratch);
  EmbedGradArgs A = {};
  A.num = d_num_ids;
  A.max_ids = max_ids;
  A.num_rows = num_rows;
  A.dim = dim;
  A.accumulate = accumulate;
  A.dy = d_dy;
  A.dy_stride = dy_stride;
  A.scale = scale;
  A.grad = d_grad;
  A.grad_stride = grad_stride;
  A.part = reinterpret_cast<float*>(scratch + S.part);
  A.part_width = G.width;
  A.row_ids = d_row_ids;
  A.num_unique = d_num_unique;
  A.tile_runs = reinterpret_cast<uint32_t*>(scratch + S.tile_runs);
  A.block_runs = reinterpret_cast<uint32_t*>(scratch + S.block_runs);
  A.tail_rank = reinterpret_cast<uint32_t*>(scratch + S.tail_rank);
  A.run_tiles = S.run_tiles;
  A.ids = d_ids;
  A.id_bytes = id_bytes;
  const bool tiny = max_ids <= kTinyIds;
  bool clear = !rows_only && !accumulate;
  if (!tiny) {
    const bool early = clear && early_clear(max_ids, num_rows);
    const Clear c = {early ? d_grad : nullptr, num_rows, dim, grad_stride, type_bytes(grad_dtype)};
    A.sorted = launch_sort(S, scratch, d_ids, id_bytes, d_num_ids, max_ids, num_rows, c, go);
    clear = clear && !early;
  }
  A.direct = max_ids <= kDirectRuns;
  if (rows_only && (max_ids == 0 || !A.direct)) {
    if (max_ids > 0) go(k_embed_runs, static_cast<unsigned>(S.run_tiles), kThreads, A);
    A.scanned = max_ids == 0 || S.run_tiles > kScanTiles;
    if (A.scanned) go(k_embed_scan, 1, kThreads, A);
  }
  with_type(dy_dtype, [&](auto t) {
    using T = decltype(t);
    if (grad_dtype == SMFG_DTYPE_F32) launch_embed_grad<T, float>(A, G, clear, go);
    else launch_embed_grad<T, T>(A, G, clear, go);
  });
  return go.result();
}

// ---- layer norm ---------------------------------------------------------------------------------

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

// Blocks of k_layer_norm at most.  Rows of 256 to 8192 halfs, 128 MiB of them: 52 to 57 us with 1024 to 4096 blocks, 60 to 67 with a block for
// every row or group of rows, whose parameters are more bytes than the row; rows of floats 95 to 108 with either.
constexpr unsigned kNormBlocks = 2048;
template <typename T>
struct LaunchNorm {
  const NormArgs& A;
  Launches& go;
  template <int V, int NV, int LANES>
  void operator()() const {
    const unsigned blocks = blocks_for(A.max_rows, norm_threads(LANES) / LANES, kNormBlocks);
    go(k_layer_norm<T, V, NV, LANES>, blocks, norm_threads(LANES), A);
  }
};

// Slices of the weight's gradient.  Rows in registers: the blocks of the launch, 16 MiB of sums, but 256 to 1024 (16 K rows of 4096 in 128 blocks
// 169 us, 256 131, 512 with the next row on its way 80).  Longer rows: 64 at most, as the columns alone are many threads.
constexpr int kNormSlices = 1024, kNormLongSlices = 64, kNormLongDim = 16384;
int64_t norm_slices(int64_t max_rows, int32_t dim) {
  int64_t s = (int64_t(16) << 20) / (8 * static_cast<int64_t>(dim));
  const int64_t least = dim <= kNormLongDim ? 256 : 1, most = dim <= kNormLongDim ? kNormSlices : kNormLongSlices;
  if (s < least) s = least;
  if (s > most) s = most;
  return s < max_rows ? s : max_rows;
}

template <typename T>
struct LaunchNormGrad {
  const NormGradArgs& A;
  int64_t& slices;
  Launches& go;
  template <int V, int NV, int LANES>
  void operator()() const {
    const int64_t blocks = ceil_div(A.max_rows, norm_threads(LANES) / LANES);
    if (blocks < slices) slices = blocks;
    go(k_layer_norm_grad<T, V, NV, LANES>, static_cast<unsigned>(slices), norm_threads(LANES), A);
  }
};

// ---- clipping -----------------------------------------------------------------------------------

bool bad_grads(const smfg_grad_t* g, int32_t n) {
  for (int i = 0; i < n; ++i) {
    if (g[i].numel < 0 || g[i].numel >= (int64_t(1) << 48) || type_bytes(g[i].dtype) == 0) return true;
    if (g[i].d_rows && (g[i].row_elems < 1 || misaligned(g[i].d_rows, 8))) return true;
    if (misaligned(g[i].grad, static_cast<uintptr_t>(type_bytes(g[i].dtype)))) return true;
    if (!g[i].out) continue;
    if ((g[i].out_dtype != g[i].dtype && g[i].out_dtype != SMFG_DTYPE_F32) || misaligned(g[i].out, static_cast<uintptr_t>(type_bytes(g[i].out_dtype)))) return true;
    if (g[i].out == g[i].grad && g[i].out_dtype != g[i].dtype) return true;
  }
  return false;
}

// Elements of a block: as few as a turn of its threads, as many as leave 4096 blocks, or 64 Ki.
int64_t clip_chunk(const smfg_grad_t* g, int32_t n) {
  double all = 0;
  for (int i = 0; i < n; ++i) all += static_cast<double>(g[i].numel);
  int64_t chunk = kClipLeast;
  while (chunk < kClipMost && all > 4096.0 * static_cast<double>(2 * chunk)) chunk *= 2;
  return chunk;
}
int64_t clip_blocks(const smfg_grad_t* g, int32_t n, int64_t chunk) {
  int64_t b = 0;
  for (int i = 0; i < n; ++i) b += ceil_div(g[i].numel, chunk);
  return b;
}

int clip_tensors(const smfg_grad_t* g, int32_t n) {
  int m = 0;
  for (int i = 0; i < n; ++i) m += g[i].numel > 0;
  return m;
}

// Scratch: the factor, the table of more tensors than the arguments hold, the blocks' sums.
struct ClipScratch {
  int64_t table, part, bytes, blocks, chunk;
  int32_t tensors;
};
ClipScratch clip_scratch(const smfg_grad_t* g, int32_t n) {
  ClipScratch S;
  S.chunk = clip_chunk(g, n);
  S.blocks = clip_blocks(g, n, S.chunk);
  S.tensors = clip_tensors(g, n);
  S.table = 256;
  S.part = S.table + (S.tensors > kClipTensors ? up256(static_cast<int64_t>(sizeof(ClipTensor)) * S.tensors) : 0);
  S.bytes = S.part + up256(8 * S.blocks);
  return S;
}

}  // namespace

extern "C" {

int smfg_embedding(const void* d_table, int64_t num_rows, int64_t table_stride, int32_t table_dtype, const void* d_ids, int32_t id_bytes,
                   const int64_t* d_num_ids, int64_t max_ids, int32_t dim, float scale, void* d_out, int64_t out_stride, int32_t out_dtype,
                   void* hip_stream) {
  if (!d_table || !d_num_ids || (max_ids > 0 && (!d_ids || !d_out))) return SMFG_ERR_NULL_PTR;
  if (bad_dim(dim) || (id_bytes != 4 && id_bytes != 8) || max_ids < 0 || max_ids >= kMaxRows || num_rows < 1 || num_rows >= kMaxRows ||
      bad_matrix(d_table, table_dtype, table_stride, dim) || bad_matrix(d_out, out_dtype, out_stride, dim) ||
      (table_dtype != SMFG_DTYPE_F32 && table_dtype != out_dtype) || misaligned(d_ids, static_cast<uintptr_t>(id_bytes)) || misaligned(d_num_ids, 8))
    return SMFG_ERR_INVALID_ARG;
  if (max_ids == 0) return SMFG_OK;
  Launches go(hip_stream);
  const EmbedArgs A = {d_table, num_rows, table_stride, dim, id_bytes, d_ids, d_num_ids, max_ids, scale, d_out, out_stride, 0};
  const int vector = static_cast<int>(16 / type_bytes(out_dtype));
  const bool vectors = dim >= vector;
  const int64_t blocks = ceil_div(max_ids * ceil_div(dim, vectors ? vector : 1), kEmbedTurns * kThreads);
  if (blocks >= kMaxRows) return SMFG_ERR_INVALID_ARG;
  with_type(out_dtype, [&](auto o) {
    using O = decltype(o);
    if (table_dtype == SMFG_DTYPE_F32) launch_embedding<float, O>(A, blocks, vectors, go);
    else launch_embedding<O, O>(A, blocks, vectors, go);
  });
  return go.result();
}

int64_t smfg_embedding_grad_scratch_bytes(int64_t max_ids, int64_t num_rows, int32_t dim) {
  if (bad_dim(dim) || max_ids < 0 || max_ids >= kMaxRows || num_rows < 1 || num_rows >= kMaxRows || too_many_blocks(max_ids, dim)) return -1;
  return embed_scratch(max_ids, dim).bytes;
}

int smfg_embedding_grad(const void* d_ids, int32_t id_bytes, const int64_t* d_num_ids, int64_t max_ids, const void* d_dy, int64_t dy_stride,
                        int32_t dy_dtype, int32_t dim, float scale, void* d_grad, int64_t num_rows, int64_t grad_stride, int32_t grad_dtype,
                        int32_t accumulate, void* d_scratch, int64_t scratch_bytes, void* hip_stream) {
  return embedding_grad(d_ids, id_bytes, d_num_ids, max_ids, d_dy, dy_stride, dy_dtype, dim, scale, d_grad, num_rows, grad_stride, grad_dtype,
                        accumulate, false, nullptr, nullptr, d_scratch, scratch_bytes, hip_stream);
}

int smfg_embedding_grad_rows(const void* d_ids, int32_t id_bytes, const int64_t* d_num_ids, int64_t max_ids, const void* d_dy, int64_t dy_stride,
                             int32_t dy_dtype, int32_t dim, float scale, int64_t num_rows, int32_t* d_row_ids, int64_t* d_num_unique, void* d_grad,
                             int64_t grad_stride, int32_t grad_dtype, void* d_scratch, int64_t scratch_bytes, void* hip_stream) {
  return embedding_grad(d_ids, id_bytes, d_num_ids, max_ids, d_dy, dy_stride, dy_dtype, dim, scale, d_grad, num_rows, grad_stride, grad_dtype, 0,
                        true, d_row_ids, d_num_unique, d_scratch, scratch_bytes, hip_stream);
}

int smfg_layer_norm(const void* d_x, int64_t x_stride, int32_t dtype, const int64_t* d_num_rows, int64_t max_rows, int32_t dim, const void* d_w,
                    const void* d_b, int32_t param_dtype, float eps, void* d_y, int64_t y_stride, float* d_mean, float* d_rstd, void* hip_stream) {
  if (!d_num_rows || (max_rows > 0 && (!d_x || !d_y))) return SMFG_ERR_NULL_PTR;
  if (bad_dim(dim) || max_rows < 0 || max_rows >= kMaxRows || bad_matrix(d_x, dtype, x_stride, dim) || bad_matrix(d_y, dtype, y_stride, dim) ||
      (param_dtype != SMFG_DTYPE_F32 && param_dtype != dtype) || misaligned(d_w, static_cast<uintptr_t>(type_bytes(param_dtype))) ||
      misaligned(d_b, static_cast<uintptr_t>(type_bytes(param_dtype))) || !(eps >= 0.f) || misaligned(d_num_rows, 8) || misaligned(d_mean, 4) ||
      misaligned(d_rstd, 4) || (d_x == d_y && x_stride != y_stride))
    return SMFG_ERR_INVALID_ARG;
  if (max_rows == 0) return SMFG_OK;
  Launches go(hip_stream);
  const NormArgs A = {d_x, x_stride, d_num_rows, max_rows, dim, param_dtype == SMFG_DTYPE_F32, d_w, d_b, eps, d_y, y_stride, d_mean, d_rstd, 0};
  with_type(dtype, [&](auto t) {
    using T = decltype(t);
    if (!with_row_shape<T, 2048>(dim, LaunchNorm<T>{A, go})) go.all(k_layer_norm_long<T, kVec<T>>, max_rows, kThreads, A);
  });
  return go.result();
}

int64_t smfg_layer_norm_grad_scratch_bytes(int64_t max_rows, int32_t dim) {
  if (bad_dim(dim) || max_rows < 0 || max_rows >= kMaxRows) return -1;
  return up256(norm_slices(max_rows, dim) * 8 * dim);
}

int smfg_layer_norm_grad(const void* d_dy, int64_t dy_stride, const void* d_x, int64_t x_stride, int32_t dtype, const int64_t* d_num_rows,
                         int64_t max_rows, int32_t dim, const void* d_w, int32_t param_dtype, const float* d_mean, const float* d_rstd, void* d_dx,
                         int64_t dx_stride, void* d_dw, void* d_db, void* d_scratch, int64_t scratch_bytes, void* hip_stream) {
  const bool sums = d_dw || d_db;
  if (!d_num_rows || (max_rows > 0 && (!d_x || !d_dy || !d_mean || !d_rstd || (sums && !d_scratch)))) return SMFG_ERR_NULL_PTR;
  if (bad_dim(dim) || max_rows < 0 || max_rows >= kMaxRows || bad_matrix(d_x, dtype, x_stride, dim) || bad_matrix(d_dy, dtype, dy_stride, dim) ||
      (d_dx && bad_matrix(d_dx, dtype, dx_stride, dim)) || (param_dtype != SMFG_DTYPE_F32 && param_dtype != dtype))
    return SMFG_ERR_INVALID_ARG;
  const uintptr_t pa = static_cast<uintptr_t>(type_bytes(param_dtype));
  if (misaligned(d_w, pa) || misaligned(d_dw, pa) || misaligned(d_db, pa) || misaligned(d_num_rows, 8) || misaligned(d_mean, 4) ||
      misaligned(d_rstd, 4) || misaligned(d_scratch, 256) || (d_dx && ((d_dx == d_dy && dx_stride != dy_stride) || (d_dx == d_x && dx_stride != x_stride))))
    return SMFG_ERR_INVALID_ARG;
  int64_t slices = norm_slices(max_rows, dim);
  if (sums && scratch_bytes < up256(slices * 8 * dim)) return SMFG_ERR_CAPACITY;
  Launches go(hip_stream);
  float* part = sums ? static_cast<float*>(d_scratch) : nullptr;
  const NormGradArgs A = {d_dy, dy_stride, d_x, x_stride, d_num_rows, max_rows, dim, param_dtype == SMFG_DTYPE_F32, d_w, d_mean, d_rstd, d_dx, dx_stride, part, 0};
  if (!sums && (max_rows == 0 || !d_dx)) return SMFG_OK;
  if (max_rows > 0) {
    with_type(dtype, [&](auto t) {
      using T = decltype(t);
      constexpr int V = kVec<T>;
      if (with_row_shape<T, sizeof(T) == 4 ? 2048 : 1536>(dim, LaunchNormGrad<T>{A, slices, go})) return;
      if (sums) {
        if (slices > kNormLongSlices) slices = kNormLongSlices;
        go(k_norm_grad_columns<T, V>, dim3(static_cast<unsigned>(ceil_div(ceil_div(dim, V), kThreads)), static_cast<unsigned>(slices)), kThreads, A);
      }
      if (d_dx) go.all(k_layer_norm_grad_long<T, V>, max_rows, kThreads, A);
    });
  }
  if (sums) {
    const unsigned blocks = static_cast<unsigned>(ceil_div(2 * static_cast<int64_t>(dim), kNormJoinCols));
    with_type(param_dtype, [&](auto p) {
      using P = decltype(p);
      go(k_norm_grad_join<P>, blocks, kNormJoinThreads, part, static_cast<int32_t>(slices), dim, static_cast<P*>(d_dw), static_cast<P*>(d_db));
    });
  }
  return go.result();
}

int64_t smfg_clip_grad_norm_scratch_bytes(const smfg_grad_t* grads, int32_t num_grads) {
  if (num_grads < 0 || (num_grads > 0 && !grads) || bad_grads(grads, num_grads)) return -1;
  return clip_scratch(grads, num_grads).bytes;
}

int smfg_clip_grad_norm(const smfg_grad_t* grads, int32_t num_grads, float scale, float max_norm, float* d_norm, void* d_scratch,
                        int64_t scratch_bytes, void* hip_stream) {
  if ((num_grads > 0 && !grads) || !d_norm || !d_scratch) return SMFG_ERR_NULL_PTR;
  if (num_grads < 0 || bad_grads(grads, num_grads) || !std::isfinite(scale) || !(max_norm > 0.f) || misaligned(d_norm, 4) || misaligned(d_scratch, 256))
    return SMFG_ERR_INVALID_ARG;
  for (int i = 0; i < num_grads; ++i)
    if (grads[i].numel > 0 && !grads[i].grad) return SMFG_ERR_NULL_PTR;
  const ClipScratch S = clip_scratch(grads, num_grads);
  if (S.blocks >= kMaxRows) return SMFG_ERR_INVALID_ARG;
  if (scratch_bytes < S.bytes) return SMFG_ERR_CAPACITY;
  Launches go(hip_stream);
  uint8_t* scratch = static_cast<uint8_t*>(d_scratch);
  double* part = reinterpret_cast<double*>(scratch + S.part);
  const bool table = S.tensors > kClipTensors;
  ClipArgs A;
  A.table = table ? reinterpret_cast<ClipTensor*>(scratch + S.table) : nullptr;
  A.tensors = S.tensors;
  A.first = A.here = 0;
  A.first_block = 0;
  A.blocks = 0;
  A.chunk = S.chunk;
  A.part = part;
  A.factor = static_cast<ClipFactor*>(d_scratch);
  A.norm = d_norm;
  A.scale = scale;
  A.max_norm = max_norm;
  for (int i = 0; i < num_grads; ++i) {
    const smfg_grad_t& g = grads[i];
    if (g.numel == 0) continue;
    if (A.here == kClipTensors) {
      go(k_clip_table, 1, 64, A);
      A.first += A.here;
      A.here = 0;
    }
    A.t[A.here++] = {g.grad, g.out ? g.out : const_cast<void*>(g.grad), g.numel, g.d_rows, g.d_rows ? g.row_elems : 1, A.blocks,
                     g.dtype | (g.out ? g.out_dtype : g.dtype) << 4};
    A.blocks += static_cast<uint32_t>(ceil_div(g.numel, S.chunk));
  }
  if (table) go(k_clip_table, 1, 64, A);
  if (A.blocks > 0) {
    if (table) go.all(k_clip_squares<true>, A.blocks, kThreads, A);
    else go.all(k_clip_squares<false>, A.blocks, kThreads, A);
  }
  if (A.blocks == 0 || A.blocks > kClipJoin) go(k_clip_norm, 1, kClipNormThreads, A);
  if (A.blocks > 0) {
    if (table) go.all(k_clip_scale<true>, A.blocks, kThreads, A);
    else go.all(k_clip_scale<false>, A.blocks, kThreads, A);
  }
  return go.result();
}

}  // extern "C"
