// libsmfg embedding: scaled rows of a table by id, and the table's gradient from ids sorted by row.
#ifndef SMFG_KERNELS_EMBED_H_
#define SMFG_KERNELS_EMBED_H_

#include "elements.h"

namespace smfg_dev {

// Ids of 4 or 8 bytes; one outside [0, num_rows) stands for no row and is read as num_rows.  An id's words are read without a
// condition, as a load under one is waited for before the next: an id of 4 bytes as its own upper word, which is not looked at.
__device__ __forceinline__ uint32_t row_of_id(const void* ids, int32_t id_bytes, int64_t i, int64_t num_rows) {
  const int words = id_bytes >> 2;
  const uint32_t* p = static_cast<const uint32_t*>(ids) + i * words;
  const uint32_t lower = p[0], upper = p[words - 1];
  return (lower < num_rows) & ((words == 1) | (upper == 0)) ? lower : static_cast<uint32_t>(num_rows);
}

struct EmbedArgs {
  const void* table;
  int64_t num_rows;
  int64_t table_stride;
  int32_t dim;
  int32_t id_bytes;
  const void* ids;
  const int64_t* num;
  int64_t max_ids;
  float scale;
  void* out;
  int64_t out_stride;
};

// out[i, :] = scale * table[ids[i], :].  The output is one sequence of vectors, ceil(dim / V) a row, of which a block writes
// kEmbedTurns * kThreads.
constexpr int kEmbedTurns = 4;
template <typename TI, typename TO, int V>
__global__ void __launch_bounds__(kThreads) k_embedding(EmbedArgs A) {
  const int64_t n = count_of(A.num, A.max_ids);
  const uint32_t per_row = static_cast<uint32_t>((A.dim + V - 1) / V);
  const int64_t first = static_cast<int64_t>(blockIdx.x) * (kEmbedTurns * kThreads);
  const int64_t row0 = first / per_row;
  if (row0 >= n) return;
  const uint32_t off = static_cast<uint32_t>(first - row0 * per_row);
  uint32_t row[kEmbedTurns], at[kEmbedTurns], id[kEmbedTurns];
#pragma unroll
  for (int k = 0; k < kEmbedTurns; ++k) {
    const uint32_t i = off + k * kThreads + threadIdx.x;
    row[k] = i / per_row;
    at[k] = i - row[k] * per_row;
    const int64_t r = row0 + row[k];
    id[k] = row_of_id(A.ids, A.id_bytes, r < A.max_ids ? r : A.max_ids - 1, A.num_rows);
  }
  Elems<TI, V> e[kEmbedTurns];
#pragma unroll
  for (int k = 0; k < kEmbedTurns; ++k) {
    // row 0 stands for one that there is not: a load under a condition is waited for before the next
    e[k] = *reinterpret_cast<const Elems<TI, V>*>(static_cast<const TI*>(A.table) + (id[k] < A.num_rows ? id[k] : 0u) * A.table_stride +
                                                  Columns<V>(at[k], A.dim).start);
  }
#pragma unroll
  for (int k = 0; k < kEmbedTurns; ++k) {
    if (row0 + row[k] >= n) continue;
    Elems<TO, V> o;
#pragma unroll
    for (int j = 0; j < V; ++j) o.v[j] = from_float<TO>(id[k] < A.num_rows ? A.scale * as_float(e[k].v[j]) : 0.f);
    *reinterpret_cast<Elems<TO, V>*>(static_cast<TO*>(A.out) + (row0 + row[k]) * A.out_stride + Columns<V>(at[k], A.dim).start) = o;
  }
}

// ---- ids sorted by row -------------------------------------------------------------------------
//
// A stable sort by digits of 8 bits from the lowest on, three launches a digit: count (per tile of kSortTile tokens), scan
// (a block per digit over the tiles, then every tile adds the totals of the smaller digits), scatter.  The order of equal ids is that
// of their tokens, so that a row's sum has one order, whatever the schedule.
constexpr int kSortTile = 4096;
constexpr int kSortTurns = kSortTile / kThreads;
constexpr int kSortBits = 8;
constexpr int kSortBins = 1 << kSortBits;

struct SortArgs {
  const void* ids;      // first digit: the ids
  int32_t id_bytes;
  int32_t shift;
  int64_t num_rows;
  const int64_t* num;
  int64_t max_ids;
  const uint2* in;      // other digits: (row, token)
  uint2* out;
  uint32_t* hist;       // [bins][tiles]
  uint32_t* total;      // [bins]
  int32_t tiles;
};

__device__ __forceinline__ uint2 sort_record(const SortArgs& A, int64_t i) {
  return A.in ? A.in[i] : make_uint2(row_of_id(A.ids, A.id_bytes, i, A.num_rows), static_cast<uint32_t>(i));
}

static __global__ void __launch_bounds__(kThreads) k_sort_count(SortArgs A) {
  __shared__ uint32_t count[kSortBins];
  const int64_t n = count_of(A.num, A.max_ids);
  count[threadIdx.x] = 0;
  __syncthreads();
  const int64_t base = static_cast<int64_t>(blockIdx.x) * kSortTile;
  for (int k = 0; k < kSortTurns; ++k) {
    const int64_t i = base + k * kThreads + threadIdx.x;
    if (i < n) atomicAdd(&count[(sort_record(A, i).x >> A.shift) & (kSortBins - 1)], 1u);
  }
  __syncthreads();
  A.hist[static_cast<int64_t>(threadIdx.x) * A.tiles + blockIdx.x] = count[threadIdx.x];
}

static __global__ void __launch_bounds__(kThreads) k_sort_scan(SortArgs A) {
  __shared__ uint32_t lds[kThreads / 64];
  uint32_t* h = A.hist + static_cast<int64_t>(blockIdx.x) * A.tiles;
  uint32_t before = 0;
  for (int t0 = 0; t0 < A.tiles; t0 += kThreads) {
    const int t = t0 + threadIdx.x;
    const uint32_t c = t < A.tiles ? h[t] : 0u;
    uint32_t sum;
    const uint32_t ex = block_exscan(c, lds, sum);
    if (t < A.tiles) h[t] = before + ex;
    before += sum;
  }
  if (threadIdx.x == 0) A.total[blockIdx.x] = before;
}

static __global__ void __launch_bounds__(kThreads) k_sort_scatter(SortArgs A) {
  constexpr int kWaves = kThreads / 64;
  __shared__ uint32_t next[kWaves][kSortBins];  // records of a wave so far, later where its next record goes
  __shared__ uint32_t lds[kWaves];
  const int64_t n = count_of(A.num, A.max_ids);
  const int64_t base = static_cast<int64_t>(blockIdx.x) * kSortTile;
  if (base >= n) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int q = 0; q < kWaves; ++q) next[q][threadIdx.x] = 0;
  __syncthreads();
  // a wave has consecutive records, 64 a turn: its rank among equal digits of the wave
  uint2 rec[kSortTurns];
  uint32_t rank[kSortTurns];
#pragma unroll
  for (int k = 0; k < kSortTurns; ++k) {
    const int64_t i = base + (wave * kSortTurns + k) * 64 + lane;
    const bool live = i < n;
    rec[k] = live ? sort_record(A, i) : make_uint2(0, 0);
    const uint32_t digit = (rec[k].x >> A.shift) & (kSortBins - 1);
    uint64_t same = __ballot(live);
#pragma unroll
    for (int b = 0; b < kSortBits; ++b) {
      const uint64_t set = __ballot((digit >> b) & 1u);
      same &= (digit >> b) & 1u ? set : ~set;
    }
    const uint32_t below = __popcll(same & ((1ull << lane) - 1));
    rank[k] = 0;
    if (live) rank[k] = next[wave][digit] + below;  // every lane reads before the first of each digit adds
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (live && below == 0) next[wave][digit] += __popcll(same);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
  __syncthreads();
  // where the tile's records of each digit begin: behind all smaller digits, and those of the tiles before
  uint32_t all;
  const uint32_t digits_before = block_exscan(A.total[threadIdx.x], lds, all);
  uint32_t at = digits_before + A.hist[static_cast<int64_t>(threadIdx.x) * A.tiles + blockIdx.x];
#pragma unroll
  for (int q = 0; q < kWaves; ++q) {
    const uint32_t c = next[q][threadIdx.x];
    next[q][threadIdx.x] = at;
    at += c;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kSortTurns; ++k) {
    const int64_t i = base + (wave * kSortTurns + k) * 64 + lane;
    if (i < n) A.out[next[wave][(rec[k].x >> A.shift) & (kSortBins - 1)] + rank[k]] = rec[k];
  }
}

// ---- sums over runs of equal rows --------------------------------------------------------------
//
// The sorted tokens are cut into pieces of kGradTokens, each the work of one wave, whatever the ids are, so that a frequent id is no
// one's burden.  A run that begins and ends in a piece is a row of the gradient.  Of one that crosses pieces, what a piece has of a
// run that began before it (its head) and of one that goes on behind it (its tail) is joined in the block, in the order of the
// tokens; what crosses blocks goes to `part`, from where k_embed_join adds it up.
//
// A wave has one row at a time, so that rows, their ends and the addresses are scalar: with groups of 32 lanes, two rows to a wave, ends that
// differ made both halves wait and every lane work out addresses.  A lane has V columns, as few as let 64 lanes have the whole row.
constexpr int kGradTokens = 16;
constexpr int kGradWaves = 8;
constexpr int kGradThreads = 64 * kGradWaves;
constexpr int kBlockTokens = kGradWaves * kGradTokens;
constexpr int kRunTile = 1024;     // a multiple of every block's tokens
constexpr int kScanTiles = 1024;   // more run tiles than that are scanned by a launch of their own
constexpr int grad_columns(int dim) { return dim <= 64 ? 1 : dim <= 128 ? 2 : 4; }

struct EmbedGradArgs {
  const uint2* sorted;     // (row, token)
  const int64_t* num;
  int64_t max_ids;
  int64_t num_rows;
  int32_t dim;
  int32_t accumulate;
  const void* dy;
  int64_t dy_stride;
  float scale;
  uint32_t sum_blocks, tiles;  // blocks of k_embed_sums that add up, and tiles of columns; the blocks behind all of them clear
  void* grad;
  int64_t grad_stride;
  float* part;             // [blocks][2][part_width]: head and tail
  int64_t part_width;
  int32_t clear_rows;      // rows of a block that clears
  // touched rows alone (row_ids != null): a run's row of `grad` is its rank
  int32_t scanned;         // tile_runs holds its exclusive scan
  int32_t* row_ids;
  int64_t* num_unique;
  uint32_t* tile_runs;     // runs that begin in a tile of kRunTile sorted tokens
  uint32_t* block_runs;    // runs that begin in a block's tile before it
  int64_t run_tiles;
};

static __global__ void __launch_bounds__(kThreads) k_embed_runs(EmbedGradArgs A) {
  __shared__ uint32_t lds[kThreads / 64];
  constexpr int kPer = kRunTile / kThreads;
  const int64_t n = count_of(A.num, A.max_ids);
  const int64_t p0 = static_cast<int64_t>(blockIdx.x) * kRunTile + threadIdx.x * kPer;
  const uint32_t none = static_cast<uint32_t>(A.num_rows);
  uint32_t keys[kPer + 1], sum = 0;
#pragma unroll
  for (int k = 0; k <= kPer; ++k) keys[k] = A.sorted[p0 + k > 0 && p0 + k <= A.max_ids ? p0 + k - 1 : 0].x;
#pragma unroll
  for (int k = 0; k < kPer; ++k) sum += p0 + k < n && keys[k + 1] < none && (p0 + k == 0 || keys[k] != keys[k + 1]) ? 1u : 0u;
  uint32_t total;
  const uint32_t before = block_exscan(sum, lds, total);
  if (p0 % kBlockTokens == 0 && p0 < A.max_ids) A.block_runs[p0 / kBlockTokens] = before;
  if (threadIdx.x == 0) A.tile_runs[blockIdx.x] = total;
}

// Exclusive scan of the tiles' runs, by one block; their number.
static __global__ void __launch_bounds__(kThreads) k_embed_scan(EmbedGradArgs A) {
  __shared__ uint32_t lds[kThreads / 64];
  uint32_t before = 0;
  for (int64_t t0 = 0; t0 < A.run_tiles; t0 += kThreads) {
    const int64_t t = t0 + threadIdx.x;
    const uint32_t c = t < A.run_tiles ? A.tile_runs[t] : 0u;
    uint32_t sum;
    const uint32_t ex = block_exscan(c, lds, sum);
    if (t < A.run_tiles) A.tile_runs[t] = before + ex;
    before += sum;
  }
  if (threadIdx.x == 0) *A.num_unique = before;
}

// A thread's share of the runs that begin before a block's tokens; all: of all runs, where the tiles are not scanned, for block 0.
__device__ __forceinline__ uint32_t share_of_runs(const EmbedGradArgs& A, uint32_t block, uint32_t& all) {
  const int64_t tile = static_cast<int64_t>(block) * kBlockTokens / kRunTile;
  uint32_t x = threadIdx.x == 0 ? A.block_runs[block] : 0u;
  all = 0;
  if (A.scanned) return threadIdx.x == 0 ? x + A.tile_runs[tile] : 0u;
  if (block == 0)
    for (int64_t t = threadIdx.x; t < A.run_tiles; t += blockDim.x) all += A.tile_runs[t];
  for (int64_t t = threadIdx.x; t < tile; t += blockDim.x) x += A.tile_runs[t];
  return x;
}

// V columns of a row of the gradient from their sum; those that the vector before has as well are left to it.
template <typename TG, int V>
__device__ __forceinline__ void write_grad(const EmbedGradArgs& A, int64_t row, const Columns<V>& c, const float (&sum)[V]) {
  TG* g = static_cast<TG*>(A.grad) + row * A.grad_stride + c.start;
  if (c.dup == 0) {
    Elems<TG, V> e = {};
    if (A.accumulate) e = *reinterpret_cast<const Elems<TG, V>*>(g);
#pragma unroll
    for (int j = 0; j < V; ++j) e.v[j] = from_float<TG>(as_float(e.v[j]) + A.scale * sum[j]);
    *reinterpret_cast<Elems<TG, V>*>(g) = e;
  } else if (c.dup < V) {
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (j >= c.dup) g[j] = from_float<TG>((A.accumulate ? as_float(g[j]) : 0.f) + A.scale * sum[j]);
  }
}

// First sorted place whose row is at least `key`, in [lo, hi].
__device__ __forceinline__ int64_t sorted_bound(const uint2* sorted, int64_t lo, int64_t hi, uint32_t key) {
  while (lo < hi) {
    const int64_t mid = lo + (hi - lo) / 2;
    if (sorted[mid].x < key) lo = mid + 1;
    else hi = mid;
  }
  return lo;
}
// The same by a wave, 64 places at a time.
__device__ __forceinline__ int64_t wave_sorted_bound(const uint2* sorted, int64_t lo, int64_t hi, uint32_t key) {
  const int lane = threadIdx.x & 63;
  while (lo < hi) {  // the bound is in [lo, hi]
    const int64_t step = (hi - lo + 63) / 64, at = lo + lane * step;
    const int below = __popcll(__ballot(at < hi && sorted[at < hi ? at : lo].x < key));
    if (below == 0) return lo;
    const int64_t last = lo + (below - 1) * step;  // below the bound
    hi = last + step < hi ? last + step : hi;
    lo = last + 1;
  }
  return lo;
}

// Rows of the whole table's gradient that no token names: zeros.
template <typename TG, int V>
__device__ __forceinline__ void clear_rows(const EmbedGradArgs& A, int64_t n, uint32_t block, uint32_t* lds) {
  const int64_t r0 = static_cast<int64_t>(block) * A.clear_rows;
  const int rows = static_cast<int>(A.num_rows - r0 < A.clear_rows ? A.num_rows - r0 : A.clear_rows);
  const int64_t lo = wave_sorted_bound(A.sorted, 0, n, static_cast<uint32_t>(r0));
  const int64_t hi = wave_sorted_bound(A.sorted, lo, n, static_cast<uint32_t>(r0 + rows));
  if (static_cast<int>(threadIdx.x) < rows) {
    const uint32_t key = static_cast<uint32_t>(r0) + threadIdx.x;
    const int64_t p = sorted_bound(A.sorted, lo, hi, key);
    lds[threadIdx.x] = p < hi && A.sorted[p].x == key;
  }
  __syncthreads();
  const uint32_t per_row = static_cast<uint32_t>((A.dim + V - 1) / V);
  TG* g = static_cast<TG*>(A.grad) + r0 * A.grad_stride;
  for (uint32_t i = threadIdx.x; i < rows * per_row; i += blockDim.x) {
    const uint32_t r = i / per_row;
    if (!lds[r]) *reinterpret_cast<Elems<TG, V>*>(g + r * A.grad_stride + Columns<V>(static_cast<int>(i - r * per_row), A.dim).start) = {};
  }
}

template <typename TD, typename TG, int V>
__global__ void __launch_bounds__(kGradThreads) k_embed_sums(EmbedGradArgs A) {
  __shared__ float heads[kGradWaves][64 * V];
  __shared__ uint32_t goes_on[kGradWaves];  // the wave's tokens are all of one run, that began before them and goes on behind them
  __shared__ uint32_t lds[kGradThreads];
  const uint32_t tile = blockIdx.x / A.sum_blocks, block = blockIdx.x - tile * A.sum_blocks;
  const int64_t n = count_of(A.num, A.max_ids);
  if (tile >= A.tiles) {
    clear_rows<TG, V>(A, n, blockIdx.x - A.sum_blocks * A.tiles, lds);
    return;
  }
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t b0 = static_cast<int64_t>(block) * kBlockTokens, p0 = b0 + wave * kGradTokens;
  const uint32_t none = static_cast<uint32_t>(A.num_rows);
  const int index = static_cast<int>(tile) * 64 + lane;
  const Columns<V> c(index, A.dim);
  // the wave's tokens, one to a lane, from lane 1 on; lane 0 has the one before, lane kGradTokens + 1 the one behind
  const int64_t at = p0 - 1 + lane;
  uint2 mine = A.sorted[at < 0 ? 0 : at < A.max_ids ? at : A.max_ids - 1];
  if (lane > kGradTokens + 1 || at < 0 || at >= n) mine = make_uint2(none, 0);
  uint32_t rank = 0, all = 0;
  if (A.row_ids) rank = share_of_runs(A, block, all);
  // Every row is read, also a padded place's and for columns that there are not (the last ones again), and dropped later: loads under a
  // condition are waited for one by one.  Token 0 stands for those behind the last.
  const TD* dy = static_cast<const TD*>(A.dy);
  Elems<TD, V> e[kGradTokens];
#pragma unroll
  for (int u = 0; u < kGradTokens; ++u) {
    const uint32_t token = __builtin_amdgcn_readlane(mine.y, u + 1);
    e[u] = *reinterpret_cast<const Elems<TD, V>*>(dy + token * A.dy_stride + c.start);
  }
  if (A.row_ids) {
    const uint32_t left = __shfl_up(mine.x, 1, 64);  // by all lanes: not in the condition
    const bool begins = lane >= 1 && lane <= kGradTokens && mine.x < none && mine.x != left;
    const uint64_t set = __ballot(begins);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      rank += __shfl_xor(rank, o, 64);
      if (block == 0) all += __shfl_xor(all, o, 64);
    }
    if (lane == 0) {
      lds[wave] = rank;
      lds[kGradWaves + wave] = all;
      lds[2 * kGradWaves + wave] = __popcll(set);
    }
    __syncthreads();
    rank = all = 0;
    for (int w = 0; w < kGradWaves; ++w) {
      rank += lds[w] + (w < wave ? lds[2 * kGradWaves + w] : 0u);
      all += lds[kGradWaves + w];
    }
    rank = __builtin_amdgcn_readfirstlane(rank);
    if (blockIdx.x == 0 && threadIdx.x == 0 && !A.scanned) *A.num_unique = all;
    if (begins && tile == 0) A.row_ids[rank + __popcll(set & ((1ull << lane) - 1))] = static_cast<int32_t>(mine.x);
  }
  if (b0 >= n) return;
  const uint32_t before = __builtin_amdgcn_readlane(mine.x, 0), first = __builtin_amdgcn_readlane(mine.x, 1);
  const uint32_t key = __builtin_amdgcn_readlane(mine.x, kGradTokens), behind = __builtin_amdgcn_readlane(mine.x, kGradTokens + 1);
  const bool began_before = first < none && first == before, open = key < none && key == behind;
  bool head = began_before;
  float sum[V] = {};
#pragma unroll
  for (int u = 0; u < kGradTokens; ++u) {
#pragma unroll
    for (int j = 0; j < V; ++j) sum[j] += as_float(e[u].v[j]);
    const uint32_t here = __builtin_amdgcn_readlane(mine.x, u + 1), next = __builtin_amdgcn_readlane(mine.x, u + 2);
    if (here == next) continue;  // the run goes on
    if (here < none) {
      if (head) {
#pragma unroll
        for (int j = 0; j < V; ++j) heads[wave][j * 64 + lane] = sum[j];
      } else {
        write_grad<TG, V>(A, A.row_ids ? static_cast<int64_t>(rank++) : static_cast<int64_t>(here), c, sum);
      }
    }
    head = false;
#pragma unroll
    for (int j = 0; j < V; ++j) sum[j] = 0.f;
  }
  if (open && head) {
#pragma unroll
    for (int j = 0; j < V; ++j) heads[wave][j * 64 + lane] = sum[j];
  }
  if (lane == 0) goes_on[wave] = open && head ? 1u : 0u;
  __syncthreads();
  float* part = A.part + static_cast<int64_t>(block) * 2 * A.part_width + static_cast<int64_t>(index) * V;
  if (c.dup == V) return;
  // the run that goes on behind the wave's tokens, unless it began before them
  if (open && !head) {
    int w = wave + 1;
    for (; w < kGradWaves; ++w) {
#pragma unroll
      for (int j = 0; j < V; ++j) sum[j] += heads[w][j * 64 + lane];
      if (!goes_on[w]) break;
    }
    if (w < kGradWaves) {
      write_grad<TG, V>(A, A.row_ids ? static_cast<int64_t>(rank) : static_cast<int64_t>(key), c, sum);
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) part[A.part_width + j] = sum[j];
    }
  }
  // the run that began before the block
  if (wave == 0 && began_before) {
#pragma unroll
    for (int j = 0; j < V; ++j) sum[j] = heads[0][j * 64 + lane];
    for (int w = 0; w + 1 < kGradWaves && goes_on[w]; ++w) {
#pragma unroll
      for (int j = 0; j < V; ++j) sum[j] += heads[w + 1][j * 64 + lane];
    }
#pragma unroll
    for (int j = 0; j < V; ++j) part[j] = sum[j];
  }
}

// Place of a touched row among their ascending ids.
__device__ __forceinline__ int64_t rank_of_row(const EmbedGradArgs& A, uint32_t row) {
  int64_t lo = 0, hi = *A.num_unique;
  while (lo < hi) {
    const int64_t mid = lo + (hi - lo) / 2;
    if (static_cast<uint32_t>(A.row_ids[mid]) < row) lo = mid + 1;
    else hi = mid;
  }
  return lo;
}

// Runs that cross blocks of k_embed_sums: one that ends within kJoinShort blocks behind the one it begins in by a wave, a
// longer one by a block of its own, which is the one of the first multiple of kJoinShort behind it.
constexpr int kJoinThreads = 1024;
constexpr int kJoinWaves = kJoinThreads / 64;
constexpr int kJoinShort = 16;
template <typename TG, int V>
__global__ void __launch_bounds__(kJoinThreads) k_embed_join(EmbedGradArgs A, uint32_t short_blocks) {
  __shared__ float lds[kJoinWaves][64 * V];
  const int64_t n = count_of(A.num, A.max_ids);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int index = static_cast<int>(blockIdx.y) * 64 + lane;
  const Columns<V> c(index, A.dim);
  const int64_t width = A.part_width;
  const float* part = A.part + static_cast<int64_t>(index) * V;
  float sum[V] = {};
  if (blockIdx.x < short_blocks) {
    const int64_t b = static_cast<int64_t>(blockIdx.x) * kJoinWaves + wave, p1 = (b + 1) * kBlockTokens;
    if (p1 >= n) return;
    const uint32_t key = A.sorted[p1 - 1].x;
    if (key >= A.num_rows || (b > 0 && A.sorted[b * kBlockTokens - 1].x == key)) return;  // begins before the block
    const int64_t p = p1 + lane * kBlockTokens;
    const int blocks = __popcll(__ballot(lane < kJoinShort && p < n && A.sorted[p < n ? p : p1].x == key));  // behind b that have some of the run
    if (blocks == 0 || blocks == kJoinShort) return;
    const int64_t row = A.row_ids ? rank_of_row(A, key) : static_cast<int64_t>(key);
    if (c.dup == V) return;
#pragma unroll
    for (int j = 0; j < V; ++j) sum[j] = part[(2 * b + 1) * width + j];
    for (int q = 1; q <= blocks; ++q) {
#pragma unroll
      for (int j = 0; j < V; ++j) sum[j] += part[2 * (b + q) * width + j];
    }
    write_grad<TG, V>(A, row, c, sum);
    return;
  }
  const int64_t m = (static_cast<int64_t>(blockIdx.x - short_blocks) + 1) * kJoinShort;
  if (m * kBlockTokens >= n) return;
  const uint32_t key = A.sorted[m * kBlockTokens].x;
  if (key >= A.num_rows || A.sorted[m * kBlockTokens - 1].x != key) return;
  const int64_t b = wave_sorted_bound(A.sorted, 0, m * kBlockTokens, key) / kBlockTokens;
  const int64_t last = (wave_sorted_bound(A.sorted, m * kBlockTokens, n, key + 1) - 1) / kBlockTokens;
  if (m - b > kJoinShort || last - b < kJoinShort) return;
  const int64_t row = A.row_ids ? rank_of_row(A, key) : static_cast<int64_t>(key);
  if (c.dup < V) {
    if (wave == 0) {
#pragma unroll
      for (int j = 0; j < V; ++j) sum[j] = part[(2 * b + 1) * width + j];
    }
#pragma unroll 8
    for (int64_t q = b + 1 + wave; q <= last; q += kJoinWaves) {
#pragma unroll
      for (int j = 0; j < V; ++j) sum[j] += part[2 * q * width + j];
    }
  }
#pragma unroll
  for (int j = 0; j < V; ++j) lds[wave][j * 64 + lane] = sum[j];
  __syncthreads();
  if (wave != 0 || c.dup == V) return;
  for (int w = 1; w < kJoinWaves; ++w) {
#pragma unroll
    for (int j = 0; j < V; ++j) sum[j] += lds[w][j * 64 + lane];
  }
  write_grad<TG, V>(A, row, c, sum);
}

}  // namespace smfg_dev

#endif  // SMFG_KERNELS_EMBED_H_
