// libsmfg embedding: scaled rows of a table by id, and the table's gradient from ids sorted by row.
#ifndef SMFG_KERNELS_EMBED_H_
#define SMFG_KERNELS_EMBED_H_

#include "elements.h"

namespace smfg_dev {

// Ids of 4 or 8 bytes; one outside [0, num_rows) stands for no row and is read as num_rows.
__device__ __forceinline__ uint32_t row_of_id(const void* ids, int32_t id_bytes, int64_t i, int64_t num_rows) {
  const int64_t v = id_bytes == 8 ? static_cast<const int64_t*>(ids)[i] : static_cast<const int32_t*>(ids)[i];
  return static_cast<uint32_t>(v < 0 || v >= num_rows ? num_rows : v);
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
    id[k] = row0 + row[k] < n ? row_of_id(A.ids, A.id_bytes, row0 + row[k], A.num_rows) : static_cast<uint32_t>(A.num_rows);
  }
  Elems<TI, V> e[kEmbedTurns];
#pragma unroll
  for (int k = 0; k < kEmbedTurns; ++k) {
    e[k] = {};
    if (id[k] < A.num_rows)
      e[k] = *reinterpret_cast<const Elems<TI, V>*>(static_cast<const TI*>(A.table) + id[k] * A.table_stride + Columns<V>(at[k], A.dim).start);
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
// The sorted tokens are cut into chunks of equal length, each the work of one group of lanes, whatever the ids are.  A run that
// begins and ends in a chunk is a row of the gradient; what a chunk has of a run that began before it (its head) and of one that
// goes on behind it (its tail) goes to `part`, from where k_embed_join adds it up, tail first, then the heads in their order.
struct EmbedGradArgs {
  const uint2* sorted;   // (row, token)
  const int64_t* num;
  int64_t max_ids;
  int64_t num_rows;
  int32_t chunk;         // tokens of a chunk
  int32_t dim;
  const void* dy;
  int64_t dy_stride;
  float scale;
  int32_t accumulate;
  void* grad;
  int64_t grad_stride;
  float* part;           // [chunks][2][part_width]: head and tail
  int64_t part_width;
  // touched rows alone (row_ids != null): a run's row of `grad` is its rank
  int32_t* row_ids;
  int64_t* num_unique;
  uint32_t* tile_runs;   // runs that begin in a tile of kRunTile sorted tokens
  uint32_t* chunk_runs;  // runs that begin in the tile of a chunk before it
};

constexpr int kRunTile = 1024;  // a multiple of every chunk
constexpr int kMaxChunk = 256;

// Run begins at sorted place p?
__device__ __forceinline__ bool run_begins(const EmbedGradArgs& A, int64_t p, int64_t n) {
  if (p >= n) return false;
  const uint32_t key = A.sorted[p].x;
  return key < A.num_rows && (p == 0 || A.sorted[p - 1].x != key);
}

static __global__ void __launch_bounds__(kThreads) k_embed_runs(EmbedGradArgs A) {
  __shared__ uint32_t lds[kThreads / 64];
  constexpr int kPer = kRunTile / kThreads;
  const int64_t n = count_of(A.num, A.max_ids);
  const int64_t p0 = static_cast<int64_t>(blockIdx.x) * kRunTile + threadIdx.x * kPer;
  uint32_t c[kPer], sum = 0;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    c[k] = sum;
    sum += run_begins(A, p0 + k, n) ? 1u : 0u;
  }
  uint32_t total;
  const uint32_t before = block_exscan(sum, lds, total);
#pragma unroll
  for (int k = 0; k < kPer; ++k)
    if (p0 + k < n && (p0 + k) % A.chunk == 0) A.chunk_runs[(p0 + k) / A.chunk] = before + c[k];
  if (threadIdx.x == 0) A.tile_runs[blockIdx.x] = total;
}

// Exclusive scan of the tiles' runs, by one block; their number.
static __global__ void __launch_bounds__(kThreads) k_embed_scan(EmbedGradArgs A, int64_t tiles) {
  __shared__ uint32_t lds[kThreads / 64];
  uint32_t before = 0;
  for (int64_t t0 = 0; t0 < tiles; t0 += kThreads) {
    const int64_t t = t0 + threadIdx.x;
    const uint32_t c = t < tiles ? A.tile_runs[t] : 0u;
    uint32_t sum;
    const uint32_t ex = block_exscan(c, lds, sum);
    if (t < tiles) A.tile_runs[t] = before + ex;
    before += sum;
  }
  if (threadIdx.x == 0) *A.num_unique = before;
}

// Rank among all runs of the first that begins in chunk c.
__device__ __forceinline__ uint32_t runs_before_chunk(const EmbedGradArgs& A, int64_t c) {
  return A.tile_runs[c * A.chunk / kRunTile] + A.chunk_runs[c];
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
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (j >= c.dup) g[j] = from_float<TG>((A.accumulate ? as_float(g[j]) : 0.f) + A.scale * sum[j]);
  }
}

constexpr int kGradDepth = 8;  // rows of dy on their way

// A group of LANES lanes has a chunk and LANES * V columns of it (column tile blockIdx.y).
template <typename TD, typename TG, int V, int LANES>
__global__ void __launch_bounds__(kThreads) k_embed_grad(EmbedGradArgs A) {
  constexpr int kGroups = kThreads / LANES;
  const int lane = threadIdx.x % LANES;
  const int64_t n = count_of(A.num, A.max_ids);
  const int64_t chunk = static_cast<int64_t>(blockIdx.x) * kGroups + threadIdx.x / LANES;
  const int64_t p0 = chunk * A.chunk;
  if (p0 >= n) return;
  const int len = static_cast<int>(n - p0 < A.chunk ? n - p0 : A.chunk);
  const int index = static_cast<int>(blockIdx.y) * LANES + lane;
  const Columns<V> c(index, A.dim);
  const bool live = c.dup < V;
  const uint2* rec = A.sorted + p0;
  const uint32_t none = static_cast<uint32_t>(A.num_rows);
  bool head = p0 > 0 && A.sorted[p0 - 1].x == rec[0].x;
  const uint32_t behind = p0 + len < n ? A.sorted[p0 + len].x : none;
  int64_t rank = A.row_ids ? static_cast<int64_t>(runs_before_chunk(A, chunk)) : 0;
  const TD* dy = static_cast<const TD*>(A.dy) + c.start;
  float* part = A.part + chunk * 2 * A.part_width + static_cast<int64_t>(index) * V;
  float sum[V] = {};
  uint32_t key = rec[0].x;
  for (int t0 = 0; t0 < len; t0 += kGradDepth) {
    uint32_t keys[kGradDepth];
    Elems<TD, V> e[kGradDepth];
#pragma unroll
    for (int u = 0; u < kGradDepth; ++u) {
      const uint2 r = rec[t0 + u < len ? t0 + u : len - 1];
      keys[u] = r.x;
      e[u] = {};
      if (live && t0 + u < len && r.x < none) e[u] = *reinterpret_cast<const Elems<TD, V>*>(dy + r.y * A.dy_stride);
    }
#pragma unroll
    for (int u = 0; u < kGradDepth; ++u) {
      if (t0 + u >= len) break;
      if (keys[u] != key) {  // the run of `key` ends here
        if (key < none && live) {
          if (head) {
#pragma unroll
            for (int j = 0; j < V; ++j) part[j] = sum[j];
          } else {
            write_grad<TG, V>(A, A.row_ids ? rank : static_cast<int64_t>(key), c, sum);
          }
        }
        if (!head && key < none) {
          if (A.row_ids && index == 0) A.row_ids[rank] = static_cast<int32_t>(key);
          ++rank;
        }
        head = false;
        key = keys[u];
#pragma unroll
        for (int j = 0; j < V; ++j) sum[j] = 0.f;
      }
#pragma unroll
      for (int j = 0; j < V; ++j) sum[j] += as_float(e[u].v[j]);
    }
  }
  if (key >= none) return;
  if (!head && A.row_ids && index == 0) A.row_ids[rank] = static_cast<int32_t>(key);
  if (!live) return;
  if (head || key == behind) {
    if (!head) part += A.part_width;
#pragma unroll
    for (int j = 0; j < V; ++j) part[j] = sum[j];
  } else {
    write_grad<TG, V>(A, A.row_ids ? rank : static_cast<int64_t>(key), c, sum);
  }
}

// First sorted place whose row is at least `key` (beyond: whose row is larger), from `from` on.
__device__ __forceinline__ int64_t sorted_bound(const uint2* sorted, int64_t from, int64_t n, uint32_t key, bool beyond) {
  int64_t lo = from, hi = n;
  while (lo < hi) {
    const int64_t mid = lo + (hi - lo) / 2;
    const uint32_t k = sorted[mid].x;
    if (k < key || (beyond && k == key)) lo = mid + 1;
    else hi = mid;
  }
  return lo;
}

// Runs that cross chunks: a block per chunk, which looks whether one begins in it and goes on.
template <typename TG, int V>
__global__ void __launch_bounds__(kThreads) k_embed_join(EmbedGradArgs A) {
  constexpr int kLanes = 16, kGroups = kThreads / kLanes;
  __shared__ float lds[kThreads * V];
  const int64_t n = count_of(A.num, A.max_ids);
  const int64_t chunk = blockIdx.x, p1 = (chunk + 1) * A.chunk;
  if (p1 >= n) return;
  const uint32_t key = A.sorted[p1 - 1].x;
  if (key >= A.num_rows || A.sorted[p1].x != key) return;
  const int64_t p0 = chunk * A.chunk;
  if (A.sorted[p0].x == key && p0 > 0 && A.sorted[p0 - 1].x == key) return;  // it began before
  const int64_t last = (sorted_bound(A.sorted, p1, n, key, true) - 1) / A.chunk;
  int64_t row = key;
  if (A.row_ids) {  // the last run that begins in the chunk
    row = static_cast<int64_t>(runs_before_chunk(A, chunk + 1)) - 1;
  }
  const int lane = threadIdx.x % kLanes, group = threadIdx.x / kLanes;
  const int vectors = (A.dim + V - 1) / V;
  for (int i0 = 0; i0 < vectors; i0 += kLanes) {
    const int index = i0 + lane;
    float sum[V] = {};
    if (index < vectors) {
      const float* part = A.part + static_cast<int64_t>(index) * V;
      if (group == 0) {
#pragma unroll
        for (int j = 0; j < V; ++j) sum[j] = part[(2 * chunk + 1) * A.part_width + j];
      }
      for (int64_t q = chunk + 1 + group; q <= last; q += kGroups) {
#pragma unroll
        for (int j = 0; j < V; ++j) sum[j] += part[2 * q * A.part_width + j];
      }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < V; ++j) lds[j * kThreads + threadIdx.x] = sum[j];
    __syncthreads();
    if (group == 0 && index < vectors) {
      for (int g = 1; g < kGroups; ++g) {
#pragma unroll
        for (int j = 0; j < V; ++j) sum[j] += lds[j * kThreads + g * kLanes + lane];
      }
      write_grad<TG, V>(A, row, Columns<V>(index, A.dim), sum);
    }
  }
}

// Rows of the whole table's gradient before the touched ones are written.
template <typename TG, int V>
__global__ void __launch_bounds__(kThreads) k_embed_clear(void* grad, int64_t grad_stride, int64_t num_rows, int32_t dim) {
  const int64_t per_row = (dim + V - 1) / V, all = num_rows * per_row;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < all; i += static_cast<int64_t>(gridDim.x) * kThreads) {
    const int64_t row = i / per_row;
    *reinterpret_cast<Elems<TG, V>*>(static_cast<TG*>(grad) + row * grad_stride + Columns<V>(static_cast<int>(i - row * per_row), dim).start) = {};
  }
}

}  // namespace smfg_dev

#endif  // SMFG_KERNELS_EMBED_H_
