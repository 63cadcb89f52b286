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
  uint32_t first_block;  // of the launch
};

// out[i, :] = scale * table[ids[i], :].  The output is one sequence of vectors, ceil(dim / V) a row, of which a block writes
// kEmbedTurns * kThreads: a thread's ids, then its rows are on their way together.  Memory bounds it: 540 K rows of 128 floats to half 84 us,
// 4.9 TB/s (82 to 85 with 1 to 8 turns; 16 K rows of 4096 bfloat16 51, 46, 43, 44 us with 1, 2, 4, 8).  Reading past the caches took 8 % less for
// half rows of a table far beyond them, but 20 to 27 % more where ids repeat, so the rows are read like anything else.
constexpr int kEmbedTurns = 4;
template <typename TI, typename TO, int V>
__global__ void __launch_bounds__(kThreads) k_embedding(EmbedArgs A) {
  const int64_t n = count_of(A.num, A.max_ids);
  const uint32_t per_row = static_cast<uint32_t>((A.dim + V - 1) / V);
  const int64_t first = (static_cast<int64_t>(A.first_block) + blockIdx.x) * (kEmbedTurns * kThreads);
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
    const Elems<TI, V>* p = reinterpret_cast<const Elems<TI, V>*>(static_cast<const TI*>(A.table) + (id[k] < A.num_rows ? id[k] : 0u) * A.table_stride +
                                                  Columns<V>(at[k], A.dim).start);
    e[k] = *p;
  }
#pragma unroll
  for (int k = 0; k < kEmbedTurns; ++k) {
    if (row0 + row[k] >= n) continue;
    Elems<TO, V> o;
#pragma unroll
    for (int j = 0; j < V; ++j) o.v[j] = from_float<TO>(id[k] < A.num_rows ? A.scale * as_float(e[k].v[j]) : 0.f);
    Elems<TO, V>* p = reinterpret_cast<Elems<TO, V>*>(static_cast<TO*>(A.out) + (row0 + row[k]) * A.out_stride + Columns<V>(at[k], A.dim).start);
    *p = o;
  }
}

// ---- ids sorted by row -------------------------------------------------------------------------
//
// (row, token), stable: equal ids stay in the order of their tokens, so that the parts of a row's sum are the same whatever the schedule.
//
// Up to kSmallSort ids: every token counts the ids that belong before its own, in one launch.  More: digits of at most kSortBits
// bits from the lowest on, a launch that counts the digits of every tile and one that scatters.  Up to kSortColumns tiles the block
// that scatters adds up the counts of all tiles itself; more of them are scanned by a launch between the two.  A thread has TURNS
// records of a tile, two as long as the tiles are few enough then, else four: a digit of 16 K, 154 K and 480 K ids 8.8, 10.3 and 14.9 us with two,
// 10.9, 12.8 and 16.4 with four, of 900 K 17.2 with four, 28 with two that add up 440 tiles.
struct SortArgs {
  const void* ids;      // first digit: the ids
  int32_t id_bytes;
  int32_t shift, bits;
  int64_t num_rows;
  const int64_t* num;
  int64_t max_ids;
  const uint2* in;      // other digits: (row, token)
  uint2* out;
  uint16_t* hist;       // [tiles][bins]
  uint32_t* starts;     // [tiles][bins] records of a digit in the tiles before, if scanned
  uint32_t* totals;     // [bins] records of a digit, if scanned
  int32_t tiles;
  // rows of the whole table's gradient that the blocks behind the sort's own set to zero meanwhile, in units of 2 bytes
  uint32_t own_blocks;
  uint16_t* clear;
  int64_t clear_rows, clear_width, clear_stride;
};

// The sort leaves most of the chip idle and waits for memory, so part of the gradient is cleared beside each of its launches where most rows are
// untouched (see early_clear): 16 K tokens of 1024 columns into 50 K rows of floats 72.6 -> 69.0 us, 300 K of 64 into 2 M 172 -> 149 (with sums that
// took longer than now).  Of n blocks that clear, each has every n-th piece of blockDim vectors, or every n-th row where rows are apart.
__device__ __forceinline__ void clear_beside(const SortArgs& A) {
  typedef Elems<uint16_t, 8> Vector;
  const uint32_t block = blockIdx.x - A.own_blocks, blocks = gridDim.x - A.own_blocks;
  const bool whole = A.clear_stride == A.clear_width;  // one long row
  const int64_t rows = whole ? 1 : A.clear_rows, width = whole ? A.clear_width * A.clear_rows : A.clear_width;
  const int64_t step = static_cast<int64_t>(whole ? blocks : 1u) * blockDim.x, first = static_cast<int64_t>(whole ? block : 0u) * blockDim.x + threadIdx.x;
  for (int64_t r = whole ? 0 : block; r < rows; r += blocks) {
    uint16_t* row = A.clear + r * A.clear_stride;
    if (width >= 8) {
      for (int64_t i = first; i * 8 < width; i += step) *reinterpret_cast<Vector*>(row + (i * 8 + 8 <= width ? i * 8 : width - 8)) = {};
    } else {
      for (int64_t i = first; i < width; i += step) row[i] = 0;
    }
  }
}

constexpr int kSmallSort = 8192;
constexpr int kSmallTokens = 32;   // tokens of a block of k_sort_small

__device__ __forceinline__ uint2 sort_record(const SortArgs& A, int64_t i) {
  return A.in ? A.in[i] : make_uint2(row_of_id(A.ids, A.id_bytes, i, A.num_rows), static_cast<uint32_t>(i));
}

// Two lanes have a token, each half wave a share of the ids to compare with: four at a time, the same for all its lanes.  Two instructions a
// comparison: of equal ids those before the block's tokens count, those behind them do not, and only among its own it depends on the lane.
// 8192 ids 11.5 us, two digits in four launches 22.
constexpr int kSmallThreads = 512;
constexpr int kSmallShares = kSmallThreads / kSmallTokens;
template <typename Counts>
__device__ __forceinline__ uint32_t count_keys(const uint4* keys, int from, int to, int share, Counts counts) {
  uint32_t c = 0;
#pragma unroll 4
  for (int q = from + share; q < to; q += kSmallShares) {
    const uint4 k = keys[q];
    c += counts(k.x, 4 * q) ? 1u : 0u;
    c += counts(k.y, 4 * q + 1) ? 1u : 0u;
    c += counts(k.z, 4 * q + 2) ? 1u : 0u;
    c += counts(k.w, 4 * q + 3) ? 1u : 0u;
  }
  return c;
}
static __global__ void __launch_bounds__(kSmallThreads) k_sort_small(SortArgs A) {
  if (blockIdx.x >= A.own_blocks) return clear_beside(A);
  __shared__ uint4 keys[kSmallSort / 4];
  __shared__ uint32_t smaller[kSmallShares][kSmallTokens];
  const int n = static_cast<int>(count_of(A.num, A.max_ids));
  const int i0 = static_cast<int>(blockIdx.x) * kSmallTokens;
  if (i0 >= n) return;
  uint32_t* flat = reinterpret_cast<uint32_t*>(keys);
  const int padded = (n + 63) / 64 * 64;
#pragma unroll 8
  for (int i = threadIdx.x; i < padded; i += kSmallThreads) {
    const uint32_t key = row_of_id(A.ids, A.id_bytes, i < A.max_ids ? i : 0, A.num_rows);
    flat[i] = i < n ? key : ~0u;
  }
  __syncthreads();
  const int share = threadIdx.x / kSmallTokens, i = i0 + static_cast<int>(threadIdx.x) % kSmallTokens;
  const uint32_t key = flat[i];
  uint32_t count = count_keys(keys, 0, i0 / 4, share, [&](uint32_t k, int) { return k <= key; });
  count += count_keys(keys, i0 / 4, (i0 + kSmallTokens) / 4, share, [&](uint32_t k, int j) { return k < key || (k == key && j < i); });
  count += count_keys(keys, (i0 + kSmallTokens) / 4, padded / 4, share, [&](uint32_t k, int) { return k < key; });
  smaller[share][threadIdx.x % kSmallTokens] = count;
  __syncthreads();
  if (share != 0 || i >= n) return;
#pragma unroll
  for (int w = 1; w < kSmallShares; ++w) count += smaller[w][threadIdx.x];
  A.out[count] = make_uint2(key, static_cast<uint32_t>(i));
}

constexpr int kSortThreads = 1024;
constexpr int kSortWaves = kSortThreads / 64;
constexpr int kSortBits = 9;
constexpr int kSortBins = 1 << kSortBits;
constexpr int kSortColumns = 256;

template <int TURNS>
__global__ void __launch_bounds__(kSortThreads) k_sort_count(SortArgs A) {
  if (blockIdx.x >= A.own_blocks) return clear_beside(A);
  constexpr int kSortTurns = TURNS, kSortTile = kSortThreads * TURNS;
  __shared__ uint32_t count[kSortBins];
  const int64_t n = count_of(A.num, A.max_ids);
  const int bins = 1 << A.bits;
  const int64_t base = static_cast<int64_t>(blockIdx.x) * kSortTile;
  uint32_t digit[kSortTurns];
#pragma unroll
  for (int k = 0; k < kSortTurns; ++k) {
    const int64_t i = base + k * kSortThreads + threadIdx.x;
    digit[k] = (sort_record(A, i < A.max_ids ? i : A.max_ids - 1).x >> A.shift) & (bins - 1);
  }
  if (threadIdx.x < kSortBins) count[threadIdx.x] = 0;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kSortTurns; ++k)
    if (base + k * kSortThreads + threadIdx.x < n) atomicAdd(&count[digit[k]], 1u);
  __syncthreads();
  if (static_cast<int>(threadIdx.x) < bins)
    A.hist[static_cast<int64_t>(blockIdx.x) * bins + threadIdx.x] = static_cast<uint16_t>(count[threadIdx.x]);
}

// Records of every digit in the tiles before each, and in all of them: a block has kScanPairs pairs of digits, 64 groups of threads a range of the
// tiles each, whose counts are read once for their sum and once for the running one.
constexpr int kScanPairs = 16;
static __global__ void __launch_bounds__(kSortThreads) k_sort_scan(SortArgs A) {
  static_assert(kSortThreads / kScanPairs == 64, "the groups' sums are scanned by a wave");
  __shared__ uint32_t sums[64][2 * kScanPairs + 1];
  const int pairs = (1 << A.bits) / 2, pair = static_cast<int>(blockIdx.x) * kScanPairs + static_cast<int>(threadIdx.x) % kScanPairs;
  const int group = static_cast<int>(threadIdx.x) / kScanPairs, here = static_cast<int>(threadIdx.x) % kScanPairs;
  const int64_t each = (A.tiles + 63) / 64, from = group * each, to = from + each < A.tiles ? from + each : A.tiles;
  const uint32_t* hist = reinterpret_cast<const uint32_t*>(A.hist) + (pair < pairs ? pair : 0);
  uint32_t s0 = 0, s1 = 0;
#pragma unroll 8
  for (int64_t t = from; t < to; ++t) {
    const uint32_t c = hist[t * pairs];
    s0 += c & 0xFFFFu;
    s1 += c >> 16;
  }
  sums[group][2 * here] = s0;
  sums[group][2 * here + 1] = s1;
  __syncthreads();
  const int lane = threadIdx.x & 63;
  for (int d = threadIdx.x >> 6; d < 2 * kScanPairs; d += kSortWaves) {
    const uint32_t s = sums[lane][d], in = wave_inscan(s);
    sums[lane][d] = in - s;
    const int digit = static_cast<int>(blockIdx.x) * 2 * kScanPairs + d;
    if (lane == 63 && digit < 2 * pairs) A.totals[digit] = in;
  }
  __syncthreads();
  if (pair >= pairs) return;
  s0 = sums[group][2 * here];
  s1 = sums[group][2 * here + 1];
#pragma unroll 8
  for (int64_t t = from; t < to; ++t) {
    const uint32_t c = hist[t * pairs];
    reinterpret_cast<uint2*>(A.starts)[t * pairs + pair] = make_uint2(s0, s1);
    s0 += c & 0xFFFFu;
    s1 += c >> 16;
  }
}

template <int TURNS>
__global__ void __launch_bounds__(kSortThreads) k_sort_scatter(SortArgs A) {
  if (blockIdx.x >= A.own_blocks) return clear_beside(A);
  constexpr int kSortTurns = TURNS, kSortTile = kSortThreads * TURNS;
  __shared__ uint32_t next[kSortWaves][kSortBins];  // records of a wave so far, later where in the tile its next record goes
  __shared__ union {
    uint32_t sums[kSortWaves][2 * kSortBins];
    uint2 rec[kSortTile];                            // the tile's records, sorted by digit
  } s;
  __shared__ uint32_t shift_of[kSortBins];           // from the place in the tile to that among all records
  __shared__ unsigned long long lds[kSortWaves];
  const int bins = 1 << A.bits, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t base = static_cast<int64_t>(blockIdx.x) * kSortTile;
  // a wave has consecutive records, 64 a turn
  uint2 rec[kSortTurns];
#pragma unroll
  for (int k = 0; k < kSortTurns; ++k) {
    const int64_t i = base + (wave * kSortTurns + k) * 64 + lane;
    rec[k] = sort_record(A, i < A.max_ids ? i : A.max_ids - 1);
  }
  for (int i = threadIdx.x; i < kSortWaves * kSortBins; i += kSortThreads) next[0][i] = 0;
  const int64_t n = count_of(A.num, A.max_ids);
  if (base >= n) return;
  // where the tile's records of a digit begin: behind all smaller digits, and those of the tiles before; in pairs of digits, the tiles
  // dealt to groups of threads
  uint32_t at = 0, all = 0;
  const int pairs = bins / 2, groups = kSortThreads / pairs < kSortWaves ? kSortThreads / pairs : kSortWaves;
  if (!A.starts) {
    const int pair = static_cast<int>(threadIdx.x) % pairs, group = static_cast<int>(threadIdx.x) / pairs;
    if (group < groups) {
      uint32_t all0 = 0, all1 = 0, before0 = 0, before1 = 0;
      const int mine = static_cast<int>(blockIdx.x);
#pragma unroll 8
      for (int t = group; t < A.tiles; t += groups) {
        const uint32_t c = reinterpret_cast<const uint32_t*>(A.hist)[t * pairs + pair];
        all0 += c & 0xFFFFu;
        all1 += c >> 16;
        before0 += t < mine ? c & 0xFFFFu : 0u;
        before1 += t < mine ? c >> 16 : 0u;
      }
      s.sums[group][2 * pair] = all0;
      s.sums[group][2 * pair + 1] = all1;
      s.sums[group][kSortBins + 2 * pair] = before0;
      s.sums[group][kSortBins + 2 * pair + 1] = before1;
    }
  } else if (static_cast<int>(threadIdx.x) < bins) {
    at = A.starts[static_cast<int64_t>(blockIdx.x) * bins + threadIdx.x];
    all = A.totals[threadIdx.x];
  }
  __syncthreads();
  // its rank among equal digits of the wave
  uint32_t rank[kSortTurns];
#pragma unroll
  for (int k = 0; k < kSortTurns; ++k) {
    const bool live = base + (wave * kSortTurns + k) * 64 + lane < n;
    const uint32_t digit = (rec[k].x >> A.shift) & (bins - 1);
    const uint64_t lives = __ballot(live);
    uint32_t same0 = static_cast<uint32_t>(lives), same1 = static_cast<uint32_t>(lives >> 32);
#pragma unroll
    for (int b = 0; b < kSortBits; ++b) {  // a bit that no digit has changes nothing
      const uint64_t set = __ballot(digit & (1u << b));
      const uint32_t mine = static_cast<uint32_t>(__builtin_amdgcn_sbfe(static_cast<int>(digit), b, 1));
      same0 &= ~(static_cast<uint32_t>(set) ^ mine);
      same1 &= ~(static_cast<uint32_t>(set >> 32) ^ mine);
    }
    const uint32_t below = __builtin_amdgcn_mbcnt_hi(same1, __builtin_amdgcn_mbcnt_lo(same0, 0));
    uint32_t* slot = &next[wave][digit];
    rank[k] = *slot + below;  // every lane reads before the first of each digit adds
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (live && below == 0) *slot = rank[k] + __popc(same0) + __popc(same1);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
  __syncthreads();  // a digit's records are those of all waves
  if (!A.starts && static_cast<int>(threadIdx.x) < bins)
    for (int g = 0; g < groups; ++g) {
      all += s.sums[g][threadIdx.x];
      at += s.sums[g][kSortBins + threadIdx.x];
    }
  uint32_t mine = 0;
  if (static_cast<int>(threadIdx.x) < bins) {
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) mine += next[w][threadIdx.x];
  }
  unsigned long long total;
  const unsigned long long before = block_exscan<kSortThreads>(static_cast<unsigned long long>(all) << 32 | mine, lds, total);
  if (static_cast<int>(threadIdx.x) < bins) {
    uint32_t here = static_cast<uint32_t>(before);
    shift_of[threadIdx.x] = at + static_cast<uint32_t>(before >> 32) - here;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
      const uint32_t c = next[w][threadIdx.x];
      next[w][threadIdx.x] = here;
      here += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kSortTurns; ++k)
    if (base + (wave * kSortTurns + k) * 64 + lane < n) s.rec[next[wave][(rec[k].x >> A.shift) & (bins - 1)] + rank[k]] = rec[k];
  __syncthreads();
  // in the order of their digits, so that neighbours go to neighbouring places
  const int here = static_cast<int>(n - base < kSortTile ? n - base : kSortTile);
#pragma unroll
  for (int k = 0; k < kSortTurns; ++k) {
    const int i = k * kSortThreads + static_cast<int>(threadIdx.x);
    if (i < here) {
      const uint2 r = s.rec[i];
      A.out[shift_of[(r.x >> A.shift) & (bins - 1)] + static_cast<uint32_t>(i)] = r;
    }
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
// 480 K x 100 halfs into touched rows 41 us for 216 MB in lines of 128 bytes (5.2 TB/s, more than a copy); pieces of 8 and 32 tokens made that
// call 107 and 105 us where 16 made it 102, few ids often 108 and 76 instead of 84, 4096 ids of 1024 columns 20 and 26 instead of 22.
constexpr int kGradTokens = 16;
constexpr int kGradWaves = 8;
constexpr int kGradThreads = 64 * kGradWaves;
constexpr int kBlockTokens = kGradWaves * kGradTokens;
// Up to kTinyIds ids are the work of one block a tile of columns, of twice the waves, which sorts them itself: one launch instead of three, or
// of four for touched rows alone.
constexpr int kTinyIds = 256;
constexpr int kTinyThreads = 1024;
static_assert(kTinyThreads / 64 * kGradTokens == kTinyIds, "a piece a wave");
constexpr int kRunTile = 1024;     // a multiple of every block's tokens
constexpr int kScanTiles = 1024;   // more run tiles than that are scanned by a launch of their own
constexpr int grad_columns(int dim) { return dim <= 64 ? 1 : dim <= 128 ? 2 : 4; }

struct EmbedGradArgs {
  const void* ids;         // for up to kTinyIds of them
  int32_t id_bytes;
  const uint2* sorted;     // (row, token)
  const int64_t* num;
  int64_t max_ids;
  int64_t num_rows;
  int32_t dim;
  int32_t accumulate;
  const void* dy;
  int64_t dy_stride;
  float scale;
  uint32_t first_block;        // of the launch of k_embed_sums
  uint32_t sum_blocks, tiles;  // blocks of k_embed_sums that add up, and tiles of columns; the blocks behind all of them clear
  void* grad;
  int64_t grad_stride;
  float* part;             // [blocks][2][part_width]: head and tail
  int64_t part_width;
  int32_t clear_rows;      // rows of a block that clears
  // touched rows alone (row_ids != null): a run's row of `grad` is its rank
  int32_t direct;          // blocks count the runs before their own from the sorted tokens
  int32_t scanned;         // tile_runs holds its exclusive scan
  int32_t* row_ids;
  int64_t* num_unique;
  uint32_t* tile_runs;     // runs that begin in a tile of kRunTile sorted tokens
  uint32_t* block_runs;    // runs that begin in a block's tile before it
  uint32_t* tail_rank;     // rank of the run that begins in a block and goes on behind it
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

// A thread's share of the runs that begin before a block's tokens; all: of all runs, where the tiles are not scanned, for block 0.  Up to
// kDirectRuns ids need no k_embed_runs: their blocks look at all tokens before theirs (1000 ids of 32 floats 16.1 -> 13.5 us, 4000 of 128 the same with
// either, 8192 25.8 instead of 23.1).
constexpr int kDirectRuns = 2048;
__device__ __forceinline__ uint32_t share_of_runs(const EmbedGradArgs& A, uint32_t block, int64_t n, uint32_t& all) {
  const int64_t tile = static_cast<int64_t>(block) * kBlockTokens / kRunTile;
  all = 0;
  if (A.direct) {
    const int to = static_cast<int>(block == 0 ? n : static_cast<int64_t>(block) * kBlockTokens < n ? static_cast<int64_t>(block) * kBlockTokens : n);
    uint32_t runs = 0;
#pragma unroll 4
    for (int q = threadIdx.x; q < to; q += blockDim.x) {
      const uint32_t key = A.sorted[q].x, left = A.sorted[q > 0 ? q - 1 : 0].x;
      runs += key < A.num_rows && (q == 0 || left != key) ? 1u : 0u;
    }
    if (block == 0) all = runs;
    return block == 0 ? 0u : runs;
  }
  uint32_t x = threadIdx.x == 0 ? A.block_runs[block] : 0u;
  if (A.scanned) return threadIdx.x == 0 ? x + A.tile_runs[tile] : 0u;
  if (block == 0)
    for (int64_t t = threadIdx.x; t < A.run_tiles; t += blockDim.x) all += A.tile_runs[t];
  for (int64_t t = threadIdx.x; t < tile; t += blockDim.x) x += A.tile_runs[t];
  return x;
}

// V columns of a row of the gradient from their sum and, where it is added to, what they hold.  Columns that the vector before has as well are
// left to it where the row is added to, as that may be another block's; else both write the same, and a lane without columns the last ones again: no
// lane is masked (480 K x 100 halfs 47 -> 41 us).
template <typename TG, int V>
__device__ __forceinline__ TG* grad_at(const EmbedGradArgs& A, int64_t row, const Columns<V>& c) {
  return static_cast<TG*>(A.grad) + row * A.grad_stride + c.start;
}
template <typename TG, int V>
__device__ __forceinline__ void write_row(const EmbedGradArgs& A, int64_t row, const Columns<V>& c, const float (&sum)[V]) {
  Elems<TG, V> e;
#pragma unroll
  for (int j = 0; j < V; ++j) e.v[j] = from_float<TG>(A.scale * sum[j]);
  *reinterpret_cast<Elems<TG, V>*>(grad_at<TG, V>(A, row, c)) = e;
}
template <typename TG, int V>
__device__ __forceinline__ void add_to_row(const EmbedGradArgs& A, int64_t row, const Columns<V>& c, const float (&sum)[V], Elems<TG, V> e) {
  TG* g = grad_at<TG, V>(A, row, c);
#pragma unroll
  for (int j = 0; j < V; ++j) e.v[j] = from_float<TG>(as_float(e.v[j]) + A.scale * sum[j]);
  if (c.dup == 0) {
    *reinterpret_cast<Elems<TG, V>*>(g) = e;
  } else if (c.dup < V) {
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (j >= c.dup) g[j] = e.v[j];
  }
}
template <typename TG, int V>
__device__ __forceinline__ void write_grad(const EmbedGradArgs& A, int64_t row, const Columns<V>& c, const float (&sum)[V]) {
  if (A.accumulate) add_to_row<TG, V>(A, row, c, sum, *reinterpret_cast<const Elems<TG, V>*>(grad_at<TG, V>(A, row, c)));
  else write_row<TG, V>(A, row, c, sum);
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
__device__ __forceinline__ void clear_unnamed(const EmbedGradArgs& A, int64_t r0, int rows, const uint32_t* named) {
  const uint32_t per_row = static_cast<uint32_t>((A.dim + V - 1) / V);
  TG* g = static_cast<TG*>(A.grad) + r0 * A.grad_stride;
  for (uint32_t i = threadIdx.x; i < rows * per_row; i += blockDim.x) {
    const uint32_t r = i / per_row;
    if (!named[r]) *reinterpret_cast<Elems<TG, V>*>(g + r * A.grad_stride + Columns<V>(static_cast<int>(i - r * per_row), A.dim).start) = {};
  }
}
template <typename TG, bool TINY>
__device__ __forceinline__ void clear_rows(const EmbedGradArgs& A, int64_t n, uint32_t block, uint32_t* lds) {
  const int64_t r0 = static_cast<int64_t>(block) * A.clear_rows;
  const int rows = static_cast<int>(A.num_rows - r0 < A.clear_rows ? A.num_rows - r0 : A.clear_rows);
  if constexpr (TINY) {
    if (static_cast<int>(threadIdx.x) < rows) lds[threadIdx.x] = 0;
    __syncthreads();
    if (threadIdx.x < n) {
      const int64_t at = static_cast<int64_t>(row_of_id(A.ids, A.id_bytes, threadIdx.x, A.num_rows)) - r0;
      if (at >= 0 && at < rows) lds[at] = 1;
    }
  } else {
    const int64_t lo = wave_sorted_bound(A.sorted, 0, n, static_cast<uint32_t>(r0));
    const int64_t hi = wave_sorted_bound(A.sorted, lo, n, static_cast<uint32_t>(r0 + rows));
    if (static_cast<int>(threadIdx.x) < rows) {
      const uint32_t key = static_cast<uint32_t>(r0) + threadIdx.x;
      const int64_t p = sorted_bound(A.sorted, lo, hi, key);
      lds[threadIdx.x] = p < hi && A.sorted[p].x == key;
    }
  }
  __syncthreads();
  constexpr int V = 16 / sizeof(TG);
  if (A.dim >= V) clear_unnamed<TG, V>(A, r0, rows, lds);
  else clear_unnamed<TG, 1>(A, r0, rows, lds);
}

// The ids in sorted[1 ..], between two entries that stand for no row.  By the block: four threads a token compare its row with a quarter of the others each.
__device__ __forceinline__ void sort_tiny(const EmbedGradArgs& A, int n, uint2* sorted, uint4* quads, uint32_t (*smaller)[kTinyIds]) {
  uint32_t* keys = reinterpret_cast<uint32_t*>(quads);
  const uint32_t none = static_cast<uint32_t>(A.num_rows);
  const int i = threadIdx.x % kTinyIds, quarter = threadIdx.x / kTinyIds;
  if (quarter == 0) {
    const uint32_t key = row_of_id(A.ids, A.id_bytes, i < A.max_ids ? i : 0, A.num_rows);
    keys[i] = i < n ? key : none;
  }
  if (threadIdx.x == 0) sorted[0] = sorted[kTinyIds + 1] = make_uint2(none, 0);
  __syncthreads();
  const uint32_t key = keys[i];
  uint32_t count = 0;
  const auto belongs_before = [&](uint32_t k, int j) { return (k < key) | ((k == key) & (j < i)) ? 1u : 0u; };
#pragma unroll
  for (int q = 0; q < kTinyIds / 16; ++q) {
    const int at = quarter * (kTinyIds / 16) + q;
    const uint4 k = quads[at];
    count += belongs_before(k.x, 4 * at) + belongs_before(k.y, 4 * at + 1) + belongs_before(k.z, 4 * at + 2) + belongs_before(k.w, 4 * at + 3);
  }
  smaller[quarter][i] = count;
  __syncthreads();
  if (quarter == 0) sorted[1 + smaller[0][i] + smaller[1][i] + smaller[2][i] + smaller[3][i]] = make_uint2(key, i < n ? static_cast<uint32_t>(i) : 0u);
  __syncthreads();
}

// ADD: the sums are added to what the rows hold, which is asked for a few tokens ahead, whether a token ends a run or not: asked for only where
// one does, every row was waited for in turn.  (No other wave writes a row that a run of this one ends in.)
template <typename TD, typename TG, int V, bool TINY, bool ADD>
__global__ void __launch_bounds__(TINY ? kTinyThreads : kGradThreads) k_embed_sums(EmbedGradArgs A) {
  constexpr int kWaves = (TINY ? kTinyThreads : kGradThreads) / 64;
  __shared__ float heads[kWaves][64 * V];
  __shared__ uint32_t goes_on[kWaves];  // the wave's tokens are all of one run, that began before them and goes on behind them
  __shared__ uint32_t lds[kWaves * 64];
  const uint32_t number = A.first_block + blockIdx.x, tile = number / A.sum_blocks, block = number - tile * A.sum_blocks;
  const int64_t n = count_of(A.num, A.max_ids);
  if (tile >= A.tiles) {
    clear_rows<TG, TINY>(A, n, number - A.sum_blocks * A.tiles, lds);
    return;
  }
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t b0 = static_cast<int64_t>(block) * kBlockTokens, p0 = b0 + wave * kGradTokens;
  const uint32_t none = static_cast<uint32_t>(A.num_rows);
  const int index = static_cast<int>(tile) * 64 + lane;
  const Columns<V> c(index, A.dim);
  // the wave's tokens, one to a lane, from lane 1 on; lane 0 has the one before, lane kGradTokens + 1 the one behind
  uint2 mine;
  uint32_t share = 0, all = 0;
  if constexpr (TINY) {
    __shared__ uint2 sorted[kTinyIds + 2];
    __shared__ uint4 keys[kTinyIds / 4];
    __shared__ uint32_t smaller[4][kTinyIds];
    sort_tiny(A, static_cast<int>(n), sorted, keys, smaller);
    mine = lane <= kGradTokens + 1 ? sorted[wave * kGradTokens + lane] : make_uint2(none, 0);
  } else {
    const int64_t at = p0 - 1 + lane;
    mine = A.sorted[at < 0 ? 0 : at < A.max_ids ? at : A.max_ids - 1];
    if (lane > kGradTokens + 1 || at < 0 || at >= n) mine = make_uint2(none, 0);
    if (A.row_ids) share = share_of_runs(A, block, n, all);
  }
  // Every row is read, also a padded place's and for columns that there are not (the last ones again), and dropped later: loads under a
  // condition are waited for one by one.  Token 0 stands for those behind the last.
  const TD* dy = static_cast<const TD*>(A.dy);
  Elems<TD, V> e[kGradTokens];
#pragma unroll
  for (int u = 0; u < kGradTokens; ++u) {
    const uint32_t token = __builtin_amdgcn_readlane(mine.y, u + 1);
    e[u] = *reinterpret_cast<const Elems<TD, V>*>(dy + token * A.dy_stride + c.start);
  }
  uint32_t rank = 0;  // of the next run that begins; the same in all lanes, and in a scalar register
  if (A.row_ids) {
    const uint32_t left = __shfl_up(mine.x, 1, 64);  // by all lanes: not in the condition
    const bool begins = lane >= 1 && lane <= kGradTokens && mine.x < none && mine.x != left;
    const uint64_t set = __ballot(begins);
    if constexpr (!TINY) {
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        share += __shfl_xor(share, o, 64);
        if (block == 0) all += __shfl_xor(all, o, 64);
      }
    }
    if (lane == 0) {
      lds[wave] = share;
      lds[kWaves + wave] = TINY ? __popcll(set) : all;
      lds[2 * kWaves + wave] = __popcll(set);
    }
    __syncthreads();
    share = all = 0;
    for (int w = 0; w < kWaves; ++w) {
      share += lds[w] + (w < wave ? lds[2 * kWaves + w] : 0u);
      all += lds[kWaves + w];
    }
    rank = __builtin_amdgcn_readfirstlane(share);
    if (number == 0 && threadIdx.x == 0 && (TINY || !A.scanned)) *A.num_unique = all;
    if (begins && tile == 0) A.row_ids[rank + __popcll(set & ((1ull << lane) - 1))] = static_cast<int32_t>(mine.x);
  }
  if (b0 >= n) return;
  const uint32_t before = __builtin_amdgcn_readlane(mine.x, 0), first = __builtin_amdgcn_readlane(mine.x, 1);
  const uint32_t key = __builtin_amdgcn_readlane(mine.x, kGradTokens), behind = __builtin_amdgcn_readlane(mine.x, kGradTokens + 1);
  const bool began_before = first < none && first == before, open = key < none && key == behind;
  bool head = began_before;
  float sum[V] = {};
  constexpr int kAhead = kGradTokens / V;  // 16 registers of rows that are added to
  Elems<TG, V> held[ADD ? kAhead : 1];
#pragma unroll
  for (int u = 0; u < kGradTokens; ++u) {
    if constexpr (ADD) {
      if (u % kAhead == 0) {
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
          const uint32_t row = __builtin_amdgcn_readlane(mine.x, u + q + 1);
          held[q] = *reinterpret_cast<const Elems<TG, V>*>(grad_at<TG, V>(A, row < none ? row : 0u, c));
        }
      }
    }
#pragma unroll
    for (int j = 0; j < V; ++j) sum[j] += as_float(e[u].v[j]);
    const uint32_t here = __builtin_amdgcn_readlane(mine.x, u + 1), next = __builtin_amdgcn_readlane(mine.x, u + 2);
    if (here == next) continue;  // the run goes on
    if (here < none) {
      if (head) {
#pragma unroll
        for (int j = 0; j < V; ++j) heads[wave][j * 64 + lane] = sum[j];
      } else {
        const int64_t row = A.row_ids ? static_cast<int64_t>(rank++) : static_cast<int64_t>(here);
        if constexpr (ADD) add_to_row<TG, V>(A, row, c, sum, held[u % kAhead]);
        else write_row<TG, V>(A, row, c, sum);
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
    for (; w < kWaves; ++w) {
#pragma unroll
      for (int j = 0; j < V; ++j) sum[j] += heads[w][j * 64 + lane];
      if (!goes_on[w]) break;
    }
    if (w < kWaves) {
      write_grad<TG, V>(A, A.row_ids ? static_cast<int64_t>(rank) : static_cast<int64_t>(key), c, sum);
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) part[A.part_width + j] = sum[j];
      if (A.row_ids && index == 0) A.tail_rank[block] = rank;
    }
  }
  // the run that began before the block
  if (wave == 0 && began_before) {
#pragma unroll
    for (int j = 0; j < V; ++j) sum[j] = heads[0][j * 64 + lane];
    for (int w = 0; w + 1 < kWaves && goes_on[w]; ++w) {
#pragma unroll
      for (int j = 0; j < V; ++j) sum[j] += heads[w + 1][j * 64 + lane];
    }
#pragma unroll
    for (int j = 0; j < V; ++j) part[j] = sum[j];
  }
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
    const int64_t row = A.row_ids ? static_cast<int64_t>(A.tail_rank[b]) : static_cast<int64_t>(key);
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
  // the block it begins in: as many before m as end with the run; the last block that begins with it
  const int64_t p = (m - lane) * kBlockTokens - 1;
  const int64_t b = m - __popcll(__ballot(lane <= kJoinShort && p >= 0 && A.sorted[p < 0 ? 0 : p].x == key));
  int64_t last = m;
  for (int64_t step = 1, hi = (n - 1) / kBlockTokens; last < hi;) {  // it is in [last, hi]
    step = (hi - last + 63) / 64;
    const int64_t q = last + (lane + 1) * step;
    const int more = __popcll(__ballot(q <= hi && A.sorted[(q <= hi ? q : hi) * kBlockTokens].x == key));
    last += more * step;
    hi = last + step - 1 < hi ? last + step - 1 : hi;
  }
  if (m - b > kJoinShort || last - b < kJoinShort) return;
  const int64_t row = A.row_ids ? static_cast<int64_t>(A.tail_rank[b]) : static_cast<int64_t>(key);
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
