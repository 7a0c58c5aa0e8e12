// Rows of an embedding by token id, and the gradient of the embedding: for every token the sum of its rows' gradients.
//
// The gradient of up to 1024 rows compares all ids with one another.  Otherwise it sorts (id, row) pairs by id, rows of one id staying in order, and then walks the sorted pairs in pieces of
// equal length, whatever the ids: a token that makes up a tenth of the batch is shared by many workgroups like any other rows.  A run of equal ids inside a piece is summed and written by
// its workgroup; of one that crosses pieces each leaves its part, and a second kernel adds the parts in order.
//
// Bound by HBM.  The lookup of 16381 rows of 4096 in bf16, 268 MB (of which text repeats some), 34 us.  The gradient of 20483 such rows into a vocabulary of 151936, of which 2.49 GB
// are written and 0.17 read, 450 us, 5.9 TB/s: zeros and ranks 356, merging 9, sums 81 (they write their rows again), joining 6; of 2897 rows of 1024 in fp32 into 32000, 143 MB that the Infinity
// Cache holds, 28 us: ranks and zeros 19.2, sums 6.5, joining 3.8.  Added to a gradient that is there (tied weights), the first 120 us: 0.44 GB, rows once and the 8422 ids' rows of the gradient twice.
#include "nat_internal.h"
#include "mfma_tile.hip.h"

#include <type_traits>

namespace nat {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float bf16_to_f32(uint32_t bits) { return __builtin_bit_cast(float, bits << 16); }

// 16 bytes of a row: 8 elements of bf16, 4 of f32
template <typename T> struct Piece;
template <>
struct Piece<uint16_t> {
  static constexpr int kElements = 8;
  __device__ __forceinline__ static void add(float (&acc)[8], u32x4 x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      acc[2 * i] += bf16_to_f32(x[i] & 0xffff);
      acc[2 * i + 1] += bf16_to_f32(x[i] >> 16);
    }
  }
  __device__ __forceinline__ static u32x4 scaled(u32x4 x, float s) {
    bf16x8 y;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      y[2 * i] = (__bf16)(bf16_to_f32(x[i] & 0xffff) * s);
      y[2 * i + 1] = (__bf16)(bf16_to_f32(x[i] >> 16) * s);
    }
    return __builtin_bit_cast(u32x4, y);
  }
};
template <>
struct Piece<float> {
  static constexpr int kElements = 4;
  __device__ __forceinline__ static void add(float (&acc)[4], u32x4 x) {
    const f32x4 y = __builtin_bit_cast(f32x4, x);
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] += y[i];
  }
  __device__ __forceinline__ static u32x4 scaled(u32x4 x, float s) { return __builtin_bit_cast(u32x4, __builtin_bit_cast(f32x4, x) * s); }
};

struct EmbedArgs {
  const int32_t* ids;
  const char* E;
  char* out;
  int64_t n_rows, row_bytes, out_bytes, first;      // first: the row that the launch begins with
  int32_t V;
  int lanes_log2;                                   // lanes per row
  float scale;
};

template <typename T>
__global__ void __launch_bounds__(256) embed_kernel(EmbedArgs a) {
  const int64_t row = a.first + (((int64_t)blockIdx.x * 256 + threadIdx.x) >> a.lanes_log2);
  if (row >= a.n_rows) return;
  const int lanes = 1 << a.lanes_log2, id = a.ids[row];
  const bool there = (uint32_t)id < (uint32_t)a.V;
  const char* from = a.E + (there ? id : 0) * a.row_bytes;
  char* to = a.out + row * a.out_bytes;
#pragma unroll 2
  for (int64_t at = (int64_t)(threadIdx.x & (lanes - 1)) * 16; at < a.row_bytes; at += (int64_t)lanes * 16) {
    u32x4 x = {0, 0, 0, 0};
    if (there) x = Piece<T>::scaled(*(const u32x4*)(from + at), a.scale);
    *(u32x4*)(to + at) = x;
  }
}

// ------------------------------------------------------------------ the sort ----
struct SortArgs {
  const int32_t *ids_in, *rows_in;      // rows_in NULL: the first pass, ids as the caller has them
  int32_t *ids_out, *rows_out, *counts;
  int64_t n;
  int32_t V;
  int shift, bits, tiles;
  bool scanned;                         // counts hold places
  unsigned blocks;                      // the workgroups behind these write zeros
  f32x4* zeros;
  int64_t chunks;                       // of 16 bytes
};

// Zeros into the whole gradient, before the sums write the rows that have pairs.  Into the other rows alone, found in the sorted ids beside the sums, there are fewer, but short rows cost
// more to look for than to write: 300000 pairs over 152064 ids, all of them random, 225 us at 128 elements (1000000 pairs) and 454, 234 and 301 at 512, 393 and 391 at 1024; long ones,
// where so many random pairs leave few rows out, are slower by up to 8 percent (64000 pairs of 4096 over 32000 ids 319 us and 294).
//
// A gradient that the Infinity Cache holds for the most part: by workgroups of the sort's first launch, which leaves most of the chip idle.  2897 rows into 131 MB 28.6 us in all; beside
// the sums, and only into the rows that no pair has, 32.1.
__device__ __forceinline__ bool zero_block(const SortArgs& a) {
  if (blockIdx.x < a.blocks) return false;
  const int64_t i = (int64_t)(blockIdx.x - a.blocks) * blockDim.x + threadIdx.x;
  if (i < a.chunks) a.zeros[i] = f32x4{};
  return true;
}

__device__ __forceinline__ int32_t key_of(int32_t id, int32_t V) { return (uint32_t)id < (uint32_t)V ? id : V; }

// Up to kRanked pairs: a pair's place is the number of pairs before it, counted outright, two instructions each.  A workgroup takes 16 pairs, each in four lanes of all its
// wavefronts, which share the others in blocks of 64.  2897 pairs 5.3 us; sorted by digits in one workgroup they took 18.  Up to kMerged pairs are ranked in tiles of kMergeTile
// first, 64 of them to a workgroup, which merge_kernel then joins.
constexpr int kRanked = 8192, kRankWaves = 16, kRankPairs = 16, kTilePairs = 64;
constexpr int kMergeTile = 4096, kMerged = 32768;
constexpr int kBlock = 64, kBlockPitch = kBlock + 4;       // four lanes' blocks in different banks
template <int kPairs, int kMost, int W>
__global__ void __launch_bounds__(64 * W) rank_kernel(SortArgs a) {
  typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
  constexpr int kLanes = 64 / kPairs;                      // of a pair
  __shared__ __attribute__((aligned(16))) int32_t keys[kMost / kBlock * kBlockPitch];
  __shared__ int counts[W][kPairs];
  if (zero_block(a)) return;
  const int base = (int)(blockIdx.x / (kMost / kPairs)) * kMost;       // of the tile
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = a.n - base < kMost ? (int)a.n - base : kMost, blocks = (n + kBlock - 1) / kBlock;
  for (int i = threadIdx.x; i < kBlock * blocks; i += 64 * W)
    keys[i / kBlock * kBlockPitch + i % kBlock] = i < n ? key_of(a.ids_in[base + i], a.V) : INT32_MAX;
  __syncthreads();
  const int mine = (int)(blockIdx.x % (kMost / kPairs)) * kPairs + lane % kPairs, own = mine / kBlock, it = own < blocks ? keys[own * kBlockPitch + mine % kBlock] : 0;
  const int key = it < INT32_MAX ? it : 0;                 // (what a place without a pair counts is not used)
  int before = 0;
  for (int b = wave * kLanes + lane / kPairs; b < blocks; b += kLanes * W) {
    const int32_t* block = keys + b * kBlockPitch;
    // keys that are not there are never below; of the own block those before this pair may be equal
    if (b != own) {
      const int limit = b < own ? key + 1 : key;
#pragma unroll
      for (int j = 0; j < kBlock; j += 4) {
        const i32x4 x = *(const i32x4*)(block + j);
#pragma unroll
        for (int u = 0; u < 4; ++u) before += x[u] < limit;
      }
    } else {
      const int at = mine % kBlock;
#pragma unroll 2
      for (int j = 0; j < kBlock; j += 4) {            // (unrolled all the way the limits of all places are kept in registers)
        const i32x4 x = *(const i32x4*)(block + j);
#pragma unroll
        for (int u = 0; u < 4; ++u) before += x[u] < key + (j + u < at);
      }
    }
  }
#pragma unroll
  for (int d = kPairs; d < 64; d <<= 1) before += __shfl_xor(before, d, 64);
  if (lane < kPairs) counts[wave][lane] = before;
  __syncthreads();
  if (threadIdx.x >= kPairs || mine >= n) return;
  before = 0;
#pragma unroll
  for (int w = 0; w < W; ++w) before += counts[w][lane];
  a.ids_out[base + before] = key;
  a.rows_out[base + before] = base + mine;
}

// Sorted tiles into one: a pair's place is its place in its tile and, of each other tile, the number of pairs before it, which a search in LDS finds.  20483 pairs 7.6 us and
// 12.9 for the ranks in the tiles; two passes by digits took 29.
__global__ void __launch_bounds__(1024) merge_kernel(SortArgs a) {
  typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
  extern __shared__ __attribute__((aligned(16))) int32_t keys[];
  const int n = (int)a.n;
  for (int i0 = 4 * threadIdx.x; i0 < n; i0 += 16384) {    // (the array is 256-byte aligned and has room for whole 16 bytes)
    i32x4 x[4];
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (i0 + 4096 * u < n) x[u] = *(const i32x4*)(a.ids_in + i0 + 4096 * u);
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (i0 + 4096 * u < n) *(i32x4*)(keys + i0 + 4096 * u) = x[u];
  }
  __syncthreads();
  const int i = blockIdx.x * 1024 + (int)threadIdx.x;
  if (i >= n) return;
  const int key = keys[i], tiles = (n + kMergeTile - 1) / kMergeTile, own = i / kMergeTile;
  int place = i - own * kMergeTile;
  for (int t = 0; t < tiles; ++t) {
    if (t == own) continue;
    const int32_t* tile = keys + t * kMergeTile;
    const int limit = t < own ? key + 1 : key;             // equal ones of tiles before are before
    int at = 0, len = n - t * kMergeTile < kMergeTile ? n - t * kMergeTile : kMergeTile;
    while (len > 0) {
      const int half = len >> 1;
      const bool below = tile[at + half] < limit;
      at = below ? at + half + 1 : at;
      len = below ? len - half - 1 : half;
    }
    place += at;
  }
  a.ids_out[place] = key;
  a.rows_out[place] = a.rows_in[i];
}

// More pairs: by digits from the lowest on, each pass stable.  A workgroup of W wavefronts takes a tile of 64 W kPer pairs, each wavefront ranking 64 at a time by
// ballots over the digit's bits.
constexpr int kMostBits = 9, kMostBins = 1 << kMostBits;
constexpr int kPer = 4;                                    // pairs per thread
constexpr int kFewWaves = 4, kManyWaves = 16;              // of a tile: few, for the time that one takes; many for few tiles
constexpr int kDirectTiles = 64;                           // up to so many tiles, each adds up the counts of those before it by itself

// Exclusive prefix sum over the workgroup
template <int W>
__device__ __forceinline__ int block_scan(int x, int* wave_sums) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int sum = x;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int y = __shfl_up(sum, d, 64);
    if (lane >= d) sum += y;
  }
  if (lane == 63) wave_sums[wave] = sum;
  __syncthreads();
  int before = 0;
#pragma unroll
  for (int w = 0; w < W; ++w) before += w < wave ? wave_sums[w] : 0;
  __syncthreads();
  return before + sum - x;
}

template <int W>
struct SortShared {
  int counts[W][kMostBins];               // of a wavefront and digit; then the place of its first pair
  int wave_sums[W];
};

// place[e]: where pair e of this thread (number wave * 64 * kPer + 64 e + lane of the tile) lies in the tile sorted by its digit
template <int W>
__device__ __forceinline__ void rank_tile(SortShared<W>& s, const int (&digit)[kPer], int bits, int (&place)[kPer]) {
  constexpr int kThreads = 64 * W;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, bins = 1 << bits;
  for (int i = threadIdx.x; i < W * bins; i += kThreads) s.counts[i >> bits][i & (bins - 1)] = 0;
  __syncthreads();
  volatile int* mine = s.counts[wave];
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    uint64_t same = ~uint64_t{0};
    for (int b = 0; b < bits; ++b) {
      const bool set = (digit[e] >> b) & 1;
      const uint64_t with = __ballot(set);
      same &= set ? with : ~with;
    }
    const int before = mine[digit[e]];
    place[e] = before + __popcll(same & ((uint64_t{1} << lane) - 1));
    __builtin_amdgcn_wave_barrier();
    if ((same >> lane) == 1) mine[digit[e]] = before + __popcll(same);       // the last of them
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
  __syncthreads();
  // digits in order, of each the wavefronts in order: some entries per thread, or threads without any
  const int total = bins * W, per = total > kThreads ? total / kThreads : 1, first = threadIdx.x * per;
  int sum = 0;
  for (int i = first; i < first + per && i < total; ++i) sum += s.counts[i % W][i / W];
  sum = block_scan<W>(sum, s.wave_sums);
  for (int i = first; i < first + per && i < total; ++i) {
    const int n = s.counts[i % W][i / W];
    s.counts[i % W][i / W] = sum;
    sum += n;
  }
  __syncthreads();
#pragma unroll
  for (int e = 0; e < kPer; ++e) place[e] += s.counts[wave][digit[e]];
}

// counts[bin][tile] for the scan, else counts[tile][bin]
template <int W>
__global__ void __launch_bounds__(64 * W) sort_count_kernel(SortArgs a) {
  constexpr int kThreads = 64 * W;
  __shared__ int bins[kMostBins];
  if (zero_block(a)) return;
  const int n_bins = 1 << a.bits;
  for (int i = threadIdx.x; i < n_bins; i += kThreads) bins[i] = 0;
  __syncthreads();
  const int64_t first = (int64_t)blockIdx.x * kThreads * kPer;
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    const int64_t i = first + e * kThreads + threadIdx.x;
    if (i < a.n) atomicAdd(&bins[(key_of(a.ids_in[i], a.V) >> a.shift) & (n_bins - 1)], 1);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n_bins; i += kThreads) a.counts[a.scanned ? (int64_t)i * a.tiles + blockIdx.x : (int64_t)blockIdx.x * n_bins + i] = bins[i];
}

// counts[bin][tile] -> those of the tiles before, and behind them all tiles' of the bin, in counts[bins * tiles + bin]
__global__ void __launch_bounds__(64 * kManyWaves) sort_scan_kernel(SortArgs a) {
  constexpr int kThreads = 64 * kManyWaves;
  __shared__ int wave_sums[kManyWaves], all;
  int32_t* of = a.counts + (int64_t)blockIdx.x * a.tiles;
  int before = 0;
  for (int first = 0; first < a.tiles; first += kThreads) {
    const int i = first + (int)threadIdx.x, x = i < a.tiles ? of[i] : 0;
    const int sum = block_scan<kManyWaves>(x, wave_sums);
    if (i < a.tiles) of[i] = before + sum;
    if (threadIdx.x == kThreads - 1) all = sum + x;
    __syncthreads();
    before += all;
    __syncthreads();
  }
  if (threadIdx.x == 0) a.counts[((int64_t)a.tiles << a.bits) + blockIdx.x] = before;
}

template <int W>
__global__ void __launch_bounds__(64 * W) sort_scatter_kernel(SortArgs a) {
  constexpr int kThreads = 64 * W, kTile = kThreads * kPer, kBins = (kMostBins + kThreads - 1) / kThreads;
  __shared__ SortShared<W> s;
  __shared__ int to[kMostBins];           // place of the tile's first pair of a digit, minus its place inside the tile
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n_bins = 1 << a.bits, tile = blockIdx.x;
  // the thread's digits kBins * thread, ...: pairs of these in all tiles, and in those before this one
  int all[kBins] = {}, before[kBins] = {}, sum = 0;
#pragma unroll
  for (int b = 0; b < kBins; ++b) {
    const int bin = (int)threadIdx.x * kBins + b;
    if (bin >= n_bins) continue;
    if (a.scanned) {
      before[b] = a.counts[(int64_t)bin * a.tiles + tile];
      all[b] = a.counts[((int64_t)a.tiles << a.bits) + bin];
    } else {
      for (int t0 = 0; t0 < a.tiles; t0 += 16) {            // (in a row they would be a chain of loads)
        int x[16];
#pragma unroll
        for (int u = 0; u < 16; ++u) x[u] = t0 + u < a.tiles ? a.counts[(t0 + u) * n_bins + bin] : 0;
#pragma unroll
        for (int u = 0; u < 16; ++u) {
          all[b] += x[u];
          before[b] += t0 + u < tile ? x[u] : 0;
        }
      }
    }
    sum += all[b];
  }
  sum = block_scan<W>(sum, s.wave_sums);
  int key[kPer], row[kPer], digit[kPer], place[kPer];
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    const int64_t i = (int64_t)tile * kTile + wave * 64 * kPer + 64 * e + lane;
    key[e] = i < a.n ? key_of(a.ids_in[i], a.V) : INT32_MAX;             // behind all others, in every pass
    row[e] = i < a.n ? a.rows_in ? a.rows_in[i] : (int32_t)i : -1;
    digit[e] = (key[e] >> a.shift) & (n_bins - 1);
  }
  rank_tile<W>(s, digit, a.bits, place);
#pragma unroll
  for (int b = 0; b < kBins; ++b) {
    const int bin = (int)threadIdx.x * kBins + b;
    if (bin < n_bins) to[bin] = sum + before[b] - s.counts[0][bin];
    sum += all[b];
  }
  __syncthreads();
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    if (row[e] < 0) continue;
    const int at = to[digit[e]] + place[e];
    a.ids_out[at] = key[e];
    a.rows_out[at] = row[e];
  }
}

// ------------------------------------------------------------------ the sums ----
struct SumArgs {
  const int32_t *ids, *rows;            // sorted
  const char* dout;
  float *dE, *part;                     // part: [pieces][2][H], of the run that came in from the piece before, of the one that goes on behind
  int64_t n, dout_bytes;
  int32_t V, H;
  int piece, slabs;                     // pairs per piece, at most 64; workgroups per row
  float scale;
  int accumulate;
};

template <typename T>
__device__ __forceinline__ void write_run(const SumArgs& a, int32_t id, int at, const float (&acc)[Piece<T>::kElements]) {
  float* to = a.dE + (int64_t)id * a.H + at;
#pragma unroll
  for (int i = 0; i < Piece<T>::kElements; i += 4) {
    f32x4 x = f32x4{acc[i], acc[i + 1], acc[i + 2], acc[i + 3]} * a.scale;
    if (a.accumulate) x += *(const f32x4*)(to + i);
    *(f32x4*)(to + i) = x;
  }
}

// Rows are read past the caches, which hold what is written (20483 of 4096 into 151936, then, in all 456 us, otherwise 471; 20000 into 20000 122 and 148, and 197 and 211 between the launches that
// write the rows and read the sums).
template <typename T>
__global__ void __launch_bounds__(256) embed_sum_kernel(SumArgs a) {
  constexpr int kE = Piece<T>::kElements, kAhead = 8;
  const int slab = blockIdx.x % a.slabs, lane = threadIdx.x & 63;
  const int64_t piece = blockIdx.x / a.slabs, p0 = piece * a.piece;
  const int count = p0 + a.piece < a.n ? a.piece : (int)(a.n - p0), at = (slab * (int)blockDim.x + (int)threadIdx.x) * kE;
  // the piece's pairs, one per lane, and the ids beside it
  const int64_t p = p0 + (lane < count ? lane : count - 1);
  const int ids = a.ids[p], rows = a.rows[p];
  const int first = __builtin_amdgcn_readfirstlane(ids);
  const bool from_before = p0 > 0 && a.ids[p0 - 1] == first, goes_on = p0 + count < a.n && a.ids[p0 + count] == __builtin_amdgcn_readlane(ids, count - 1);
  const bool there = at < a.H;          // (all lanes stay: others read theirs)
  const char* from = a.dout + (there ? at : 0) * (int64_t)sizeof(T);
  float acc[kE] = {};
  bool first_run = true;
  for (int j0 = 0; j0 < count; j0 += kAhead) {
    u32x4 x[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (j0 + u < count) x[u] = __builtin_nontemporal_load((const u32x4*)(from + __builtin_amdgcn_readlane(rows, j0 + u) * a.dout_bytes));
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int j = j0 + u;
      if (j >= count) continue;
      Piece<T>::add(acc, x[u]);
      const int id = __builtin_amdgcn_readlane(ids, j);
      const bool last = j + 1 == count;
      if (!last && __builtin_amdgcn_readlane(ids, j + 1) == id) continue;
      if (id < a.V && there) {
        const int side = first_run && from_before ? 0 : last && goes_on ? 1 : -1;
        if (side < 0) {
          write_run<T>(a, id, at, acc);
        } else {
          float* to = a.part + (piece * 2 + side) * a.H + at;
#pragma unroll
          for (int i = 0; i < kE; i += 4) *(f32x4*)(to + i) = f32x4{acc[i], acc[i + 1], acc[i + 2], acc[i + 3]};
        }
      }
      first_run = false;
#pragma unroll
      for (int i = 0; i < kE; ++i) acc[i] = 0.f;
    }
  }
}

// The parts of a run that begins in this piece and goes on behind it: the workgroup's groups of `threads` take every so many parts, eight loads ahead, without a branch around them (a
// place that is not there is the last one's, and not added), and the first group adds up theirs in order.  6000 pairs of 1024 with two ids 50 us in all, by one group of 256 threads and 16
// loads ahead 76; 20000 of 128 with 50 ids 31 and 43.
constexpr int kJoinThreads = 512;
template <typename T>
__global__ void __launch_bounds__(kJoinThreads) embed_join_kernel(SumArgs a, int threads) {
  constexpr int kE = Piece<T>::kElements, kAhead = 8;
  __shared__ __attribute__((aligned(16))) float sums[kJoinThreads * kE];
  const int slab = blockIdx.x % a.slabs, lane = threadIdx.x & 63;
  const int64_t piece = blockIdx.x / a.slabs, p0 = piece * a.piece, p1 = p0 + a.piece;
  if (p1 >= a.n) return;
  const int32_t id = a.ids[p1], behind = a.ids[p1 - 1], first = a.ids[p0], before = a.ids[p0 > 0 ? p0 - 1 : 0];
  if (id >= a.V || behind != id || (first == id && p0 > 0 && before == id)) return;
  const int group = threadIdx.x / threads, groups = blockDim.x / threads, thread = threadIdx.x - group * threads;
  const int at = (slab * threads + thread) * kE;
  const bool there = at < a.H;
  float acc[kE] = {};
  if (there && group == 0) {
    const float* from = a.part + (piece * 2 + 1) * a.H + at;
#pragma unroll
    for (int i = 0; i < kE; ++i) acc[i] = from[i];
  }
  // 64 pieces at a time: those that begin with the run
  for (int64_t c0 = piece + 1;; c0 += 64) {
    const int64_t q = (c0 + lane) * a.piece;
    const uint64_t with = __ballot(q < a.n && a.ids[q < a.n ? q : 0] == id);
    const int parts = with == ~uint64_t{0} ? 64 : __builtin_ctzll(~with);
    if (there) {
      const float* from = a.part + c0 * 2 * a.H + at;
      for (int c = group * kAhead; c < parts; c += groups * kAhead) {
        f32x4 x[kAhead][kE / 4];
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
#pragma unroll
          for (int i = 0; i < kE / 4; ++i)
            x[u][i] = *(const f32x4*)(from + (c + u < parts ? c + u : parts - 1) * (int64_t)2 * a.H + 4 * i);
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
#pragma unroll
          for (int i = 0; i < kE; ++i) acc[i] += c + u < parts ? x[u][i >> 2][i & 3] : 0.f;
      }
    }
    if (parts < 64) break;
  }
#pragma unroll
  for (int i = 0; i < kE; ++i) sums[threadIdx.x * kE + i] = acc[i];
  __syncthreads();
  if (group || !there) return;
  for (int g = 1; g < groups; ++g)
#pragma unroll
    for (int i = 0; i < kE; ++i) acc[i] += sums[(g * threads + thread) * kE + i];
  write_run<T>(a, id, at, acc);
}

// Up to kFew pairs in one launch, without a sort: a workgroup per pair and 64 lanes, which compares its id with all of them, a wavefront with a quarter, and ends unless its pair is the
// id's first.  Each wavefront adds up those of its quarter, the first wavefront their sums in order.
//
// Zeros by other workgroups, kFewSteps 16 bytes per thread, into the rows that no pair has, or none (chunks 0).  As each reads all ids, many pairs and many zeros are left to the sort:
// 200 pairs over 131 MB 19 us, by the sort 26; 500 19.6 and 26; 1024 over 262 MB 45 and 42.  1000 pairs of 1024 over 8 MB 10.3 us and 15.5, of which the host takes ten.
constexpr int kFew = 1024, kFewSteps = 4;
constexpr int64_t kFewWork = int64_t{1} << 33;             // pairs times 16 bytes
struct FewArgs : SumArgs {
  unsigned sum_blocks;
  int64_t chunks;                       // of 16 bytes
};
template <typename T>
__global__ void __launch_bounds__(256) embed_few_kernel(FewArgs a) {
  constexpr int kE = Piece<T>::kElements, kAhead = 8;
  if (blockIdx.x >= a.sum_blocks) {
    __shared__ uint32_t used[256 * kFewSteps / 32 + 1];    // a row has 16 bytes or more
    const int64_t first = (int64_t)(blockIdx.x - a.sum_blocks) * 256 * kFewSteps;
    const int row = a.H / 4, v0 = (int)(first / row);
    const uint32_t rest = (uint32_t)(first - (int64_t)v0 * row);
    for (int i = threadIdx.x; i < 256 * kFewSteps / 32 + 1; i += 256) used[i] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < a.n; i += 256) {
      const int64_t r = (int64_t)a.ids[i] - v0;
      if (r >= 0 && r <= 256 * kFewSteps) atomicOr(&used[r >> 5], 1u << (r & 31));
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kFewSteps; ++u) {
      const uint32_t at = u * 256 + threadIdx.x, r = (rest + at) / (uint32_t)row;
      if (first + at < a.chunks && !(used[r >> 5] >> (r & 31) & 1)) ((f32x4*)a.dE)[first + at] = f32x4{};
    }
    return;
  }
  __shared__ uint64_t masks[kFew / 64];
  __shared__ __attribute__((aligned(16))) float sums[4][64 * kE];
  const int p = blockIdx.x / a.slabs, slab = blockIdx.x % a.slabs, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = (int)a.n;
  const int blocks = (n + 63) / 64, each = (blocks + 3) / 4;           // of 64 pairs, per wavefront
  const int id = a.ids[p];
  for (int b = wave * each; b < (wave + 1) * each && b < blocks; ++b) {
    const int q = 64 * b + lane;
    const uint64_t same = __ballot(q < n && a.ids[q < n ? q : p] == id);
    if (lane == 0) masks[b] = same;
  }
  __syncthreads();
  const bool before = lane < blocks && 64 * lane < p && (masks[lane < blocks ? lane : 0] & (p - 64 * lane >= 64 ? ~uint64_t{0} : (uint64_t{1} << (p - 64 * lane)) - 1));
  if ((uint32_t)id >= (uint32_t)a.V || __ballot(before)) return;       // the whole workgroup
  const int at = (slab * 64 + lane) * kE;
  const bool there = at < a.H;
  const char* from = a.dout + (there ? at : 0) * (int64_t)sizeof(T);
  float acc[kE] = {};
  for (int b = wave * each; b < (wave + 1) * each && b < blocks; ++b) {
    uint64_t same = masks[b];
    while (same) {
      u32x4 x[kAhead];
      int rows[kAhead], with = 0;
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        rows[u] = same ? 64 * b + __builtin_ctzll(same) : p;
        with += same != 0;
        same &= same - 1;
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (u < with) x[u] = *(const u32x4*)(from + rows[u] * a.dout_bytes);
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (u < with) Piece<T>::add(acc, x[u]);
    }
  }
#pragma unroll
  for (int i = 0; i < kE; ++i) sums[wave][lane * kE + i] = acc[i];
  __syncthreads();
  if (wave || !there) return;
#pragma unroll
  for (int w = 1; w < 4; ++w)
#pragma unroll
    for (int i = 0; i < kE; ++i) acc[i] += sums[w][lane * kE + i];
  write_run<T>(a, id, at, acc);
}

bool misaligned(const void* p, uintptr_t to = 16) { return ((uintptr_t)p & (to - 1)) != 0; }

nat_status embed_shape(int64_t n_rows, int32_t V, int32_t H, int32_t dtype, float scale, int64_t stride, int* size) {
  if (dtype != NAT_DTYPE_BF16 && dtype != NAT_DTYPE_F32) return NAT_UNSUPPORTED_DTYPE;
  *size = dtype == NAT_DTYPE_BF16 ? 2 : 4;
  if (n_rows < 0 || n_rows > INT32_MAX || !(scale > -INFINITY && scale < INFINITY)) return NAT_INVALID_ARG;
  if (V <= 0 || H <= 0 || H > (1 << 30) || (int64_t)H * *size % 16 || (stride != 0 && (stride < H || stride * *size % 16 || stride > INT32_MAX))) return NAT_BAD_SHAPE;
  return NAT_OK;
}

struct SortPlan {
  int passes, bits, tiles, piece;
  bool few;                             // tiles of kFewWaves wavefronts
  int64_t pieces;
  size_t pairs, counts, parts;          // bytes of each of four arrays of pairs, of the counts, of the parts
};
SortPlan sort_plan(int64_t n, int32_t V, int32_t H) {
  SortPlan p{};
  const int bits = 32 - __builtin_clz((unsigned)V);
  p.passes = (bits + kMostBits - 1) / kMostBits;
  p.bits = (bits + p.passes - 1) / p.passes;
  p.few = n <= kDirectTiles * 64 * kFewWaves * kPer;
  const int64_t tile = 64 * (p.few ? kFewWaves : kManyWaves) * kPer;
  p.tiles = (int)((n + tile - 1) / tile);
  p.piece = 8;
  while (p.piece < 64 && n / p.piece * ((H + 1023) / 1024) > 2048) p.piece *= 2;
  p.pieces = (n + p.piece - 1) / p.piece;
  auto whole = [](size_t x) { return (x + 255) / 256 * 256; };
  p.pairs = whole((size_t)n * 4);
  p.counts = n > kMerged ? whole((((size_t)p.tiles + 1) << p.bits) * 4) : 0;
  p.parts = whole((size_t)p.pieces * 2 * H * 4);
  return p;
}

// A larger one: by workgroups of 256 threads, 16 bytes per thread and 4 KB per workgroup, in order, of which LDS that nobody uses keeps three on a CU.  2.49 GB 340 us, 7.3 TB/s; with eight
// on a CU 365, in workgroups of 1024 392, four pieces to a workgroup 381 to 417.  Behind those of the sort's first launch, then of four wavefronts, or in a launch of their own where it is
// another: 20483 rows of 4096 into 151936 450 us in all; a launch of their own 457, beside sixteen wavefronts 490, beside the sums and into the rows without a pair alone 470.
// Where one ends and the other begins, us in all, beside the sort or few rows' sums and in order: 20483 rows of 1024 in bf16 into 311 MB 77 and 85, 377 MB 99 and 98, 438 MB 113 and 107, 623 MB 144
// and 136; 2897 of 1024 in fp32 into 311 MB 56 and 59, 377 MB 76 and 70, 438 MB 88 and 78; 9000 of 4096 into 344 MB 92 and 100, 410 MB 109 and 108; 40000 of 512 into 311 MB 95 and 100, 369 MB 110 and
// 111, 430 MB 124 and 121; 500 of 1024 into 344 MB 65 and 56.
constexpr int64_t kManyZeros = 360 << 20;                  // bytes
constexpr size_t kZeroLds = 52000;
__global__ void __launch_bounds__(256) zero_kernel(f32x4* to, int64_t chunks) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i < chunks) to[i] = f32x4{};
}
nat_status write_all_zeros(float* dE, int64_t chunks, hipStream_t s) {
  constexpr int64_t most = kMaxWorkItems / 256;
  for (int64_t at = 0; at < chunks; at += most * 256) {
    const int64_t left = chunks - at, blocks = (left + 255) / 256;
    zero_kernel<<<(unsigned)(blocks < most ? blocks : most), 256, kZeroLds, s>>>((f32x4*)dE + at, left);
    NAT_LAUNCH_CHECK();
  }
  return NAT_OK;
}

template <int W>
nat_status sort_pass(SortArgs a, hipStream_t s) {
  a.blocks = a.tiles;
  sort_count_kernel<W><<<(unsigned)(a.tiles + (a.chunks + 64 * W - 1) / (64 * W)), 64 * W, 0, s>>>(a);
  NAT_LAUNCH_CHECK();
  if (a.scanned) {
    sort_scan_kernel<<<1 << a.bits, 64 * kManyWaves, 0, s>>>(a);
    NAT_LAUNCH_CHECK();
  }
  sort_scatter_kernel<W><<<a.tiles, 64 * W, 0, s>>>(a);
  NAT_LAUNCH_CHECK();
  return NAT_OK;
}

}  // namespace
}  // namespace nat

using namespace nat;

extern "C" nat_status nat_embed(const int32_t* d_ids, int64_t n_rows, const void* d_E, int32_t V, int32_t H, int32_t dtype, float scale, void* d_out,
                                int64_t out_stride, void* stream) {
  int size;
  const nat_status st = embed_shape(n_rows, V, H, dtype, scale, out_stride, &size);
  if (st != NAT_OK) return st;
  if (n_rows == 0) return NAT_OK;
  if (!d_ids || !d_E || !d_out || misaligned(d_E) || misaligned(d_out)) return NAT_INVALID_ARG;
  EmbedArgs a{d_ids, (const char*)d_E, (char*)d_out, n_rows, (int64_t)H * size, (out_stride ? out_stride : H) * size, 0, V, 0, scale};
  while (a.lanes_log2 < 8 && (16 << a.lanes_log2) < a.row_bytes) ++a.lanes_log2;
  hipStream_t s = (hipStream_t)stream;
  ProfScope prof(PC_EMBED, s);
  const int64_t per = 256 >> a.lanes_log2, most = kMaxWorkItems / 256;
  for (; a.first < n_rows; a.first += most * per) {
    const int64_t blocks = (n_rows - a.first + per - 1) / per;
    const unsigned n = (unsigned)(blocks < most ? blocks : most);
    if (dtype == NAT_DTYPE_BF16) embed_kernel<uint16_t><<<n, 256, 0, s>>>(a);
    else embed_kernel<float><<<n, 256, 0, s>>>(a);
    NAT_LAUNCH_CHECK();
  }
  return NAT_OK;
}

extern "C" size_t nat_embed_bwd_workspace_bytes(int64_t n_rows, int32_t V, int32_t H) {
  if (n_rows <= 0 || n_rows >= (int64_t{1} << 29) || V <= 0 || V > (1 << 30) || H <= 0) return 0;
  const SortPlan p = sort_plan(n_rows, V, H);
  return 4 * p.pairs + p.counts + p.parts;
}

extern "C" nat_status nat_embed_bwd(const int32_t* d_ids, int64_t n_rows, const void* d_dout, int64_t dout_stride, int32_t V, int32_t H, int32_t dtype,
                                    float scale, float* d_dE, int32_t accumulate, void* d_ws, size_t ws_bytes, void* stream) {
  int size;
  const nat_status st = embed_shape(n_rows, V, H, dtype, scale, dout_stride, &size);
  if (st != NAT_OK) return st;
  if (V > (1 << 30) || n_rows >= (int64_t{1} << 29)) return NAT_BAD_SHAPE;
  const SortPlan p = sort_plan(n_rows > 0 ? n_rows : 1, V, H);
  // 16 bytes per thread, up to 256 threads
  const int64_t lanes = (int64_t)H * size / 16;
  const int threads = lanes >= 256 ? 256 : (int)((lanes + 63) / 64 * 64), slabs = (int)((lanes + threads - 1) / threads);
  const int64_t chunks = (int64_t)V * H / 4, sum_blocks = p.pieces * slabs;
  if (sum_blocks > kMaxWorkItems / kJoinThreads) return NAT_BAD_SHAPE;
  if (!d_dE || misaligned(d_dE)) return NAT_INVALID_ARG;
  if (n_rows > 0 && (!d_ids || !d_dout || misaligned(d_dout))) return NAT_INVALID_ARG;
  if (n_rows > 0 && (!d_ws || ws_bytes < nat_embed_bwd_workspace_bytes(n_rows, V, H))) return NAT_WORKSPACE_TOO_SMALL;
  if (misaligned(d_ws, 256)) return NAT_INVALID_ARG;
  hipStream_t s = (hipStream_t)stream;
  ProfScope prof(PC_EMBED, s);
  if (n_rows == 0) return accumulate ? NAT_OK : write_all_zeros(d_dE, chunks, s);
  // zeros beside others of the launch, or in a launch of their own
  const int64_t beside = !accumulate && chunks * 16 <= kManyZeros ? chunks : 0;
  const bool many = !accumulate && beside == 0, by_ranks = n_rows <= kMerged && chunks <= kMaxWorkItems - (1 << 24);
  const int64_t few_slabs = (lanes + 63) / 64;
  const bool few = n_rows <= kFew && n_rows * beside <= kFewWork && few_slabs <= 1 << 13;
  if (many && (few || !by_ranks)) {
    const nat_status zeros = write_all_zeros(d_dE, chunks, s);
    if (zeros != NAT_OK) return zeros;
  }
  if (few) {
    FewArgs f{};
    f.ids = d_ids;
    f.dout = (const char*)d_dout;
    f.dE = d_dE;
    f.n = n_rows;
    f.dout_bytes = (dout_stride ? dout_stride : H) * size;
    f.V = V;
    f.H = H;
    f.slabs = (int)few_slabs;
    f.scale = scale;
    f.accumulate = accumulate != 0;
    f.sum_blocks = (unsigned)(n_rows * few_slabs);
    f.chunks = beside;
    const unsigned blocks = f.sum_blocks + (unsigned)((beside + 256 * kFewSteps - 1) / (256 * kFewSteps));
    if (dtype == NAT_DTYPE_BF16) embed_few_kernel<uint16_t><<<blocks, 256, 0, s>>>(f);
    else embed_few_kernel<float><<<blocks, 256, 0, s>>>(f);
    NAT_LAUNCH_CHECK();
    return NAT_OK;
  }
  char* ws = (char*)d_ws;
  int32_t* pair[4];
  for (int i = 0; i < 4; ++i) pair[i] = (int32_t*)(ws + i * p.pairs);
  SortArgs a{d_ids, nullptr, pair[0], pair[1], (int32_t*)(ws + 4 * p.pairs), n_rows, V, 0, p.bits, p.tiles, p.tiles > kDirectTiles,
             0, (f32x4*)d_dE, many && by_ranks ? chunks : beside};
  auto rank = [&](auto pairs, auto most) {
    constexpr int kPairs = decltype(pairs)::value, kMost = decltype(most)::value;
    a.blocks = (unsigned)((n_rows + kPairs - 1) / kPairs);
    const int threads = many ? 256 : 64 * kRankWaves;
    const unsigned blocks = a.blocks + (unsigned)((a.chunks + threads - 1) / threads);
    if (many) rank_kernel<kPairs, kMost, 4><<<blocks, threads, kZeroLds - kMost / kBlock * kBlockPitch * 4, s>>>(a);
    else rank_kernel<kPairs, kMost, kRankWaves><<<blocks, threads, 0, s>>>(a);
  };
  if (n_rows <= kRanked) {
    rank(std::integral_constant<int, kRankPairs>{}, std::integral_constant<int, kRanked>{});
    NAT_LAUNCH_CHECK();
  } else if (n_rows <= kMerged) {
    rank(std::integral_constant<int, kTilePairs>{}, std::integral_constant<int, kMergeTile>{});
    NAT_LAUNCH_CHECK();
    a.ids_in = pair[0];
    a.rows_in = pair[1];
    a.ids_out = pair[2];
    a.rows_out = pair[3];
    merge_kernel<<<(unsigned)((n_rows + 1023) / 1024), 1024, (size_t)(n_rows + 3) / 4 * 16, s>>>(a);
    NAT_LAUNCH_CHECK();
  } else {
    for (int pass = 0; pass < p.passes; ++pass) {
      a.shift = pass * p.bits;
      a.ids_out = pair[pass & 1 ? 2 : 0];
      a.rows_out = pair[pass & 1 ? 3 : 1];
      const nat_status sorted = p.few ? sort_pass<kFewWaves>(a, s) : sort_pass<kManyWaves>(a, s);
      if (sorted != NAT_OK) return sorted;
      a.ids_in = a.ids_out;
      a.rows_in = a.rows_out;
      a.chunks = 0;
    }
  }
  SumArgs b{a.ids_out, a.rows_out, (const char*)d_dout, d_dE, (float*)(ws + 4 * p.pairs + p.counts), n_rows, (dout_stride ? dout_stride : H) * size, V, H,
            p.piece, slabs, scale, accumulate != 0};
  if (dtype == NAT_DTYPE_BF16) embed_sum_kernel<uint16_t><<<(unsigned)sum_blocks, threads, 0, s>>>(b);
  else embed_sum_kernel<float><<<(unsigned)sum_blocks, threads, 0, s>>>(b);
  NAT_LAUNCH_CHECK();
  if (p.pieces == 1) return NAT_OK;
  if (dtype == NAT_DTYPE_BF16) embed_join_kernel<uint16_t><<<(unsigned)sum_blocks, kJoinThreads / threads * threads, 0, s>>>(b, threads);
  else embed_join_kernel<float><<<(unsigned)sum_blocks, kJoinThreads / threads * threads, 0, s>>>(b, threads);
  NAT_LAUNCH_CHECK();
  return NAT_OK;
}
