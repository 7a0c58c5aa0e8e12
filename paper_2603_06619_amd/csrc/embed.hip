// Rows of an embedding by token id, and the gradient of the embedding: for every token the sum of its rows' gradients.
//
// The gradient sorts (id, row) pairs by id, rows of one id staying in order, and then walks the sorted pairs in pieces of equal length, whatever the ids: a token that
// makes up a tenth of the batch is shared by many workgroups like any other rows.  A run of equal ids inside a piece is summed and written by its workgroup; of one that
// crosses pieces each leaves its part, and a second kernel adds the parts in order.
#include "nat_internal.h"
#include "mfma_tile.hip.h"

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
  for (int64_t at = (int64_t)(threadIdx.x & (lanes - 1)) * 16; at < a.row_bytes; at += (int64_t)lanes * 16) {
    u32x4 x = {0, 0, 0, 0};
    if (there) x = Piece<T>::scaled(*(const u32x4*)(from + at), a.scale);
    *(u32x4*)(to + at) = x;
  }
}

// ------------------------------------------------------------------ the sort ----
// By digits from the lowest on, each pass stable.  A workgroup takes a tile of 1024 x kPer pairs; inside it, a wavefront ranks 64 pairs at a time by ballots
// over the digit's bits.
constexpr int kThreads = 1024, kSortWaves = kThreads / 64, kMostBits = 9, kMostBins = 1 << kMostBits;
constexpr int kSmallPer = 8, kPer = 4;                     // pairs per thread: all of a small call in one workgroup; a tile of a larger one
constexpr int kSmall = kThreads * kSmallPer, kTile = kThreads * kPer;
constexpr int kDirectTiles = 64;                           // up to so many tiles, each adds up the counts of those before it by itself

// Exclusive prefix sum over the workgroup
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
  for (int w = 0; w < kSortWaves; ++w) before += w < wave ? wave_sums[w] : 0;
  __syncthreads();
  return before + sum - x;
}

struct SortShared {
  int counts[kSortWaves][kMostBins];      // of a wavefront and digit; then the place of its first pair
  int wave_sums[kSortWaves];
};

// place[e]: where pair e of this thread (number wave * 64 * P + 64 e + lane of the tile) lies in the tile sorted by its digit
template <int P>
__device__ __forceinline__ void rank_tile(SortShared& s, const int (&digit)[P], int bits, int (&place)[P]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, bins = 1 << bits;
  for (int i = threadIdx.x; i < kSortWaves * bins; i += kThreads) s.counts[i >> bits][i & (bins - 1)] = 0;
  __syncthreads();
  volatile int* mine = s.counts[wave];
#pragma unroll
  for (int e = 0; e < P; ++e) {
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
  // digits in order, of each the wavefronts in order: bins * 16 entries, some per thread, or threads without any
  const int total = bins * kSortWaves, per = total > kThreads ? total / kThreads : 1, first = threadIdx.x * per;
  int sum = 0;
  for (int i = first; i < first + per && i < total; ++i) sum += s.counts[i % kSortWaves][i / kSortWaves];
  sum = block_scan(sum, s.wave_sums);
  for (int i = first; i < first + per && i < total; ++i) {
    const int n = s.counts[i % kSortWaves][i / kSortWaves];
    s.counts[i % kSortWaves][i / kSortWaves] = sum;
    sum += n;
  }
  __syncthreads();
#pragma unroll
  for (int e = 0; e < P; ++e) place[e] += s.counts[wave][digit[e]];
}

struct SortArgs {
  const int32_t *ids_in, *rows_in;      // rows_in NULL: the first pass, ids as the caller has them
  int32_t *ids_out, *rows_out, *counts;
  int64_t n;
  int32_t V;
  int shift, bits, tiles, passes;
  bool scanned;                         // counts hold places
};

__device__ __forceinline__ int32_t key_of(int32_t id, int32_t V) { return (uint32_t)id < (uint32_t)V ? id : V; }

// All passes of a small call
__global__ void __launch_bounds__(kThreads) sort_small_kernel(SortArgs a) {
  __shared__ SortShared s;
  __shared__ int32_t keys[kSmall];
  __shared__ uint16_t rows[kSmall];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int key[kSmallPer], row[kSmallPer], digit[kSmallPer], place[kSmallPer];
#pragma unroll
  for (int e = 0; e < kSmallPer; ++e) {
    const int i = wave * 64 * kSmallPer + 64 * e + lane;
    key[e] = i < a.n ? key_of(a.ids_in[i], a.V) : INT32_MAX;       // behind all others, in every pass
    row[e] = i;
  }
  for (int pass = 0; pass < a.passes; ++pass) {
    const int shift = pass * a.bits, mask = (1 << a.bits) - 1;
#pragma unroll
    for (int e = 0; e < kSmallPer; ++e) digit[e] = (key[e] >> shift) & mask;
    rank_tile<kSmallPer>(s, digit, a.bits, place);
#pragma unroll
    for (int e = 0; e < kSmallPer; ++e) {
      keys[place[e]] = key[e];
      rows[place[e]] = (uint16_t)row[e];
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < kSmallPer; ++e) {
      const int i = wave * 64 * kSmallPer + 64 * e + lane;
      key[e] = keys[i];
      row[e] = rows[i];
    }
    __syncthreads();
  }
#pragma unroll
  for (int e = 0; e < kSmallPer; ++e) {
    const int i = wave * 64 * kSmallPer + 64 * e + lane;
    if (i < a.n) {
      a.ids_out[i] = key[e];
      a.rows_out[i] = row[e];
    }
  }
}

// counts[bin][tile]
__global__ void __launch_bounds__(kThreads) sort_count_kernel(SortArgs a) {
  __shared__ int bins[kMostBins];
  const int n_bins = 1 << a.bits;
  if ((int)threadIdx.x < n_bins) bins[threadIdx.x] = 0;
  __syncthreads();
  const int64_t first = (int64_t)blockIdx.x * kTile;
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    const int64_t i = first + e * kThreads + threadIdx.x;
    if (i < a.n) atomicAdd(&bins[(key_of(a.ids_in[i], a.V) >> a.shift) & (n_bins - 1)], 1);
  }
  __syncthreads();
  if ((int)threadIdx.x < n_bins) a.counts[(int64_t)threadIdx.x * a.tiles + blockIdx.x] = bins[threadIdx.x];
}

// counts[bin][tile] -> those of the tiles before, and behind them all tiles' of the bin, in counts[bins * tiles + bin]
__global__ void __launch_bounds__(kThreads) sort_scan_kernel(SortArgs a) {
  __shared__ int wave_sums[kSortWaves], all;
  int32_t* of = a.counts + (int64_t)blockIdx.x * a.tiles;
  int before = 0;
  for (int first = 0; first < a.tiles; first += kThreads) {
    const int i = first + (int)threadIdx.x, x = i < a.tiles ? of[i] : 0;
    const int sum = block_scan(x, wave_sums);
    if (i < a.tiles) of[i] = before + sum;
    if (threadIdx.x == kThreads - 1) all = sum + x;
    __syncthreads();
    before += all;
    __syncthreads();
  }
  if (threadIdx.x == 0) a.counts[((int64_t)a.tiles << a.bits) + blockIdx.x] = before;
}

__global__ void __launch_bounds__(kThreads) sort_scatter_kernel(SortArgs a) {
  __shared__ SortShared s;
  __shared__ int to[kMostBins];           // place of the tile's first pair of a digit, minus its place inside the tile
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n_bins = 1 << a.bits, tile = blockIdx.x;
  int all = 0, before = 0;
  if ((int)threadIdx.x < n_bins) {
    const int32_t* of = a.counts + (int64_t)threadIdx.x * a.tiles;
    if (a.scanned) {
      before = of[tile];
      all = a.counts[((int64_t)a.tiles << a.bits) + threadIdx.x];
    } else {
      for (int t = 0; t < a.tiles; ++t) {
        const int x = of[t];
        all += x;
        before += t < tile ? x : 0;
      }
    }
  }
  before += block_scan(all, s.wave_sums);
  int key[kPer], row[kPer], digit[kPer], place[kPer];
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    const int64_t i = (int64_t)tile * kTile + wave * 64 * kPer + 64 * e + lane;
    key[e] = i < a.n ? key_of(a.ids_in[i], a.V) : INT32_MAX;
    row[e] = i < a.n ? a.rows_in ? a.rows_in[i] : (int32_t)i : -1;
    digit[e] = (key[e] >> a.shift) & (n_bins - 1);
  }
  rank_tile<kPer>(s, digit, a.bits, place);
  if ((int)threadIdx.x < n_bins) to[threadIdx.x] = before - s.counts[0][threadIdx.x];
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
  int piece, slabs;                     // pairs per piece; groups of four 16-byte columns of 64 lanes
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

template <typename T>
__global__ void __launch_bounds__(256) embed_sum_kernel(SumArgs a) {
  constexpr int kE = Piece<T>::kElements;
  const int slab = blockIdx.x % a.slabs;
  const int64_t piece = blockIdx.x / a.slabs, p0 = piece * a.piece, p1 = p0 + a.piece < a.n ? p0 + a.piece : a.n;
  const int at = (slab * 256 + (int)threadIdx.x) * kE;
  if (at >= a.H) return;
  const bool from_before = p0 > 0 && a.ids[p0 - 1] == a.ids[p0], goes_on = p1 < a.n && a.ids[p1 - 1] == a.ids[p1];
  int32_t id = a.ids[p0];
  bool first_run = true;
  float acc[kE] = {};
  auto flush = [&](bool last) {
    if (id >= a.V) return;
    const int side = first_run && from_before ? 0 : last && goes_on ? 1 : -1;
    if (side < 0) {
      write_run<T>(a, id, at, acc);
    } else {
      float* to = a.part + (piece * 2 + side) * a.H + at;
#pragma unroll
      for (int i = 0; i < kE; i += 4) *(f32x4*)(to + i) = f32x4{acc[i], acc[i + 1], acc[i + 2], acc[i + 3]};
    }
  };
  for (int64_t p = p0; p < p1; ++p) {
    const int32_t next = a.ids[p];
    if (next != id) {
      flush(false);
      first_run = false;
      id = next;
#pragma unroll
      for (int i = 0; i < kE; ++i) acc[i] = 0.f;
    }
    Piece<T>::add(acc, *(const u32x4*)(a.dout + a.rows[p] * a.dout_bytes + at * (int64_t)sizeof(T)));
  }
  flush(true);
}

// The parts of a run that begins in this piece and goes on behind it
template <typename T>
__global__ void __launch_bounds__(256) embed_join_kernel(SumArgs a) {
  constexpr int kE = Piece<T>::kElements;
  const int slab = blockIdx.x % a.slabs;
  const int64_t piece = blockIdx.x / a.slabs, p0 = piece * a.piece, p1 = p0 + a.piece;
  const int at = (slab * 256 + (int)threadIdx.x) * kE;
  if (at >= a.H || p1 >= a.n) return;
  const int32_t id = a.ids[p1];
  if (id >= a.V || a.ids[p1 - 1] != id || (a.ids[p0] == id && p0 > 0 && a.ids[p0 - 1] == id)) return;
  float acc[kE];
  const float* from = a.part + (piece * 2 + 1) * a.H + at;
#pragma unroll
  for (int i = 0; i < kE; ++i) acc[i] = from[i];
  for (int64_t c = piece + 1; c * a.piece < a.n && a.ids[c * a.piece] == id; ++c) {
    from = a.part + c * 2 * a.H + at;
#pragma unroll
    for (int i = 0; i < kE; ++i) acc[i] += from[i];
  }
  write_run<T>(a, id, at, acc);
}

bool misaligned(const void* p, uintptr_t to = 16) { return ((uintptr_t)p & (to - 1)) != 0; }

nat_status embed_shape(int64_t n_rows, int32_t V, int32_t H, int32_t dtype, float scale, int64_t stride, int* size) {
  if (dtype != NAT_DTYPE_BF16 && dtype != NAT_DTYPE_F32) return NAT_UNSUPPORTED_DTYPE;
  *size = dtype == NAT_DTYPE_BF16 ? 2 : 4;
  if (n_rows < 0 || n_rows > INT32_MAX || !(scale > -INFINITY && scale < INFINITY)) return NAT_INVALID_ARG;
  if (V <= 0 || H <= 0 || (int64_t)H * *size % 16 || (stride != 0 && (stride < H || stride * *size % 16 || stride > INT32_MAX))) return NAT_BAD_SHAPE;
  return NAT_OK;
}

struct SortPlan {
  int passes, bits, tiles, piece, slabs;
  int64_t pieces;
  size_t pairs, counts, parts;          // bytes of each of four arrays of pairs, of the counts, of the parts
};
SortPlan sort_plan(int64_t n, int32_t V, int32_t H) {
  SortPlan p{};
  const int bits = 32 - __builtin_clz((unsigned)V);
  p.passes = (bits + kMostBits - 1) / kMostBits;
  p.bits = (bits + p.passes - 1) / p.passes;
  p.tiles = (int)((n + kTile - 1) / kTile);
  p.slabs = (H + 1023) / 1024;          // of f32; bf16 has half as many
  p.piece = 8;
  while (p.piece < 64 && n / p.piece * p.slabs > 2048) p.piece *= 2;
  p.pieces = (n + p.piece - 1) / p.piece;
  auto whole = [](size_t x) { return (x + 255) / 256 * 256; };
  p.pairs = whole((size_t)n * 4);
  p.counts = n > kSmall ? whole((((size_t)p.tiles + 1) << p.bits) * 4) : 0;
  p.parts = whole((size_t)p.pieces * 2 * H * 4);
  return p;
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
  const SortPlan p = sort_plan(n_rows, V, H);
  const int slabs = dtype == NAT_DTYPE_BF16 ? (p.slabs + 1) / 2 : p.slabs;
  if (p.pieces * slabs > kMaxWorkItems / 256) return NAT_BAD_SHAPE;
  if (!d_dE || misaligned(d_dE)) return NAT_INVALID_ARG;
  if (n_rows > 0 && (!d_ids || !d_dout || misaligned(d_dout))) return NAT_INVALID_ARG;
  if (n_rows > 0 && (!d_ws || ws_bytes < nat_embed_bwd_workspace_bytes(n_rows, V, H))) return NAT_WORKSPACE_TOO_SMALL;
  if (misaligned(d_ws, 256)) return NAT_INVALID_ARG;
  hipStream_t s = (hipStream_t)stream;
  ProfScope prof(PC_EMBED, s);
  if (!accumulate) {
    const nat_status filled = fill_zero_f32(d_dE, (size_t)V * H, s);
    if (filled != NAT_OK) return filled;
  }
  if (n_rows == 0) return NAT_OK;
  char* ws = (char*)d_ws;
  int32_t* pair[4];
  for (int i = 0; i < 4; ++i) pair[i] = (int32_t*)(ws + i * p.pairs);
  SortArgs a{d_ids, nullptr, pair[0], pair[1], (int32_t*)(ws + 4 * p.pairs), n_rows, V, 0, p.bits, p.tiles, p.passes, p.tiles > kDirectTiles};
  if (n_rows <= kSmall) {
    sort_small_kernel<<<1, kThreads, 0, s>>>(a);
    NAT_LAUNCH_CHECK();
  } else {
    for (int pass = 0; pass < p.passes; ++pass) {
      a.shift = pass * p.bits;
      a.ids_out = pair[pass & 1 ? 2 : 0];
      a.rows_out = pair[pass & 1 ? 3 : 1];
      sort_count_kernel<<<p.tiles, kThreads, 0, s>>>(a);
      NAT_LAUNCH_CHECK();
      if (a.scanned) {
        sort_scan_kernel<<<1 << p.bits, kThreads, 0, s>>>(a);
        NAT_LAUNCH_CHECK();
      }
      sort_scatter_kernel<<<p.tiles, kThreads, 0, s>>>(a);
      NAT_LAUNCH_CHECK();
      a.ids_in = a.ids_out;
      a.rows_in = a.rows_out;
    }
  }
  SumArgs b{a.ids_out, a.rows_out, (const char*)d_dout, d_dE, (float*)(ws + 4 * p.pairs + p.counts), n_rows, (dout_stride ? dout_stride : H) * size, V, H,
            p.piece, slabs, scale, accumulate != 0};
  const int64_t blocks = p.pieces * slabs;
  if (dtype == NAT_DTYPE_BF16) embed_sum_kernel<uint16_t><<<(unsigned)blocks, 256, 0, s>>>(b);
  else embed_sum_kernel<float><<<(unsigned)blocks, 256, 0, s>>>(b);
  NAT_LAUNCH_CHECK();
  if (dtype == NAT_DTYPE_BF16) embed_join_kernel<uint16_t><<<(unsigned)blocks, 256, 0, s>>>(b);
  else embed_join_kernel<float><<<(unsigned)blocks, 256, 0, s>>>(b);
  NAT_LAUNCH_CHECK();
  return NAT_OK;
}
