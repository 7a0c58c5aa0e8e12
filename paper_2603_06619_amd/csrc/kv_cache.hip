// Paged key-value cache: writing rows into it (as they are, in 8 bits, or in 4), reading sequences back, and attention of one new token per sequence.
//
// A page holds page_size tokens of every key head, [head][token][head_dim], so that a head's tokens of a page are contiguous.  In the 8-bit format
// (4 exponent bits, 3 mantissa bits, largest 448) a row (token, head) has one scale 2^e, the smallest power of two that brings its largest magnitude to 448 or
// less: multiplying by a power of two rounds nothing, so the one rounding is that to 3 mantissa bits, and reading back is exact.  A power of two loses
// no precision against a scale that reaches 448 exactly (the format is floating), and costs 1 byte per row.
//
// In the 4-bit format (2 exponent bits, 1 mantissa bit, largest 6) every group of 32 elements of a row has a scale of its own: with so few values one large element would
// leave nothing of the others of a whole row.  The hardware's conversions take the scale along; every value is exact in bf16.
#include "nat_internal.h"
#include "mfma_tile.hip.h"

#include <type_traits>

namespace nat {
namespace {

constexpr float kLog2E = 1.4426950408889634f;

struct CacheArgs {
  char *k, *v;                   // rows of head_dim elements
  uint8_t *k_exp, *v_exp;
  int n_pages, hkv, page_log2;
};

__device__ __forceinline__ int64_t cache_row(const CacheArgs& c, int64_t page, int head, int at) {
  return ((page * c.hkv + head) << c.page_log2) + at;
}

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float bf16_to_f32(uint32_t bits) { return __builtin_bit_cast(float, bits << 16); }
__device__ __forceinline__ float power_of_two(int biased) { return __builtin_bit_cast(float, (uint32_t)biased << 23); }

// Four 8-bit values to four bf16, exactly
__device__ __forceinline__ u32x2 widen_fp8(uint32_t x) {
  const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.f, false), hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.f, true);
  return u32x2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
}

// Eight 4-bit values times 2^(exp - 127) to eight bf16, exactly (exp = 255: NaN)
constexpr int kGroup = 32;                // elements that share a scale in 4 bits
__device__ __forceinline__ u32x4 widen_fp4(uint32_t x, uint32_t exp) {
  const float scale = power_of_two((int)exp);
  return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 0)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 1)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 2)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 3))};
}

struct WriteArgs {
  CacheArgs c;
  const uint16_t *k, *v;
  int64_t k_stride, v_stride, n_rows, first;      // first: (row, head) pair that the launch begins with
  const int64_t* slots;
};

// One row (token, head) per D / 8 lanes, 16 bytes of the input each.  32749 tokens of 8 heads of 128: 202 MB in 37 us, 5.5 TB/s (a copy: 4.9); 64 tokens 3.4 us,
// the time of a launch.
template <int D, int kFormat>
__device__ __forceinline__ void write_row(const uint16_t* row, char* cache, uint8_t* exps, int64_t to, int lane) {
  const u32x4 x = *(const u32x4*)(row + 8 * lane);
  if constexpr (kFormat == NAT_KV_BF16) {
    *(u32x4*)(cache + (to * D + 8 * lane) * 2) = x;
  } else if constexpr (kFormat == NAT_KV_FP4) {
    uint32_t largest = 0;                    // magnitude as bits of bf16, of the group that four lanes hold
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t lo = x[i] & 0x7fff, hi = (x[i] >> 16) & 0x7fff;
      if (lo > largest) largest = lo;
      if (hi > largest) largest = hi;
    }
#pragma unroll
    for (int d = 1; d < kGroup / 8; d <<= 1) {
      const uint32_t other = __shfl_xor(largest, d, 64);
      largest = other > largest ? other : largest;
    }
    // largest = 1.f 2^(E - 127) <= 1.5 2^(2 + e); at 2^125 values of 3.5 2^127 and more become 6 2^125, which bf16 still holds
    int e = (int)(largest >> 7) - 2 + ((largest & 0x7f) > 0x40);
    e = e < 2 ? 2 : e > 252 ? 252 : e;
    const float scale = power_of_two(e);
    const bool finite = largest < 0x7f80;
    // (of an element of a vector as it stands, the cast takes the first one's bits)
    auto pair = [&](int i) { const uint32_t two = x[i]; return __builtin_bit_cast(bf16x2, two); };
    uint32_t out = 0;
    if (finite) {
      out = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(out, pair(0), scale, 0);
      out = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(out, pair(1), scale, 1);
      out = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(out, pair(2), scale, 2);
      out = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(out, pair(3), scale, 3);
    }
    *(uint32_t*)(cache + to * (D / 2) + 4 * lane) = out;
    if (lane % (kGroup / 8) == 0) exps[to * (D / kGroup) + lane / (kGroup / 8)] = (uint8_t)(finite ? e : 255);
  } else {
    uint32_t largest = 0;                    // of the finite magnitudes, as bits of bf16
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t lo = x[i] & 0x7fff, hi = (x[i] >> 16) & 0x7fff;
      if (lo < 0x7f80 && lo > largest) largest = lo;
      if (hi < 0x7f80 && hi > largest) largest = hi;
    }
#pragma unroll
    for (int d = 1; d < D / 8; d <<= 1) {
      const uint32_t other = __shfl_xor(largest, d, 64);
      largest = other > largest ? other : largest;
    }
    // largest = 1.f 2^(E - 127) <= 1.75 2^(8 + e)
    int e = (int)(largest >> 7) - 127 - 8 + ((largest & 0x7f) > 0x60);
    if (e < -126) e = -126;
    u32x2 out = {0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float a = bf16_to_f32(x[i] & 0xffff), b = bf16_to_f32(x[i] >> 16);
      a = ldexpf(a, -e);
      b = ldexpf(b, -e);
      // the format has no infinity: what is not finite is NaN
      if ((x[i] & 0x7f80) == 0x7f80) a = NAN;
      if ((x[i] & 0x7f800000) == 0x7f800000) b = NAN;
      if (i & 1) out[i >> 1] = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, out[i >> 1], true);
      else out[i >> 1] = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, out[i >> 1], false);
    }
    *(u32x2*)(cache + to * D + 8 * lane) = out;
    if (lane == 0) exps[to] = (uint8_t)(e + 127);
  }
}

template <int D, int kFormat>
__global__ void __launch_bounds__(256) kv_write_kernel(WriteArgs a) {
  constexpr int kLanes = D / 8;
  const int lane = threadIdx.x % kLanes;
  const int64_t id = a.first + (int64_t)blockIdx.x * (256 / kLanes) + threadIdx.x / kLanes, row = id / a.c.hkv;
  if (row >= a.n_rows) return;
  const int head = (int)(id - row * a.c.hkv);
  const int64_t slot = a.slots[row];
  if (slot < 0 || (slot >> a.c.page_log2) >= a.c.n_pages) return;
  const int64_t to = cache_row(a.c, slot >> a.c.page_log2, head, (int)(slot & ((1 << a.c.page_log2) - 1)));
  write_row<D, kFormat>(a.k + row * a.k_stride + head * D, a.c.k, a.c.k_exp, to, lane);
  write_row<D, kFormat>(a.v + row * a.v_stride + head * D, a.c.v, a.c.v_exp, to, lane);
}

struct ReadArgs {
  CacheArgs c;
  const int32_t *table, *cu;
  int table_width, n_seqs;
  int64_t n_rows, k_stride, v_stride, first;      // first: as in WriteArgs
  uint16_t *k, *v;
};

// 8 elements of a row as the cache has them
template <int D, int kFormat>
struct Stored {
  typedef uint32_t Bits __attribute__((ext_vector_type(kFormat == NAT_KV_BF16 ? 4 : 2)));
  std::conditional_t<kFormat == NAT_KV_FP4, uint32_t, Bits> x;
  uint8_t exp;
  __device__ __forceinline__ void load(const char* cache, const uint8_t* exps, int64_t from, int lane) {
    constexpr int kBytes = sizeof(x);
    x = *(const decltype(x)*)(cache + (from * (D / 8) + lane) * kBytes);
    if constexpr (kFormat == NAT_KV_FP4) exp = exps[from * (D / kGroup) + lane / (kGroup / 8)];
    if constexpr (kFormat == NAT_KV_FP8) exp = exps[from];
  }
  __device__ __forceinline__ u32x4 bf16() const {
    if constexpr (kFormat == NAT_KV_BF16) {
      return x;
    } else if constexpr (kFormat == NAT_KV_FP4) {
      return widen_fp4(x, exp);
    } else {
      const float scale = power_of_two(exp);
      u32x4 y;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(x[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(x[i], true);
        y[2 * i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(lo * scale, bf16x2));
        y[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_convertvector(hi * scale, bf16x2));
      }
      return y;
    }
  }
};

// The sequence of a packed row is searched for by the lanes that read it, once for the two rows that each of them reads: a chain of five or six loads, after which both rows of keys and of
// values are under way.  106 MB of 6 sequences from 8 bits in 18.4 us (18.9 with a profiler), 5.8 TB/s, most of it written, where a copy writes half; 102 MB from 4 bits in 18.1 (19.0), behind a launch that fills the
// Infinity Cache and with one that reads the rows 56 (a row per lane 20.3, 20.9 and 64; four rows 19.2, 18.1 and 57).
constexpr int kReadRows = 2;
template <int D, int kFormat>
__global__ void __launch_bounds__(256) kv_read_kernel(ReadArgs a) {
  constexpr int kLanes = D / 8, kPairs = 256 / kLanes;
  const int lane = threadIdx.x % kLanes;
  const int64_t first = a.cu[0], last = a.cu[a.n_seqs] < a.n_rows ? a.cu[a.n_seqs] : a.n_rows;
  int seq = 0, page[kReadRows], head[kReadRows];
  int64_t begin = 0, end = 0, row[kReadRows], at[kReadRows];
#pragma unroll
  for (int u = 0; u < kReadRows; ++u) {
    const int64_t id = a.first + ((int64_t)blockIdx.x * kReadRows + u) * kPairs + threadIdx.x / kLanes;
    row[u] = id / a.c.hkv;
    head[u] = (int)(id - row[u] * a.c.hkv);
    if (row[u] < first || row[u] >= last) row[u] = -1;
    if (row[u] >= end) {
      seq = rollout_of_pos(a.cu, 0, a.n_seqs, row[u]);
      begin = a.cu[seq];
      end = a.cu[seq + 1];
    }
    at[u] = row[u] - begin;
    const int64_t place = at[u] >> a.c.page_log2;
    page[u] = -1;
    if (row[u] >= 0 && place < a.table_width) page[u] = a.table[(int64_t)seq * a.table_width + place];
  }
  Stored<D, kFormat> k[kReadRows], v[kReadRows];
#pragma unroll
  for (int u = 0; u < kReadRows; ++u) {
    if (page[u] >= a.c.n_pages) page[u] = -1;
    const int64_t from = page[u] >= 0 ? cache_row(a.c, page[u], head[u], (int)(at[u] & ((1 << a.c.page_log2) - 1))) : 0;
    k[u].load(a.c.k, a.c.k_exp, from, lane);
    v[u].load(a.c.v, a.c.v_exp, from, lane);
  }
#pragma unroll
  for (int u = 0; u < kReadRows; ++u) {
    if (row[u] < 0) continue;
    *(u32x4*)(a.k + row[u] * a.k_stride + head[u] * D + 8 * lane) = page[u] >= 0 ? k[u].bf16() : u32x4{0, 0, 0, 0};
    *(u32x4*)(a.v + row[u] * a.v_stride + head[u] * D + 8 * lane) = page[u] >= 0 ? v[u].bf16() : u32x4{0, 0, 0, 0};
  }
}

// ------------------------------------------------------------------ one new token ----
// out = sum_j P_j v_j, P_j = exp(scale q . k_j - lse) for every query head, over the cached tokens of its sequence.
//
// A workgroup takes a chunk of one sequence's tokens for one key head and up to 16 of the query heads that share it: the columns of 16 x 16 x 32 products.  Its
// four wavefronts take 32 tokens each in turn, with a running maximum and sum of their own, and join at the end; chunks are joined by a second kernel
// where there is more than one.  Every cached byte is read once for all heads of the group; the products cost nothing beside that (a group of fewer than 16 heads
// leaves columns of them empty).  The next 32 tokens are in registers while these are worked on: at two wavefronts per SIMD, 64 KB in flight per compute unit.
// 128 sequences of up to 8192 tokens (32 heads on 8 of 128, 8-bit) 235 us, 5.3 TB/s; one of 32768 (28 on 4, bf16) 15.5 us, 4.3 TB/s: 256 tokens per
// workgroup, of which the first loads are a third of the time.  The first from 4 bits 123 us, 5.4 TB/s.
// Rounded to fewer bits are the probabilities, to bf16 for the product (with an 8-bit row's power of two in them, which rounds nothing).  From 4 bits, where values are exact in bf16, what
// that rounding leaves is a second bf16, and both are multiplied: together good to 2^-16.  A group of up to 8 query heads leaves half of the columns empty; there these are kHalves, and the second
// numbers take that half (lanes n >= 8, which hold the scores of head n - 8), so that there are no more products than before; larger groups have twice as many.  Error in the 2-norm 0.0017, the
// result's rounding; with probabilities of 8 bits 0.0021.
// 128 sequences of up to 8192 tokens (32 heads on 8 of 128) 127.6 us, rounded once 125.3; of up to 2048 39.9 and 39.5, with heads of 64 27.1 and 25.8 (with twice the products 41.8 and 28.7).
constexpr int kTokens = 32;               // tokens per step of a wavefront
constexpr int kHeads = 16;                // query heads per workgroup
constexpr int kMaxChunk = 4096, kMinChunk = 256;

struct DecodeArgs {
  CacheArgs c;
  const uint16_t* q;
  uint16_t* out;
  float* lse;
  const int32_t *table, *lens;
  int table_width, n_seqs, hq, group, head_blocks, chunk, n_chunks;
  int64_t q_stride, out_stride;
  float scale;
  float *part_out, *part_ml;     // [n_seqs][hq][n_chunks][D], [..][2]
};

__device__ __forceinline__ int length_of(const DecodeArgs& a, int seq) {
  const int64_t most = (int64_t)a.table_width << a.c.page_log2;
  const int l = a.lens[seq];
  return l < 0 ? 0 : l < most ? l : (int)most;
}

__device__ __forceinline__ f32x4 mfma16x16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// over the four groups of 16 lanes
__device__ __forceinline__ float max_groups(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
  return max_halves(fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1])));
}
__device__ __forceinline__ float sum_groups(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
  return sum_halves(__builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]));
}

// 32 tokens of keys and values in flight.  Keys are operands as they lie in memory (lane l: token l % 16 of a block of 16, elements by l / 16); the
// order of the elements is the same in the query's fragments.
template <int D, int kFormat>
struct TokenTile {
  static constexpr bool kFp4 = kFormat == NAT_KV_FP4;
  static constexpr int kRowBytes = kFormat == NAT_KV_BF16 ? 2 * D : kFp4 ? D / 2 : D;
  static constexpr int kKeyBytes = kRowBytes / 4 < 16 ? kRowBytes / 4 : 16;      // per load
  static constexpr int kKeyLoads = kRowBytes / 4 / kKeyBytes;         // per block of 16 tokens
  static constexpr int kRowLanes = kRowBytes / 16;                    // lanes per row of values
  static constexpr int kValueLoads = kTokens * kRowLanes / 64;
  typedef uint32_t Key __attribute__((ext_vector_type(kKeyBytes / 4)));
  Key k[2][kKeyLoads];
  u32x4 v[kValueLoads];
  uint32_t k_exp[2], v_exp[kFp4 ? kValueLoads : 2];

  // row and 16 bytes of it that a lane has of load i of values.  In 4 bits a lane writes four chunks of LDS for its 16 bytes, and lanes next to each other take rows next to
  // each other, whose chunks lie in different banks; four lanes to a row would meet in the same ones (two thirds of the LDS cycles of a decoding call were conflicts)
  __device__ __forceinline__ static int value_row(int i, int lane) { return i * (64 / kRowLanes) + (kFp4 ? lane % (64 / kRowLanes) : lane / kRowLanes); }
  __device__ __forceinline__ static int value_at(int lane) { return kFp4 ? lane / (64 / kRowLanes) : lane % kRowLanes; }

  // first of the eight elements of fragment s of a key that lane group g has
  __device__ __forceinline__ static int element(int s, int g) {
    if constexpr (kFp4) return D / 4 * g + 8 * s;
    else if constexpr (kFormat == NAT_KV_FP8) return 64 * (s >> 1) + 16 * g + 8 * (s & 1);
    else return 32 * s + 8 * g;
  }

  // Of a cache in 4 bits past the chip's caches: nobody reads it again before the next token, and the other layers come in between.  128 sequences of up to 8192 tokens 128.5 us, otherwise
  // 142; after a launch that has filled the Infinity Cache 126 and 175, 16 of up to 16384 45 and 62, one of 32768 16.4 and 21.5, 128 of up to 2048 with heads of 64 26.6 and 34 (which,
  // called again and again, the cache holds: 27.4 and 26.9).  Tables that name the same pages for two, four or eight sequences next to each other, after such a launch: 112, 108 and 103,
  // otherwise 116, 104 and 103.
  template <typename V>
  __device__ __forceinline__ static V once(const V* p) {
    if constexpr (kFp4) return __builtin_nontemporal_load(p);
    else return *p;
  }

  // p0, p1: pages of the two blocks of 16 tokens, at: place of the first in its page
  __device__ __forceinline__ void load(const CacheArgs& c, int p0, int p1, int head, int t0, int lane) {
    const int mask = (1 << c.page_log2) - 1, n = lane & 15, g = lane >> 4;
    const int64_t r0 = cache_row(c, p0 < 0 ? 0 : p0, head, t0 & mask), r1 = cache_row(c, p1 < 0 ? 0 : p1, head, (t0 + 16) & mask);
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const char* row = c.k + ((b ? r1 : r0) + n) * kRowBytes + kKeyBytes * g;
#pragma unroll
      for (int i = 0; i < kKeyLoads; ++i) k[b][i] = once((const Key*)(row + 64 * i));
      if constexpr (kFp4) k_exp[b] = once(c.k_exp + ((b ? r1 : r0) + n) * (D / kGroup) + D / 4 * g / kGroup);
      if constexpr (kFormat == NAT_KV_FP8) {
        k_exp[b] = *(const uint32_t*)(c.k_exp + (b ? r1 : r0) + 4 * g);
        v_exp[b] = *(const uint32_t*)(c.v_exp + (b ? r1 : r0) + 4 * g);
      }
    }
#pragma unroll
    for (int i = 0; i < kValueLoads; ++i) {
      const int row = value_row(i, lane);
      v[i] = once((const u32x4*)(c.v + ((row < 16 ? r0 : r1 - 16) + row) * kRowBytes + value_at(lane) * 16));
      if constexpr (kFp4) v_exp[i] = once(c.v_exp + ((row < 16 ? r0 : r1 - 16) + row) * (D / kGroup) + value_at(lane));
    }
  }

  __device__ __forceinline__ bf16x8 key_fragment(int b, int s) const {
    if constexpr (kFormat == NAT_KV_BF16) {
      return __builtin_bit_cast(bf16x8, k[b][s]);
    } else if constexpr (kFp4) {
      return __builtin_bit_cast(bf16x8, widen_fp4(k[b][0][s], k_exp[b]));
    } else {
      const u32x4 x = k[b][s >> 1];
      const u32x2 lo = widen_fp8(x[2 * (s & 1)]), hi = widen_fp8(x[2 * (s & 1) + 1]);
      return __builtin_bit_cast(bf16x8, u32x4{lo[0], lo[1], hi[0], hi[1]});
    }
  }

  // values to LDS as bf16, rows of tokens that are not there as zeros
  __device__ __forceinline__ void store_values(char* tile, bool whole, int first_live, int end_live, int lane) const {
#pragma unroll
    for (int i = 0; i < kValueLoads; ++i) {
      const int row = value_row(i, lane), at = value_at(lane);
      u32x4 x = v[i];
      if (!whole && (row < first_live || row >= end_live)) x = u32x4{0, 0, 0, 0};
      if constexpr (kFormat == NAT_KV_BF16) {
        *(u32x4*)(tile + RowTile<D>::chunk_at(row, at)) = x;
      } else if constexpr (kFp4) {
        const uint32_t e = !whole && (row < first_live || row >= end_live) ? 127 : v_exp[i];            // (a place that is not there may hold 255)
#pragma unroll
        for (int j = 0; j < 4; ++j) *(u32x4*)(tile + RowTile<D>::chunk_at(row, 4 * at + j)) = widen_fp4(x[j], e);
      } else {
        const u32x2 a = widen_fp8(x[0]), b = widen_fp8(x[1]), c = widen_fp8(x[2]), d = widen_fp8(x[3]);
        *(u32x4*)(tile + RowTile<D>::chunk_at(row, 2 * at)) = u32x4{a[0], a[1], b[0], b[1]};
        *(u32x4*)(tile + RowTile<D>::chunk_at(row, 2 * at + 1)) = u32x4{c[0], c[1], d[0], d[1]};
      }
    }
  }
};

template <int D, int kFormat, bool kHalves>
__global__ void __launch_bounds__(256, kFormat == NAT_KV_FP4 ? 4 : 2) decode_kernel(DecodeArgs a) {
  __shared__ __attribute__((aligned(16))) char values[4][kTokens * D * 2];       // and, at the end, the wavefronts' results
  __shared__ int32_t pages[kMaxChunk / 16];
  __shared__ float wave_m[4][kHeads], wave_sum[4][kHeads], joined_m[kHeads], joined_sum[kHeads];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  int id = blockIdx.x;
  const int block = id % a.head_blocks;
  id /= a.head_blocks;
  const int head = id % a.c.hkv;
  id /= a.c.hkv;
  const int seq = id % a.n_seqs, chunk = id / a.n_seqs;
  const int len = length_of(a, seq), first = chunk * a.chunk;
  if (first >= len && chunk > 0) return;
  const int end = len - first < a.chunk ? len - first : a.chunk;      // tokens of the chunk (0: an empty sequence)
  const int heads_here = a.group - block * kHeads < kHeads ? a.group - block * kHeads : kHeads;
  const int head0 = head * a.group + block * kHeads, column = kHalves ? n % (kHeads / 2) : n;       // the lane's query head
  // minus one for the lanes that take what rounding left, as either half of two bf16
  uint32_t minus = kHalves && n < kHeads / 2 ? 0 : 0xbf80;
  asm("" : "+v"(minus));                   // (as a constant the compiler writes it as -1 in 32 bits, which is the other half)
  const bf16x2 of_low = __builtin_bit_cast(bf16x2, minus), of_high = __builtin_bit_cast(bf16x2, minus << 16);

  for (int i = threadIdx.x; i < (end + 15) / 16; i += 256) {
    const int p = a.table[(int64_t)seq * a.table_width + ((first + 16 * i) >> a.c.page_log2)];
    pages[i] = p < a.c.n_pages ? p : -1;
  }
  bf16x8 q[D / 32];
#pragma unroll
  for (int s = 0; s < D / 32; ++s) {
    q[s] = bf16x8{};
    if (column < heads_here) q[s] = *(const bf16x8*)(a.q + seq * a.q_stride + (head0 + column) * D + TokenTile<D, kFormat>::element(s, g));
  }
  __syncthreads();

  const float to_log2 = a.scale * kLog2E;
  float m = -INFINITY, sum = 0.f;
  f32x4 acc[D / 16] = {};
  char* vt = values[wave];
  auto load = [&](TokenTile<D, kFormat>& t, int t0) {
    const int last = (end - 1) / 16, b = t0 / 16;
    t.load(a.c, __builtin_amdgcn_readfirstlane(pages[b]), __builtin_amdgcn_readfirstlane(pages[b < last ? b + 1 : last]), head, first + t0, lane);
  };
  // In 4 bits one tile, loaded again as soon as its keys and values have been read: 125 registers, four workgroups per compute unit (128 sequences of up to 8192 tokens 128.5 us; with a second
  // tile 136, three workgroups; of up to 2048 40 and 45, with heads of 64 27.4 and 28.4; 100 of up to 3000 55.4 and 52).
  constexpr int kTiles = kFormat == NAT_KV_FP4 ? 1 : 2;
  auto step = [&](TokenTile<D, kFormat>& t, int t0, int ahead) {
    const int last = (end - 1) / 16, b0 = t0 / 16;
    const bool there0 = pages[b0] >= 0, there1 = b0 < last && pages[b0 + 1] >= 0;
    const bool whole = t0 + kTokens <= end && there0 && there1;
    const int first_live = there0 ? 0 : 16, end_live = !there1 ? (end - t0 < 16 ? end - t0 : 16) : end - t0;
    t.store_values(vt, whole, first_live, end_live, lane);
    f32x4 st[2] = {};
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int s = 0; s < D / 32; ++s) st[b] = mfma16x16(t.key_fragment(b, s), q[s], st[b]);
    if constexpr (kTiles == 1) {
      if (ahead < end) load(t, ahead);
    }
    if constexpr (kFormat == NAT_KV_FP8) {
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) st[b][i] *= power_of_two((t.k_exp[b] >> (8 * i)) & 0xff);
    }
    if (!whole) {
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int row = 16 * b + 4 * g + i;
          if (row < first_live || row >= end_live) st[b][i] = -INFINITY;
        }
    }
    float top = m;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) top = fmaxf(top, st[b][i]);
    top = max_groups(top);
    if (__any(top > m)) {
      const float f = top == -INFINITY ? 1.f : exp2_fast((m - top) * to_log2);
      sum *= f;
#pragma unroll
      for (int db = 0; db < D / 16; ++db) acc[db] *= f;
      m = top;
    }
    const float shift = m == -INFINITY ? 0.f : m * to_log2;
    bf16x8 p, rest;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < 4; i += 2) {
        f32x2 x;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          x[u] = exp2_fast(fmaf(st[b][i + u], to_log2, -shift));
          sum += x[u];
          if constexpr (kFormat == NAT_KV_FP8) {
            const float scaled = x[u] * power_of_two((t.v_exp[b] >> (8 * (i + u))) & 0xff);
            x[u] = whole || st[b][i + u] != -INFINITY ? scaled : 0.f;       // the scale of a token that is not there may be anything
          }
        }
        const bf16x2 rounded = __builtin_convertvector(x, bf16x2);
        p[4 * b + i] = rounded[0];
        p[4 * b + i + 1] = rounded[1];
        if constexpr (kFormat == NAT_KV_FP4) {
          x[0] = __builtin_amdgcn_fdot2_f32_bf16(rounded, of_low, x[0], false);
          x[1] = __builtin_amdgcn_fdot2_f32_bf16(rounded, of_high, x[1], false);
          const bf16x2 left = __builtin_convertvector(x, bf16x2);
          (kHalves ? p : rest)[4 * b + i] = left[0];
          (kHalves ? p : rest)[4 * b + i + 1] = left[1];
        }
      }
#pragma unroll
    for (int db = 0; db < D / 16; ++db) {
      typedef short s16x8 __attribute__((ext_vector_type(8)));
      const int i = lane & 15;
      const s16x4 x = lds_transposed(vt + RowTile<D>::chunk_at(4 * g + (i >> 2), 2 * db + ((i & 3) >> 1)) + 8 * (i & 1));
      const s16x4 y = lds_transposed(vt + RowTile<D>::chunk_at(16 + 4 * g + (i >> 2), 2 * db + ((i & 3) >> 1)) + 8 * (i & 1));
      const s16x8 both = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
      acc[db] = mfma16x16(__builtin_bit_cast(bf16x8, both), p, acc[db]);
      if constexpr (kFormat == NAT_KV_FP4 && !kHalves) acc[db] = mfma16x16(__builtin_bit_cast(bf16x8, both), rest, acc[db]);
    }
  };
  TokenTile<D, kFormat> tiles[kTiles];
  int at = wave * kTokens;
  if (at < end) load(tiles[0], at);
  while (at < end) {
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
      if (at >= end) break;
      const int ahead = at + 4 * kTokens;
      if (kTiles > 1 && ahead < end) load(tiles[(i + 1) % kTiles], ahead);
      step(tiles[i], at, ahead);
      at += 4 * kTokens;
    }
  }

  // join the wavefronts: every one scales its result by the chunk's maximum, the sum of the four leaves
  sum = sum_groups(sum);
  if (g == 0) {
    wave_m[wave][n] = m;
    wave_sum[wave][n] = sum;
  }
  __syncthreads();
  float all_m = -INFINITY, all_sum = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) all_m = fmaxf(all_m, wave_m[w][n]);
  const float base = all_m == -INFINITY ? 0.f : all_m;       // (without any token, or if all scores are NaN: the sums then are 0, or NaN)
#pragma unroll
  for (int w = 0; w < 4; ++w) all_sum += wave_sum[w][n] * exp2_fast((wave_m[w][n] - base) * to_log2);
  const float f = exp2_fast((m - base) * to_log2);
  float* mine = (float*)values[wave];
#pragma unroll
  for (int db = 0; db < D / 16; ++db) *(f32x4*)(mine + n * D + 16 * db + 4 * g) = acc[db] * f;
  if (wave == 0 && g == 0) {
    joined_m[n] = all_m;
    joined_sum[n] = all_sum;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < heads_here * (D / 4); i += 256) {
    const int h = i / (D / 4), d = i % (D / 4) * 4;
    f32x4 x = {};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      x += *(const f32x4*)((const float*)values[w] + h * D + d);
      if constexpr (kHalves) x += *(const f32x4*)((const float*)values[w] + (h + kHeads / 2) * D + d);
    }
    const int64_t row = (int64_t)seq * a.hq + head0 + h;
    if (a.n_chunks > 1) {
      *(f32x4*)(a.part_out + (row * a.n_chunks + chunk) * D + d) = x;
      if (d == 0) *(f32x2*)(a.part_ml + (row * a.n_chunks + chunk) * 2) = f32x2{joined_m[h], joined_sum[h]};
    } else {
      const float total = joined_sum[h];
      *(bf16x4*)(a.out + seq * a.out_stride + (head0 + h) * D + d) = __builtin_convertvector(x * (total == 0.f ? 0.f : 1.f / total), bf16x4);
      if (d == 0) a.lse[row] = total == 0.f ? -INFINITY : fmaf(joined_m[h], a.scale, __logf(total));
    }
  }
}

// One workgroup per (sequence, query head): the chunks' results, scaled to their common maximum, over the sum of their sums.  Of up to kMaxJoinWaves wavefronts
// each takes kJoinChunks chunks at a time, whose loads are all under way before the maximum is known (28 heads of 128 chunks 4.5 us, with four
// wavefronts in turn 6.1; 4096 of up to 4 with one wavefront 6.1, with four 8.2).
constexpr int kJoinChunks = 8, kMaxJoinWaves = 16;
template <int D>
__global__ void __launch_bounds__(64 * kMaxJoinWaves) decode_join_kernel(DecodeArgs a) {
  __shared__ __attribute__((aligned(16))) float part[kMaxJoinWaves][D];
  __shared__ float part_sum[kMaxJoinWaves];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const int64_t row = blockIdx.x;
  const int seq = (int)(row / a.hq), qh = (int)(row % a.hq);
  const int len = length_of(a, seq), n = len > 0 ? (len + a.chunk - 1) / a.chunk : 1;
  const float* ml = a.part_ml + row * a.n_chunks * 2;
  const float* from = a.part_out + row * a.n_chunks * D + (2 * lane < D ? 2 * lane : 0);
  const float to_log2 = a.scale * kLog2E;
  f32x2 of[kJoinChunks], y[kJoinChunks];
  auto load = [&](int i0) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < kJoinChunks; ++u) {
      const int i = i0 + u * waves;
      of[u] = f32x2{-INFINITY, 0.f};
      y[u] = f32x2{};
      if (i < n) {
        of[u] = *(const f32x2*)(ml + 2 * i);
        y[u] = *(const f32x2*)(from + (int64_t)i * D);
      }
    }
  };
  load(wave);
  float m = -INFINITY;
  for (int i = lane; i < n; i += 64) m = fmaxf(m, ml[2 * i]);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) m = fmaxf(m, __shfl_xor(m, d, 64));
  const float shift = m == -INFINITY ? 0.f : m;
  float sum = 0.f;
  f32x2 x = {};
  for (int i = wave;;) {
#pragma unroll
    for (int u = 0; u < kJoinChunks; ++u) {
      const float f = exp2_fast((of[u][0] - shift) * to_log2);
      sum = fmaf(of[u][1], f, sum);
      x += y[u] * f;
    }
    i += kJoinChunks * waves;
    if (i >= n) break;
    load(i);
  }
  if (2 * lane < D) *(f32x2*)(part[wave] + 2 * lane) = x;
  if (lane == 0) part_sum[wave] = sum;
  __syncthreads();
  if (wave != 0) return;
  sum = 0.f;
  for (int w = 0; w < waves; ++w) sum += part_sum[w];
  if (4 * lane < D) {
    f32x4 z = {};
    for (int w = 0; w < waves; ++w) z += *(const f32x4*)(part[w] + 4 * lane);
    *(bf16x4*)(a.out + seq * a.out_stride + qh * D + 4 * lane) = __builtin_convertvector(z * (sum == 0.f ? 0.f : 1.f / sum), bf16x4);
  }
  if (lane == 0) a.lse[row] = sum == 0.f ? -INFINITY : fmaf(m, a.scale, __logf(sum));
}

bool misaligned(const void* p) { return ((uintptr_t)p & 15) != 0; }

nat_status cache_args(const nat_kv_cache* p, CacheArgs* c) {
  if (!p) return NAT_INVALID_ARG;
  if (p->format != NAT_KV_BF16 && p->format != NAT_KV_FP8 && p->format != NAT_KV_FP4) return NAT_UNSUPPORTED_DTYPE;
  if ((p->head_dim != 64 && p->head_dim != 128) || p->n_kv_heads <= 0 || p->n_kv_heads > 4096) return NAT_BAD_SHAPE;
  int log2 = 4;
  while (log2 < 8 && (1 << log2) != p->page_size) ++log2;
  if ((1 << log2) != p->page_size) return NAT_BAD_SHAPE;
  if (p->n_pages <= 0 || !p->d_k || !p->d_v || misaligned(p->d_k) || misaligned(p->d_v)) return NAT_INVALID_ARG;
  if (p->format != NAT_KV_BF16 && (!p->d_k_exp || !p->d_v_exp || misaligned(p->d_k_exp) || misaligned(p->d_v_exp))) return NAT_INVALID_ARG;
  *c = CacheArgs{(char*)p->d_k, (char*)p->d_v, p->d_k_exp, p->d_v_exp, p->n_pages, p->n_kv_heads, log2};
  return NAT_OK;
}

// row strides in elements, 0: rows back to back
bool stride_ok(int64_t s, int64_t row) { return s == 0 || (s >= row && s % 8 == 0 && s <= INT32_MAX); }

// Tokens per workgroup, of the longest length that the table allows: 4096 chunks in all, of 1024 tokens at least (the chip holds 512 workgroups at a time, the
// lengths of a batch differ, and short chunks even them out), or 512 chunks of 256 tokens at least (two steps of each wavefront), and never more than 4096 tokens.  256 sequences of
// 304 tokens (8 key heads of 128, 8-bit) take 45 us in one chunk each, 66 in two with the join; 8 of 4096 tokens 23 in chunks of 512, 25 of 256; lengths from 33 to 8192 in
// 128 sequences 101 us in four chunks each, 110 in two.
// From 4 bits, where a token is half as many bytes, 2048 tokens take the place of 1024: 128 sequences of up to 2048 (8 key heads of 128) 40.1 us, in two chunks each 45.5; with heads of 64 27.4
// and 31.6; of up to 8192 128.5 and 129.3; but 100 of up to 3000 55.4 and 52.9.
constexpr int kFewTokens = 1024;
int chunk_of(int64_t n_seqs, int64_t blocks, int64_t most, int64_t few) {
  auto min = [](int64_t x, int64_t y) { return x < y ? x : y; };
  auto max = [](int64_t x, int64_t y) { return x > y ? x : y; };
  const int64_t all = max(1, n_seqs * blocks), least = max(1, (most + kMaxChunk - 1) / kMaxChunk);
  const int64_t n = max(least, max(min(4096 / all, most / few), min((512 + all - 1) / all, most / kMinChunk)));
  return (int)max(kMinChunk, ((most + n - 1) / n + 127) / 128 * 128);
}

template <template <int, int> class Launch, int D, class... Args>
void by_format(int format, Args... args) {
  if (format == NAT_KV_FP8) Launch<D, NAT_KV_FP8>::go(args...);
  else if (format == NAT_KV_FP4) Launch<D, NAT_KV_FP4>::go(args...);
  else Launch<D, NAT_KV_BF16>::go(args...);
}
template <template <int, int> class Launch, class... Args>
void by_shape(int head_dim, int format, Args... args) {
  if (head_dim == 128) by_format<Launch, 128>(format, args...);
  else by_format<Launch, 64>(format, args...);
}
// (row, head) pairs, `per` to a workgroup of 256, in as few launches as have room for them
template <class Args>
void launch_rows(void (*kernel)(Args), Args a, int64_t per, hipStream_t s) {
  constexpr int64_t kMost = kMaxWorkItems / 256;
  const int64_t pairs = a.n_rows * a.c.hkv;
  for (a.first = 0; a.first < pairs; a.first += kMost * per) {
    const int64_t blocks = (pairs - a.first + per - 1) / per;
    kernel<<<(unsigned)(blocks < kMost ? blocks : kMost), 256, 0, s>>>(a);
  }
}
template <int D, int kFormat>
struct LaunchWrite {
  static void go(WriteArgs a, hipStream_t s) { launch_rows(kv_write_kernel<D, kFormat>, a, 256 / (D / 8), s); }
};
template <int D, int kFormat>
struct LaunchRead {
  static void go(ReadArgs a, hipStream_t s) { launch_rows(kv_read_kernel<D, kFormat>, a, kReadRows * (256 / (D / 8)), s); }
};
template <int D, int kFormat>
struct LaunchDecode {
  static void go(DecodeArgs a, hipStream_t s) {
    const unsigned blocks = (unsigned)((int64_t)a.n_seqs * a.n_chunks * a.c.hkv * a.head_blocks);
    if (kFormat == NAT_KV_FP4 && a.group <= kHeads / 2) decode_kernel<D, kFormat, kFormat == NAT_KV_FP4><<<blocks, 256, 0, s>>>(a);
    else decode_kernel<D, kFormat, false><<<blocks, 256, 0, s>>>(a);
  }
};

struct DecodePlan { int chunk, n_chunks, head_blocks, join_waves; };
bool decode_plan(int64_t n_seqs, int64_t hq, int64_t hkv, int64_t most, int64_t few, DecodePlan* p) {
  if (n_seqs * hq > INT32_MAX) return false;
  const int64_t group = hq / hkv;
  p->head_blocks = (int)((group + kHeads - 1) / kHeads);
  p->chunk = chunk_of(n_seqs, hkv * p->head_blocks, most, few);
  const int64_t n = most > 0 ? (most + p->chunk - 1) / p->chunk : 1;
  p->n_chunks = (int)n;
  p->join_waves = (int)(n > kJoinChunks * kMaxJoinWaves ? kMaxJoinWaves : (n + kJoinChunks - 1) / kJoinChunks);
  return n_seqs * n * hkv * p->head_blocks <= kMaxWorkItems / 256 && (n == 1 || n_seqs * hq <= kMaxWorkItems / (64 * p->join_waves));
}
bool decode_shape_ok(int32_t n_seqs, int32_t hq, int32_t hkv, int32_t head_dim, int64_t most) {
  return n_seqs >= 0 && (head_dim == 64 || head_dim == 128) && hkv > 0 && hkv <= 4096 && hq > 0 && hq <= 4096 && hq % hkv == 0 && most >= 0 &&
         most <= INT32_MAX - kMaxChunk;
}

}  // namespace
}  // namespace nat

using namespace nat;

extern "C" nat_status nat_kv_write(const nat_kv_cache* cache, const void* d_k, int64_t k_stride, const void* d_v, int64_t v_stride,
                                   const int64_t* d_slots, int64_t n_rows, void* stream) {
  WriteArgs a{};
  const nat_status st = cache_args(cache, &a.c);
  if (st != NAT_OK) return st;
  const int64_t row = (int64_t)cache->n_kv_heads * cache->head_dim;
  if (n_rows < 0) return NAT_INVALID_ARG;
  if (n_rows > INT32_MAX / cache->n_kv_heads || !stride_ok(k_stride, row) || !stride_ok(v_stride, row)) return NAT_BAD_SHAPE;
  if (n_rows == 0) return NAT_OK;
  if (!d_k || !d_v || !d_slots || misaligned(d_k) || misaligned(d_v)) return NAT_INVALID_ARG;
  a.k = (const uint16_t*)d_k;
  a.v = (const uint16_t*)d_v;
  a.k_stride = k_stride ? k_stride : row;
  a.v_stride = v_stride ? v_stride : row;
  a.n_rows = n_rows;
  a.slots = d_slots;
  hipStream_t s = (hipStream_t)stream;
  ProfScope prof(PC_KV_CACHE, s);
  by_shape<LaunchWrite>(cache->head_dim, cache->format, a, s);
  NAT_LAUNCH_CHECK();
  return NAT_OK;
}

extern "C" nat_status nat_kv_read(const nat_kv_cache* cache, const int32_t* d_block_table, int32_t table_width, const int32_t* d_cu_k,
                                  int32_t n_seqs, int64_t n_rows, void* d_k, int64_t k_stride, void* d_v, int64_t v_stride, void* stream) {
  ReadArgs a{};
  const nat_status st = cache_args(cache, &a.c);
  if (st != NAT_OK) return st;
  const int64_t row = (int64_t)cache->n_kv_heads * cache->head_dim;
  if (n_rows < 0 || n_seqs < 0 || table_width < 0) return NAT_INVALID_ARG;
  if (n_rows > INT32_MAX / cache->n_kv_heads || !stride_ok(k_stride, row) || !stride_ok(v_stride, row)) return NAT_BAD_SHAPE;
  if (n_rows == 0 || n_seqs == 0) return NAT_OK;
  if ((table_width > 0 && !d_block_table) || !d_cu_k || !d_k || !d_v || misaligned(d_k) || misaligned(d_v)) return NAT_INVALID_ARG;
  a.table = d_block_table;
  a.table_width = table_width;
  a.cu = d_cu_k;
  a.n_seqs = n_seqs;
  a.n_rows = n_rows;
  a.k = (uint16_t*)d_k;
  a.v = (uint16_t*)d_v;
  a.k_stride = k_stride ? k_stride : row;
  a.v_stride = v_stride ? v_stride : row;
  hipStream_t s = (hipStream_t)stream;
  ProfScope prof(PC_KV_CACHE, s);
  by_shape<LaunchRead>(cache->head_dim, cache->format, a, s);
  NAT_LAUNCH_CHECK();
  return NAT_OK;
}

extern "C" size_t nat_attn_decode_workspace_bytes(int32_t n_seqs, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int64_t max_tokens) {
  DecodePlan p;
  if (!decode_shape_ok(n_seqs, n_q_heads, n_kv_heads, head_dim, max_tokens) || n_seqs == 0 ||
      !decode_plan(n_seqs, n_q_heads, n_kv_heads, max_tokens, kFewTokens, &p) || p.n_chunks == 1)
    return 0;
  return ((size_t)n_seqs * n_q_heads * p.n_chunks * (head_dim + 2) * 4 + 255) / 256 * 256;
}

extern "C" nat_status nat_attn_decode(const nat_kv_cache* cache, const void* d_q, int64_t q_stride, int32_t n_seqs, int32_t n_q_heads,
                                      const int32_t* d_block_table, int32_t table_width, const int32_t* d_seq_lens, float scale, void* d_out,
                                      int64_t out_stride, float* d_lse, void* d_ws, size_t ws_bytes, void* stream) {
  DecodeArgs a{};
  const nat_status st = cache_args(cache, &a.c);
  if (st != NAT_OK) return st;
  if (n_seqs < 0 || table_width < 0 || !(scale > 0.f) || !(scale < INFINITY)) return NAT_INVALID_ARG;
  const int64_t most = (int64_t)table_width * cache->page_size, row = (int64_t)n_q_heads * cache->head_dim;
  DecodePlan p;
  if (!decode_shape_ok(n_seqs, n_q_heads, cache->n_kv_heads, cache->head_dim, most) || !stride_ok(q_stride, row) || !stride_ok(out_stride, row) ||
      !decode_plan(n_seqs, n_q_heads, cache->n_kv_heads, most, cache->format == NAT_KV_FP4 ? 2 * kFewTokens : kFewTokens, &p))
    return NAT_BAD_SHAPE;
  if (n_seqs == 0) return NAT_OK;
  if (!d_q || (table_width > 0 && !d_block_table) || !d_seq_lens || !d_out || !d_lse || misaligned(d_q) || misaligned(d_out)) return NAT_INVALID_ARG;
  const size_t need = nat_attn_decode_workspace_bytes(n_seqs, n_q_heads, cache->n_kv_heads, cache->head_dim, most);
  if (need > 0 && (!d_ws || ws_bytes < need)) return NAT_WORKSPACE_TOO_SMALL;
  if ((uintptr_t)d_ws & 255) return NAT_INVALID_ARG;
  a.q = (const uint16_t*)d_q;
  a.out = (uint16_t*)d_out;
  a.lse = d_lse;
  a.table = d_block_table;
  a.lens = d_seq_lens;
  a.table_width = table_width;
  a.n_seqs = n_seqs;
  a.hq = n_q_heads;
  a.group = n_q_heads / cache->n_kv_heads;
  a.head_blocks = p.head_blocks;
  a.chunk = p.chunk;
  a.n_chunks = p.n_chunks;
  a.q_stride = q_stride ? q_stride : row;
  a.out_stride = out_stride ? out_stride : row;
  a.scale = scale;
  a.part_out = (float*)d_ws;
  a.part_ml = a.part_out + (size_t)n_seqs * n_q_heads * p.n_chunks * cache->head_dim;
  hipStream_t s = (hipStream_t)stream;
  ProfScope prof(PC_ATTN_DECODE, s);
  by_shape<LaunchDecode>(cache->head_dim, cache->format, a, s);
  NAT_LAUNCH_CHECK();
  if (p.n_chunks == 1) return NAT_OK;
  if (cache->head_dim == 128) decode_join_kernel<128><<<(unsigned)(n_seqs * n_q_heads), 64 * p.join_waves, 0, s>>>(a);
  else decode_join_kernel<64><<<(unsigned)(n_seqs * n_q_heads), 64 * p.join_waves, 0, s>>>(a);
  NAT_LAUNCH_CHECK();
  return NAT_OK;
}
