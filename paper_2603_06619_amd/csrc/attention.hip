// Attention over packed sequences with grouped heads, forward and backward, bf16 on the matrix cores.
//
//   S_ij = scale q_i . k_j,  P_ij = exp(S_ij - lse_i),  lse_i = log sum_j exp(S_ij),  out_i = sum_j P_ij v_j       over the keys j that i sees
//   dP_ij = dout_i . v_j,  delta_i = dout_i . out_i,  dS_ij = P_ij (dP_ij - delta_i)
//   dq_i = scale sum_j dS_ij k_j,  dk_j = scale sum_i dS_ij q_i,  dv_j = sum_i P_ij dout_i
//
// The G query heads that share a key head are rows of one matrix: row r of a sequence is query r / G, head r % G of the group.
// A tile of rows then reads its keys once for all heads, covers few queries (so little of the causal mask's edge is computed in vain),
// and dk, dv of a shared head are plain sums over rows.  Every wavefront owns 32 rows (forward, dq) or 32 keys (dk, dv) as the columns of its
// products: a lane holds results of one column, so that row maxima and sums stay in the lane but for one exchange of the wavefront's halves, and the
// probabilities are the next product's operand without leaving the registers (mfma_tile.hip.h).
// Products take bf16: P and dS are rounded to it as they become operands, 2^-8 of each element at most, which adds 2-norm errors of about 1.7e-3 to
// results that are rounded by as much when they are stored.  Scores, statistics and sums stay in fp32.
// Nothing is added by atomics: results do not change from run to run.
//
// Long sequences run at the power limit of the package: a prompt of 16384 tokens (32 heads on 8 of 128 elements, causal) takes 2.0 ms, 1100 TFLOP/s, at a clock of 1.6
// of 2.4 GHz, where a library product of 8192^3 random bf16 numbers reaches 1370.
#include "nat_internal.h"
#include "mfma_tile.hip.h"

#include <type_traits>

namespace nat {
namespace {

constexpr float kLog2E = 1.4426950408889634f;
constexpr int kRowTile = 128;             // rows per workgroup: 4 wavefronts of 32
constexpr int kKeyTile = 64;              // keys per step of the forward and dq kernels
constexpr int kFewKeys = 64;              // see attn_dq_kernel
constexpr float kSlack = 8.f;             // see attn_fwd_kernel
constexpr int64_t kMaxStride = 1 << 24;   // elements: 64 rows are then within the 32-bit offsets of a buffer descriptor
constexpr int kDkvKeys = 128;             // keys per workgroup of the dk, dv kernel
constexpr int kDkvRows = 64;              // rows per step of it

struct AttnArgs {
  const uint16_t *q, *k, *v;
  uint16_t* out;
  float* lse;
  const int32_t *cu_q, *cu_k;
  int n_seqs, hq, hkv, group, causal;
  int64_t n_q, n_k, q_stride, k_stride, v_stride, out_stride;
  float scale;
  // backward
  const uint16_t* dout;
  float* delta;                  // [hq, n_q]
  uint16_t *dq, *dk, *dv;
  int64_t dout_stride, dq_stride, dk_stride, dv_stride;
  int slots;                     // tile slots per key head
  int row_parts;                 // dk, dv: workgroups that share a tile's rows
  int key_parts;                 // forward: workgroups that share a tile's keys
  float* parts;                  // what they leave if there are several: dk, dv [row_parts][n_k][hkv][2][D], or sums [key_parts][n_q][hq][D]
  float* part_ml;                // and m, sum [key_parts][n_q][hq][2]
  uint32_t group_inverse;        // see small_quotient
};

// x / group for 0 <= x < 2^13, group <= 2^12: floor((x + 1/2) / group), which lies 1 / (2 group) below the next whole number at least, and the inverse,
// floor(2^31 / group) + 1, adds (x + 1/2) / 2^31 at most
__device__ __forceinline__ int small_quotient(int x, uint32_t inverse) { return (int)__umulhi((uint32_t)(2 * x + 1), inverse); }

// Offsets come from device memory: clamped to the arrays, and a sequence never has a negative length.
__device__ __forceinline__ int64_t offset_at(const int32_t* cu, int i, int64_t n) {
  const int64_t c = cu[i];
  return c < 0 ? 0 : c < n ? c : n;
}

// Sequence of a slot.  Sequence b with `mult` rows per packed row owns the slots floor(cu[b] mult / tile) + b up to that of b + 1: at least as many as
// it has tiles, so a grid of floor(n mult / tile) + n_seqs slots needs no lengths on the host and the search no prefix sums.  The wavefront looks at 64
// sequences at a time.
__device__ __forceinline__ int sequence_of_slot(const int32_t* cu, int n_seqs, int64_t n, int mult, int tile, int64_t slot, int64_t* first) {
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = n_seqs;                // the last b in [lo, hi) with first(b) <= slot
  while (hi - lo > 1) {
    const int step = (hi - lo + 63) >> 6, b = lo + lane * step;
    const bool le = b < hi && offset_at(cu, b, n) * mult / tile + b <= slot;
    const int below = __popcll(__ballot(le));
    if (below == 0) break;
    const int next = lo + (below - 1) * step;
    hi = next + step < hi ? next + step : hi;
    lo = next;
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  *first = offset_at(cu, lo, n) * mult / tile + lo;
  return lo;
}

struct Sequence {
  int64_t q0, k0;                // first packed rows
  int n_q, n_k, ahead;           // lengths; query t sees the keys 0 .. t + ahead, or all
};
__device__ __forceinline__ Sequence sequence(const AttnArgs& a, int b) {
  Sequence s;
  // the same for all lanes, and said so: what is made of them stays in scalar registers
  auto at = [](const int32_t* cu, int i, int64_t n) { return (int64_t)__builtin_amdgcn_readfirstlane((int)offset_at(cu, i, n)); };
  s.q0 = at(a.cu_q, b, a.n_q);
  s.k0 = at(a.cu_k, b, a.n_k);
  const int64_t q1 = at(a.cu_q, b + 1, a.n_q), k1 = at(a.cu_k, b + 1, a.n_k);
  s.n_q = q1 > s.q0 ? (int)(q1 - s.q0) : 0;
  s.n_k = k1 > s.k0 ? (int)(k1 - s.k0) : 0;
  s.ahead = s.n_k - s.n_q;
  return s;
}
// last key that query t sees (below 0: none)
__device__ __forceinline__ int last_key(const AttnArgs& a, const Sequence& s, int t) {
  const int l = a.causal ? t + s.ahead : s.n_k - 1;
  return l < s.n_k ? l : s.n_k - 1;
}

// Block id -> (key head, slot).  Blocks are dealt to the 8 XCDs in turn: those of one key head go to as few XCDs as possible, whose L2 then
// holds its keys and values.  Where the number of heads and 8 do not divide each other the heads just alternate.
__device__ __forceinline__ void head_and_slot(int id, int heads, int slots, int& head, int& slot) {
  if (heads % 8 == 0) {
    const int at = id >> 3;
    head = (id & 7) + 8 * (at / slots);
    slot = at % slots;
  } else if (8 % heads == 0) {
    const int per = 8 / heads;
    head = (id & 7) % heads;
    slot = (id >> 3) * per + (id & 7) / heads;       // the grid is a whole number of 8: may pass the end
  } else {
    head = id % heads;
    slot = id / heads;
  }
}
unsigned grid_of(int heads, int64_t slots) {
  return (unsigned)((heads % 8 != 0 && 8 % heads == 0) ? (slots * heads + 7) / 8 * 8 : slots * heads);
}

// A tile of kRows rows of D elements, copied to LDS without passing registers: one instruction writes 1 KB, lane l's 16 bytes at 16 l, and every lane reads from
// where its place of the permuted tile wants it.  The copies go through a buffer descriptor of the rows that there are: what lies behind them (behind a
// sequence's end) arrives as zeros by the hardware's bounds check and never meets a product.
typedef int i32x4 __attribute__((ext_vector_type(4)));
template <int D, int kRows>
struct TileCopy {
  static constexpr int kLanes = D / 8, kRowsPerCopy = 64 / kLanes, kCopies = kRows / kRowsPerCopy / 4;      // per wavefront, of four
  static __device__ __forceinline__ int row_of(int lane, int wave, int i) { return (wave * kCopies + i) * kRowsPerCopy + lane / kLanes; }
  static __device__ __forceinline__ int column_of(int lane, int row) { return ((lane % kLanes) ^ RowTile<D>::swizzle(row)) * 16; }
  // As inline assembly, which the compiler's wait counts do not see: of copies that it knows of, it would wait for all in front of every transposing read,
  // whatever either's place.  A copy has no result in registers; end_of_step() waits for them.  Nor does the compiler see what must lie in front of it: 5 wait
  // states behind a vector instruction that wrote `rows` (a spilled scalar register comes back that way), 1 behind the write of m0
  static __device__ __forceinline__ void copy(i32x4 rows, int offset, char* tile, int wave, int i) {
    const uint32_t to = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)(tile + (wave * kCopies + i) * 1024);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" : : "s"(to), "v"(offset), "s"(rows) : "memory", "m0");
  }
  static __device__ __forceinline__ i32x4 rows_at(const char* base, int bytes) {
    const uint64_t at = (uint64_t)(uintptr_t)base;
    return i32x4{(int)(uint32_t)at, (int)((uint32_t)(at >> 32) & 0xffff), bytes, 0x00027000};
  }
  // `rows` rows from `base` on (more than kRows: kRows), row_bytes apart
  static __device__ __forceinline__ void fetch(const char* base, int row_bytes, int rows, char* tile, int lane, int wave) {
    const i32x4 r = rows_at(base, rows > 0 ? ((rows < kRows ? rows : kRows) - 1) * row_bytes + D * 2 : 0);
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
      const int row = row_of(lane, wave, i);
      copy(r, row * row_bytes + column_of(lane, row), tile, wave, i);
    }
  }
  // rows of a group's matrix: `rows` of them (more than kRows: kRows; fewer: they end with a query) from head `head` of the query at `base` on
  static __device__ __forceinline__ void fetch_grouped(const char* base, int row_bytes, int group, uint32_t group_inverse, int head, int rows, char* tile, int lane,
                                                       int wave) {
    const int live = rows < kRows ? rows : kRows;
    const i32x4 r = rows_at(base, live > 0 ? small_quotient(head + live - 1, group_inverse) * row_bytes + group * D * 2 : 0);
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
      const int row = row_of(lane, wave, i), at = head + row, t = small_quotient(at, group_inverse);
      copy(r, t * row_bytes + (at - t * group) * (D * 2) + column_of(lane, row), tile, wave, i);
    }
  }
};
// The copies of this step have arrived, and all are done with the step's tiles.
__device__ __forceinline__ void end_of_step() {
  __builtin_amdgcn_s_waitcnt(0x0f70);        // vmcnt(0)
  __syncthreads();
}

// Where a mask cuts through a tile, a product multiplies masked rows by 0, and infinities or NaN in them come through as NaN.  Results that are not finite
// are therefore computed once more, carefully: at the mask's edge the product with P or dS gets zeros in the places of such elements (the tile stays as it is: scores
// and dP, whose masked elements are set, are made of it), and the columns that see them have them added by hand.  P has no sign: what it multiplies is
// added itself.  An element of k or q that is not finite makes its scores infinite, and P 0 or NaN: what dS multiplies (kNan) gives NaN.
template <int D, int kRows, bool kNan, class Sees>
__device__ __forceinline__ void add_not_finite(const char* tile, f32x16 (&acc)[D / 32], int half, const Sees& sees) {
  for (int row = 0; row < kRows; ++row) {
    if (!sees(row)) continue;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint16_t* x = (const uint16_t*)(tile + RowTile<D>::chunk_at(row, 4 * db + i) + 8 * half);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if ((x[e] & 0x7f80) == 0x7f80) acc[db][4 * i + e] += kNan ? NAN : __builtin_bit_cast(float, (uint32_t)x[e] << 16);
      }
  }
}
// transposed_fragment, with zeros in those places if `edge`
template <int D>
__device__ __forceinline__ bf16x8 finite_fragment(const char* tile, int lane, int db, int s, bool edge) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  u32x4 x = __builtin_bit_cast(u32x4, transposed_fragment<D>(tile, lane, db, s));
  const uint32_t keep = edge ? 0u : ~0u;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if ((x[i] & 0x7f80) == 0x7f80) x[i] &= 0xffff0000 | keep;
    if ((x[i] & 0x7f800000) == 0x7f800000) x[i] &= 0xffff | keep;
  }
  return __builtin_bit_cast(bf16x8, x);
}

template <int D>
struct RowFragments {            // 32 rows as an operand, one row per lane, in registers
  bf16x8 f[D / 16];
  __device__ __forceinline__ void load(const uint16_t* row, int lane) {
#pragma unroll
    for (int s = 0; s < D / 16; ++s) f[s] = *(const bf16x8*)(row + 16 * s + 8 * (lane >> 5));
  }
};

// the same for all lanes: kept in a scalar register
__device__ __forceinline__ float uniform(float x) { return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, x))); }

template <int D>
__device__ __forceinline__ bool not_finite(const f32x16 (&acc)[D / 32]) {
  float x = 0.f;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) x += acc[db][i];
  return !(fabsf(x) < INFINITY);             // (sums that overflow are looked at again too)
}

// C[32 rb ..][n] = rows of a tile of 64 rows times the columns b: fragments are read four at a time while the four before them are multiplied (the
// compiler by itself reads one and waits for it).  beside(i), i = 0 .. D / 32 - 1, is work to be done under the products.
template <int D, class Beside>
__device__ __forceinline__ void tile_times_columns(const char* tile, const bf16x8 (&b)[D / 16], f32x16 (&c)[2], int lane, const Beside& beside) {
  constexpr int kSteps = D / 16, kGroups = 2 * kSteps / 4;
  bf16x8 f[2][4];
#pragma unroll
  for (int i = 0; i < 4; ++i) f[0][i] = row_fragment<D>(tile, lane, i / kSteps, i % kSteps);
#pragma unroll
  for (int g = 0; g < kGroups; ++g) {
    if (g + 1 < kGroups) {
#pragma unroll
      for (int i = 0; i < 4; ++i) f[(g + 1) & 1][i] = row_fragment<D>(tile, lane, (4 * g + 4 + i) / kSteps, (4 * g + 4 + i) % kSteps);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int at = 4 * g + i;
      c[at / kSteps] = mfma32(f[g & 1][i], b[at % kSteps], c[at / kSteps]);
    }
    beside(g);
    __builtin_amdgcn_sched_barrier(0);
  }
}

template <int D>
__device__ __forceinline__ void tile_times_columns(const char* tile, const bf16x8 (&b)[D / 16], f32x16 (&c)[2], int lane) {
  tile_times_columns<D>(tile, b, c, lane, [](int) __attribute__((always_inline)) {});
}

// Columns of a result, 32 elements db of this lane's column n, as bf16 to its row
template <int D>
__device__ __forceinline__ void store_columns(uint16_t* row, const f32x16 (&acc)[D / 32], float factor, int lane) {
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x4 x = {acc[db][4 * i] * factor, acc[db][4 * i + 1] * factor, acc[db][4 * i + 2] * factor, acc[db][4 * i + 3] * factor};
      *(bf16x4*)(row + 32 * db + 8 * i + 4 * (lane >> 5)) = __builtin_convertvector(x, bf16x4);
    }
}

// out and lse.  A step takes 64 keys: with their values twice in LDS (64 KB at D = 128) two workgroups share a compute unit, and one's exponentials run beside
// the other's products.  At D = 128 a step is 32 products (1024 cycles) and 32 exponentials with some 120 other vector instructions (about 980 cycles) per
// wavefront: either pipe would be full at 1.7 times the speed, the power limit comes first (matrix pipes 58 % busy).  At D = 64 the vector instructions are twice the
// products: 4 x 4096 tokens of 16 heads 186 us, 740 TFLOP/s.  For the prompt of 16384 tokens, this 2.0 to 2.1 ms:
// 64 rows per wavefront with half the wavefronts 3.1, the next tile's products among this tile's exponentials 2.03, 8 wavefronts per workgroup 2.01 (701 tokens
// behind 4093 cached ones 177 us instead of 147), copies three tiles ahead 2.07.  Calls of short prompts (48 of up to 193 tokens, 16 heads on 8 of 64) are a chain of
// loads, which four workgroups per compute unit share better than three: 14.4 us, 15.7 (and 128 registers suffice).  Of a
// workgroup's 7 us 1.8 are offsets and lengths, 1.1 queries and first tile, 2.9 its 1 to 4 steps, 1.1 the stores.
// The careful pass, inlined, costs 106 spilled scalar registers at D = 128 (none at D = 64): the prompt takes 2.10 ms, without it 2.07, the 701 tokens 151 and 147 us, the
// short prompts 13.65 and 13.45.
// kSplit: key_parts workgroups share a tile's keys and leave their sums for attn_fwd_join_kernel (a kernel of its own: both in
// one take 32 registers more).
template <int D, bool kSplit>
__global__ void __launch_bounds__(256, D == 64 ? 4 : 2) attn_fwd_kernel(AttnArgs a) {
  __shared__ __attribute__((aligned(16))) char tiles[2][2][kKeyTile * D * 2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
  int head, slot;
  const int parts = kSplit ? a.key_parts : 1;
  head_and_slot(blockIdx.x, a.hkv, a.slots * parts, head, slot);
  const int part = slot % parts;
  slot /= parts;
  if (slot >= a.slots) return;
  slot = a.slots - 1 - slot;                 // causal: the last tiles of a sequence have the most keys, and go first
  int64_t first_slot;
  const Sequence s = sequence(a, sequence_of_slot(a.cu_q, a.n_seqs, a.n_q, a.group, kRowTile, slot, &first_slot));
  const int n_rows = s.n_q * a.group, tile_row = (int)(slot - first_slot) * kRowTile;
  if (slot < first_slot || tile_row >= n_rows) return;

  const int row = tile_row + wave * 32 + (lane & 31), safe_row = row < n_rows ? row : n_rows - 1;
  const int query = safe_row / a.group, of_group = safe_row - query * a.group;
  RowFragments<D> q;
  q.load(a.q + (s.q0 + query) * a.q_stride + (head * a.group + of_group) * D, lane);
  const int tile_end = tile_row + kRowTile < n_rows ? tile_row + kRowTile : n_rows;
  const int n_keys = last_key(a, s, (tile_end - 1) / a.group) + 1;      // of the tile
  int first_key = 0, end_key = n_keys;                                 // of this part
  if (kSplit) {
    const int steps = ((n_keys + kKeyTile - 1) / kKeyTile + parts - 1) / parts;
    first_key = part * steps * kKeyTile;
    end_key = n_keys - first_key > steps * kKeyTile ? first_key + steps * kKeyTile : n_keys;
  }
  const int last = last_key(a, s, query);                              // of this lane's row
  const int wave_row = tile_row + wave * 32 < n_rows ? tile_row + wave * 32 : n_rows - 1, wave_end = wave_row + 32 < n_rows ? wave_row + 32 : n_rows;
  const int wave_least = last_key(a, s, wave_row / a.group);           // keys up to here are seen by all rows of the wavefront
  const int wave_last = last_key(a, s, (wave_end - 1) / a.group);
  const char *k = (const char*)(a.k + s.k0 * a.k_stride + head * D), *v = (const char*)(a.v + s.k0 * a.v_stride + head * D);
  const int k_bytes = (int)a.k_stride * 2, v_bytes = (int)a.v_stride * 2;

  const float to_log2 = uniform(a.scale * kLog2E);
  // What exponents are shifted by, and the sum (of this lane's half).  m follows the maximum of q.k only when that has grown by a factor of 2^kSlack in the
  // exponentials: they and their sums have room for it, and the results are seldom scaled
  float m, sum;
  const float slack = uniform(fminf(kSlack / to_log2, __FLT_MAX__));       // (finite: m leaves -inf whatever the scale)
  f32x16 acc[D / 32];
  const char *next_k, *next_v;
  auto fetch = [&](int key0, char (&to)[2][kKeyTile * D * 2]) __attribute__((always_inline)) {
    TileCopy<D, kKeyTile>::fetch(next_k, k_bytes, n_keys - key0, to[0], lane, wave);
    TileCopy<D, kKeyTile>::fetch(next_v, v_bytes, n_keys - key0, to[1], lane, wave);
    next_k += (int64_t)kKeyTile * k_bytes;
    next_v += (int64_t)kKeyTile * v_bytes;
  };
  auto step = [&](int key0, char* kt, char* vt, auto careful) __attribute__((always_inline)) {
    constexpr bool kCareful = decltype(careful)::value;
    const bool edge = kCareful && key0 + kKeyTile - 1 > wave_least;
    if (key0 > wave_last) return;
    f32x16 st[2] = {};
    tile_times_columns<D>(kt, q.f, st, lane);
    if (key0 + kKeyTile - 1 > wave_least) {
#pragma unroll
      for (int rb = 0; rb < 2; ++rb)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (key0 + 32 * rb + result_row(i, half) > last) st[rb][i] = -INFINITY;
    }
    float top = m;
#pragma unroll
    for (int rb = 0; rb < 2; ++rb)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, st[rb][i]);
    top = max_halves(top);
    const bool grown = top > m + slack;
    if (__any(grown)) {                      // each row by its own: what its neighbours hold does not change its rounding
      const float f = grown ? exp2_fast((m - top) * to_log2) : 1.f;
      sum *= f;
#pragma unroll
      for (int db = 0; db < D / 32; ++db) acc[db] *= f;
      m = grown ? top : m;
    }
    const float shift = m == -INFINITY ? 0.f : m * to_log2;
    // probabilities of 16 keys at a time, while those of the 16 before them are multiplied
    bf16x8 p[2], vf[2][D / 32];
    auto ready = [&](int g) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int e = 8 * (g & 1) + i;
        st[g >> 1][e] = exp2_fast(fmaf(st[g >> 1][e], to_log2, -shift));
        sum += st[g >> 1][e];
      }
      p[g & 1] = fragment_of_result(st[g >> 1], g & 1);
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
        if constexpr (!kCareful) vf[g & 1][db] = transposed_fragment<D>(vt, lane, db, g);
    };
    ready(0);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      if (g < 3) ready(g + 1);
#pragma unroll
      for (int db = 0; db < D / 32; ++db) {
        if constexpr (kCareful) acc[db] = mfma32(finite_fragment<D>(vt, lane, db, g, edge), p[g & 1], acc[db]);
        else acc[db] = mfma32(vf[g & 1][db], p[g & 1], acc[db]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    // behind the step's scaling of what was summed before: by 0 in the first tile
    if (edge) add_not_finite<D, kKeyTile, false>(vt, acc, half, [&](int i) { return key0 + i <= last; });
  };
  auto pass = [&](auto careful) __attribute__((always_inline)) {
    m = -INFINITY;
    sum = 0.f;
#pragma unroll
    for (int db = 0; db < D / 32; ++db) acc[db] = f32x16{};
    next_k = k + (int64_t)first_key * k_bytes;
    next_v = v + (int64_t)first_key * v_bytes;
    fetch(first_key, tiles[0]);
    end_of_step();
    for (int key0 = first_key; key0 < end_key; key0 += 2 * kKeyTile) {
      if (key0 + kKeyTile < end_key) fetch(key0 + kKeyTile, tiles[1]);
      step(key0, tiles[0][0], tiles[0][1], careful);
      end_of_step();
      if (key0 + kKeyTile >= end_key) break;
      if (key0 + 2 * kKeyTile < end_key) fetch(key0 + 2 * kKeyTile, tiles[0]);
      step(key0 + kKeyTile, tiles[1][0], tiles[1][1], careful);
      end_of_step();
    }
  };
  pass(std::false_type{});
  if (__syncthreads_or(not_finite<D>(acc))) pass(std::true_type{});
  sum = sum_halves(sum);
  int thread = threadIdx.x;
  if (D == 64) asm volatile("" : "+v"(thread));          // row, query and head anew, not kept in registers all the while
  const int out_row = tile_row + (thread >> 6) * 32 + (thread & 31), out_query = out_row / a.group;
  if (out_row >= n_rows) return;
  const int64_t at = s.q0 + out_query;
  const int qh = head * a.group + out_row - out_query * a.group;
  if (kSplit) {
    const int64_t of_part = (part * a.n_q + at) * a.hq + qh;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *(f32x4*)(a.parts + of_part * D + 32 * db + 8 * i + 4 * half) = f32x4{acc[db][4 * i], acc[db][4 * i + 1], acc[db][4 * i + 2], acc[db][4 * i + 3]};
    if (half == 0) *(f32x2*)(a.part_ml + of_part * 2) = f32x2{m, sum};
    return;
  }
  store_columns<D>(a.out + at * a.out_stride + qh * D, acc, sum == 0.f ? 0.f : 1.f / sum, lane);
  // a row that sees nothing has the sum 0; one of NaN scores, whose maximum is -inf as well, NaN
  if (half == 0) a.lse[qh * a.n_q + at] = sum == 0.f ? -INFINITY : fmaf(m, a.scale, __logf(sum));
}

// Results of a tile's rows from those of its key_parts workgroups, scaled to their common maximum; two rows per wavefront, all loads of a row under way at once
constexpr int kMaxKeyParts = 16, kJoinRows = 8;
template <int D>
__global__ void __launch_bounds__(256) attn_fwd_join_kernel(AttnArgs a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int head, slot;
  head_and_slot(blockIdx.x, a.hkv, a.slots, head, slot);
  if (slot >= a.slots) return;
  int64_t first_slot;
  const Sequence s = sequence(a, sequence_of_slot(a.cu_q, a.n_seqs, a.n_q, a.group, kRowTile, slot, &first_slot));
  const int n_rows = s.n_q * a.group, tile_row = (int)(slot - first_slot) * kRowTile;
  if (slot < first_slot) return;
  const float to_log2 = a.scale * kLog2E;
  for (int row = tile_row + blockIdx.y * kJoinRows + wave; row < tile_row + (blockIdx.y + 1) * kJoinRows && row < n_rows; row += 4) {
    const int query = row / a.group, qh = head * a.group + row - query * a.group;
    const int64_t at = s.q0 + query, of = at * a.hq + qh, part_stride = a.n_q * a.hq;
    f32x2 ml[kMaxKeyParts], y[kMaxKeyParts];
#pragma unroll
    for (int p = 0; p < kMaxKeyParts; ++p) {
      ml[p] = f32x2{-INFINITY, 0.f};
      y[p] = f32x2{};
      if (p < a.key_parts) {
        ml[p] = *(const f32x2*)(a.part_ml + (of + p * part_stride) * 2);
        if (2 * lane < D) y[p] = *(const f32x2*)(a.parts + (of + p * part_stride) * D + 2 * lane);
      }
    }
    float m = -INFINITY, sum = 0.f;
#pragma unroll
    for (int p = 0; p < kMaxKeyParts; ++p) m = fmaxf(m, ml[p][0]);
    const float shift = m == -INFINITY ? 0.f : m;
    f32x2 x = {};
#pragma unroll
    for (int p = 0; p < kMaxKeyParts; ++p) {
      const float f = exp2_fast((ml[p][0] - shift) * to_log2);
      sum = fmaf(ml[p][1], f, sum);
      x += y[p] * f;
    }
    if (2 * lane < D) *(bf16x2*)(a.out + at * a.out_stride + qh * D + 2 * lane) = __builtin_convertvector(x * (sum == 0.f ? 0.f : 1.f / sum), bf16x2);
    if (lane == 0) a.lse[qh * a.n_q + at] = sum == 0.f ? -INFINITY : fmaf(m, a.scale, __logf(sum));
  }
}

enum class Pass { kDelta, kPlain, kCareful };

// dq, and delta for the dk, dv kernel behind it.  delta = dout . out takes `out` as it was rounded, which for rows of few keys is an error that dq does not
// average out (of the 2-norm about 1.7e-3 / sqrt(keys), where the rounding of dS is 1.7e-3; a single such row a few per cent).  Tiles with a row of fewer than
// kFewKeys keys go over their keys once more for it: delta = sum_j P_ij dP_ij.
// Tiles as in the forward kernel, three products of equal size instead of two; 8 rollouts of up to 4096 tokens (32 heads on 8 of 128) 645 us, 1000 TFLOP/s.  The
// exponentials under the products of dP, as in the kernel below, would want 58 registers more than two wavefronts per SIMD have: 845 us.  As it is, all 256 are
// in use at D = 128, 26 more and 77 scalar ones are spilled (without the careful pass 4 and none; the two backward kernels and the forward one then take 2080 us instead of
// 2170 to 2210).
template <int D>
__global__ void __launch_bounds__(256, 2) attn_dq_kernel(AttnArgs a) {
  __shared__ __attribute__((aligned(16))) char tiles[2][2][kKeyTile * D * 2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
  int head, slot;
  head_and_slot(blockIdx.x, a.hkv, a.slots, head, slot);
  if (slot >= a.slots) return;
  slot = a.slots - 1 - slot;
  int64_t first_slot;
  const Sequence s = sequence(a, sequence_of_slot(a.cu_q, a.n_seqs, a.n_q, a.group, kRowTile, slot, &first_slot));
  const int n_rows = s.n_q * a.group, tile_row = (int)(slot - first_slot) * kRowTile;
  if (slot < first_slot || tile_row >= n_rows) return;

  const int row = tile_row + wave * 32 + (lane & 31), safe_row = row < n_rows ? row : n_rows - 1;
  const int query = safe_row / a.group, of_group = safe_row - query * a.group;
  const int64_t at = s.q0 + query;
  const int qh = head * a.group + of_group;
  RowFragments<D> q, d;
  q.load(a.q + at * a.q_stride + qh * D, lane);
  d.load(a.dout + at * a.dout_stride + qh * D, lane);
  float delta = 0.f;
  {
    RowFragments<D> o;
    o.load(a.out + at * a.out_stride + qh * D, lane);
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) delta = fmaf((float)o.f[i][e], (float)d.f[i][e], delta);
    delta = sum_halves(delta);
  }
  const int tile_end = tile_row + kRowTile < n_rows ? tile_row + kRowTile : n_rows;
  const int n_keys = last_key(a, s, (tile_end - 1) / a.group) + 1, tile_least = last_key(a, s, tile_row / a.group);
  const int last = last_key(a, s, query);
  const int wave_row = tile_row + wave * 32 < n_rows ? tile_row + wave * 32 : n_rows - 1, wave_end = wave_row + 32 < n_rows ? wave_row + 32 : n_rows;
  const int wave_least = last_key(a, s, wave_row / a.group), wave_last = last_key(a, s, (wave_end - 1) / a.group);
  const char *k = (const char*)(a.k + s.k0 * a.k_stride + head * D), *v = (const char*)(a.v + s.k0 * a.v_stride + head * D);
  const int k_bytes = (int)a.k_stride * 2, v_bytes = (int)a.v_stride * 2;
  const float to_log2 = a.scale * kLog2E, lse = a.lse[qh * a.n_q + at], shift = lse == -INFINITY ? INFINITY : lse * kLog2E;

  f32x16 acc[D / 32];
  const char *next_k, *next_v;
  auto fetch = [&](int key0, char (&to)[2][kKeyTile * D * 2]) __attribute__((always_inline)) {
    TileCopy<D, kKeyTile>::fetch(next_k, k_bytes, n_keys - key0, to[0], lane, wave);
    TileCopy<D, kKeyTile>::fetch(next_v, v_bytes, n_keys - key0, to[1], lane, wave);
    next_k += (int64_t)kKeyTile * k_bytes;
    next_v += (int64_t)kKeyTile * v_bytes;
  };
  float p_sum = 0.f, p_dp = 0.f;
  auto step = [&](int key0, char* kt, char* vt, auto kind) __attribute__((always_inline)) {
    constexpr Pass kPass = decltype(kind)::value;
    const bool edge = kPass == Pass::kCareful && key0 + kKeyTile - 1 > wave_least;
    if (key0 > wave_last) return;
    if (edge) add_not_finite<D, kKeyTile, true>(kt, acc, half, [&](int i) { return key0 + i <= last; });
    f32x16 st[2] = {}, dp[2] = {};
    tile_times_columns<D>(kt, q.f, st, lane);
    tile_times_columns<D>(vt, d.f, dp, lane);
    if (key0 + kKeyTile - 1 > wave_least) {
#pragma unroll
      for (int rb = 0; rb < 2; ++rb)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (key0 + 32 * rb + result_row(i, half) > last) {
            st[rb][i] = -INFINITY;
            dp[rb][i] = 0.f;
          }
    }
    if constexpr (kPass == Pass::kDelta) {
#pragma unroll
      for (int rb = 0; rb < 2; ++rb)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float p = exp2_fast(fmaf(st[rb][i], to_log2, -shift));
          p_sum += p;
          p_dp = fmaf(p, dp[rb][i], p_dp);
        }
    } else {
      bf16x8 p[2], kf[2][D / 32];
      auto ready = [&](int g) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int e = 8 * (g & 1) + i;
          st[g >> 1][e] = exp2_fast(fmaf(st[g >> 1][e], to_log2, -shift)) * (dp[g >> 1][e] - delta);
        }
        p[g & 1] = fragment_of_result(st[g >> 1], g & 1);
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
          if constexpr (kPass != Pass::kCareful) kf[g & 1][db] = transposed_fragment<D>(kt, lane, db, g);
      };
      ready(0);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        if (g < 3) ready(g + 1);
#pragma unroll
        for (int db = 0; db < D / 32; ++db) {
          if constexpr (kPass == Pass::kCareful) acc[db] = mfma32(finite_fragment<D>(kt, lane, db, g, edge), p[g & 1], acc[db]);
          else acc[db] = mfma32(kf[g & 1][db], p[g & 1], acc[db]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  auto pass = [&](auto kind) __attribute__((always_inline)) {
#pragma unroll
    for (int db = 0; db < D / 32; ++db) acc[db] = f32x16{};
    next_k = k;
    next_v = v;
    fetch(0, tiles[0]);
    end_of_step();
    for (int key0 = 0; key0 < n_keys; key0 += 2 * kKeyTile) {
      if (key0 + kKeyTile < n_keys) fetch(key0 + kKeyTile, tiles[1]);
      step(key0, tiles[0][0], tiles[0][1], kind);
      end_of_step();
      if (key0 + kKeyTile >= n_keys) break;
      if (key0 + 2 * kKeyTile < n_keys) fetch(key0 + 2 * kKeyTile, tiles[0]);
      step(key0 + kKeyTile, tiles[1][0], tiles[1][1], kind);
      end_of_step();
    }
  };
  if (tile_least < kFewKeys - 1) {
    pass(std::integral_constant<Pass, Pass::kDelta>{});
    p_sum = sum_halves(p_sum);
    delta = p_sum > 0.f ? sum_halves(p_dp) / p_sum : 0.f;
  }
  pass(std::integral_constant<Pass, Pass::kPlain>{});
  if (__syncthreads_or(not_finite<D>(acc))) pass(std::integral_constant<Pass, Pass::kCareful>{});
  if (row >= n_rows) return;
  if (half == 0) a.delta[qh * a.n_q + at] = delta;
  store_columns<D>(a.dq + at * a.dq_stride + qh * D, acc, a.scale, lane);
}

// dk and dv.  A wavefront holds 32 keys and their values as operands and 32 x 2 D sums, and goes over the rows that see them, 64 at a time: four products of equal
// size (four reads of a tile per wavefront, as many cycles of LDS as of products).  At D = 128 these are 192 registers before the scores: one wavefront per
// SIMD, so the work under the products has to come from itself, and a step is one block but for the mask's edge (a branch among the exponentials: 1300 us
// instead of 1140, for 8 rollouts of up to 4096 tokens; 750 TFLOP/s, this at 1.6 GHz).  At D = 64 two fit: 16 rollouts of up to 311 tokens 19.6 us, with one 27.0; 4 of 4096,
// with dq, 554 and 645.  The careful pass, inlined, costs 121 spilled scalar registers at D = 128, 11 at D = 64.
// Where there are few tiles of keys for the chip their rows are cut into row_parts ranges, one workgroup each, whose sums go to memory in fp32 and are added in order by
// attn_dkv_join_kernel (backward of 1024 tokens, 32 heads on 8: 172 us, then 94; of 2048, 2 heads on 1: 185, then 87).
template <int D>
__global__ void __launch_bounds__(256, D == 64 ? 2 : 1) attn_dkv_kernel(AttnArgs a) {
  struct RowWords { float shift[kDkvRows], delta[kDkvRows]; int last[kDkvRows]; };
  __shared__ __attribute__((aligned(16))) char tiles[2][2][kDkvRows * D * 2];
  __shared__ __attribute__((aligned(16))) RowWords words[2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
  int head, slot;
  head_and_slot(blockIdx.x, a.hkv, a.slots * a.row_parts, head, slot);
  const int part = slot % a.row_parts;
  slot /= a.row_parts;
  if (slot >= a.slots) return;
  int64_t first_slot;
  const Sequence s = sequence(a, sequence_of_slot(a.cu_k, a.n_seqs, a.n_k, 1, kDkvKeys, slot, &first_slot));
  const int tile_key = (int)(slot - first_slot) * kDkvKeys;
  if (slot < first_slot || tile_key >= s.n_k) return;

  const int key = tile_key + wave * 32 + (lane & 31), safe_key = key < s.n_k ? key : s.n_k - 1;
  RowFragments<D> k, v;
  k.load(a.k + (s.k0 + safe_key) * a.k_stride + head * D, lane);
  v.load(a.v + (s.k0 + safe_key) * a.v_stride + head * D, lane);
  const int n_rows = s.n_q * a.group, wave_key = tile_key + wave * 32;
  // the first row that sees the tile's first key
  const int first_query = a.causal && tile_key > s.ahead ? tile_key - s.ahead : 0;
  const int seen_from = first_query < s.n_q ? first_query * a.group : n_rows;
  const int part_steps = ((n_rows - seen_from + kDkvRows - 1) / kDkvRows + a.row_parts - 1) / a.row_parts;
  const int first_row = seen_from + part * part_steps * kDkvRows, end_row = n_rows - first_row > part_steps * kDkvRows ? first_row + part_steps * kDkvRows : n_rows;
  const int wave_first = a.causal ? wave_key - s.ahead : 0;            // the first query that sees the wavefront's first key
  const int wave_all = a.causal ? wave_key + 31 - s.ahead : 0;         // queries from here on see all its keys
  const char *q = (const char*)(a.q + s.q0 * a.q_stride + head * a.group * D), *d = (const char*)(a.dout + s.q0 * a.dout_stride + head * a.group * D);
  const int q_bytes = (int)a.q_stride * 2, d_bytes = (int)a.dout_stride * 2;
  const float *lse = a.lse + (int64_t)head * a.group * a.n_q + s.q0, *delta = a.delta + (int64_t)head * a.group * a.n_q + s.q0;
  const float to_log2 = a.scale * kLog2E;

  f32x16 dk[D / 32], dv[D / 32];
  float row_lse = -INFINITY, row_delta = 0.f;
  int row_last = -1;
  // the rows from `row0` on; their first query and head are kept as they go
  int next_query, next_head, query = 0, head_of_group = 0;
  const int query_step = kDkvRows / a.group, head_step = kDkvRows - query_step * a.group;
  auto fetch = [&](int row0, char (&to)[2][kDkvRows * D * 2]) __attribute__((always_inline)) {
    if (threadIdx.x < kDkvRows) {            // in front of the copies: waiting for these loads must not wait for those
      const int at = next_head + threadIdx.x, of = small_quotient(at, a.group_inverse), t = next_query + of;
      row_lse = -INFINITY;                   // probability 0: rows past the end, and rows that see no key
      row_delta = 0.f;
      row_last = -1;
      if (row0 + (int)threadIdx.x < n_rows) {
        const int64_t w = (at - of * a.group) * a.n_q + t;
        row_lse = lse[w];
        row_delta = delta[w];
        row_last = last_key(a, s, t);
      }
    }
    TileCopy<D, kDkvRows>::fetch_grouped(q + (int64_t)next_query * q_bytes, q_bytes, a.group, a.group_inverse, next_head, n_rows - row0, to[0], lane, wave);
    TileCopy<D, kDkvRows>::fetch_grouped(d + (int64_t)next_query * d_bytes, d_bytes, a.group, a.group_inverse, next_head, n_rows - row0, to[1], lane, wave);
  };
  // what goes with the tile that was fetched last
  auto store_words = [&](RowWords& w) __attribute__((always_inline)) {
    if (threadIdx.x < kDkvRows) {
      w.shift[threadIdx.x] = row_lse == -INFINITY ? INFINITY : row_lse * kLog2E;
      w.delta[threadIdx.x] = row_delta;
      w.last[threadIdx.x] = row_last;
    }
  };
  auto advance = [&]() __attribute__((always_inline)) {
    query = next_query;
    head_of_group = next_head;
    next_query += query_step;
    next_head += head_step;
    if (next_head >= a.group) {
      next_head -= a.group;
      ++next_query;
    }
  };
  auto step = [&](char* qt, char* dt, RowWords& w, auto careful) __attribute__((always_inline)) {
    constexpr bool kCareful = decltype(careful)::value;
    if (query + small_quotient(head_of_group + kDkvRows - 1, a.group_inverse) < wave_first) return;
    const bool edge = kCareful && query < wave_all;
    if (edge) {
      add_not_finite<D, kDkvRows, true>(qt, dk, half, [&](int i) { return key <= w.last[i]; });
      add_not_finite<D, kDkvRows, false>(dt, dv, half, [&](int i) { return key <= w.last[i]; });
    }
    f32x16 p[2] = {}, dp[2] = {};
    tile_times_columns<D>(qt, k.f, p, lane);
    // Probabilities of what is masked are 0, and so are its dS if all is finite (if not, NaN leads to the careful pass, which takes them out one by one).  The
    // mask has its branch here: the exponentials run under the products of dP
    if (!kCareful && query < wave_all) {
#pragma unroll
      for (int i4 = 0; i4 < 8; ++i4) {
        const i32x4 last = *(const i32x4*)(w.last + 8 * i4 + 4 * half);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (key > last[e]) p[i4 >> 2][4 * (i4 & 3) + e] = -INFINITY;
      }
    }
    tile_times_columns<D>(dt, v.f, dp, lane, [&](int part) __attribute__((always_inline)) {
      constexpr int kFours = 8 / (D / 32);
#pragma unroll
      for (int i4 = kFours * part; i4 < kFours * part + kFours; ++i4) {
        const f32x4 shift = *(const f32x4*)(w.shift + 8 * i4 + 4 * half);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = 4 * (i4 & 3) + e;
          p[i4 >> 2][i] = exp2_fast(fmaf(p[i4 >> 2][i], to_log2, -shift[e]));
        }
        if constexpr (kCareful) {
          const i32x4 last = *(const i32x4*)(w.last + 8 * i4 + 4 * half);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (key > last[e]) p[i4 >> 2][4 * (i4 & 3) + e] = 0.f;
        }
      }
    });
    bf16x8 pf[2], df[2], dof[2][D / 32], qf[2][D / 32];
    auto ready = [&](int g) __attribute__((always_inline)) {
#pragma unroll
      for (int i4 = 0; i4 < 2; ++i4) {
        const int row = 16 * g + 8 * i4 + 4 * half;
        const f32x4 del = *(const f32x4*)(w.delta + row);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = 8 * (g & 1) + 4 * i4 + e;
          dp[g >> 1][i] = p[g >> 1][i] * (dp[g >> 1][i] - del[e]);
        }
        if constexpr (kCareful) {
          const i32x4 last = *(const i32x4*)(w.last + row);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (key > last[e]) dp[g >> 1][8 * (g & 1) + 4 * i4 + e] = 0.f;
        }
      }
      pf[g & 1] = fragment_of_result(p[g >> 1], g & 1);
      df[g & 1] = fragment_of_result(dp[g >> 1], g & 1);
#pragma unroll
      for (int db = 0; db < D / 32; ++db) {
        if constexpr (kCareful) continue;
        dof[g & 1][db] = transposed_fragment<D>(dt, lane, db, g);
        qf[g & 1][db] = transposed_fragment<D>(qt, lane, db, g);
      }
    };
    ready(0);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      if (g < 3) ready(g + 1);
#pragma unroll
      for (int db = 0; db < D / 32; ++db) {
        if constexpr (kCareful) {
          dv[db] = mfma32(finite_fragment<D>(dt, lane, db, g, edge), pf[g & 1], dv[db]);
          dk[db] = mfma32(finite_fragment<D>(qt, lane, db, g, edge), df[g & 1], dk[db]);
          __builtin_amdgcn_sched_barrier(0);
        } else {
          dv[db] = mfma32(dof[g & 1][db], pf[g & 1], dv[db]);
          dk[db] = mfma32(qf[g & 1][db], df[g & 1], dk[db]);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  auto pass = [&](auto careful) __attribute__((always_inline)) {
#pragma unroll
    for (int db = 0; db < D / 32; ++db) dk[db] = dv[db] = f32x16{};
    next_query = first_row / a.group;
    next_head = first_row - next_query * a.group;
    fetch(first_row, tiles[0]);
    store_words(words[0]);
    end_of_step();
    for (int row0 = first_row; row0 < end_row; row0 += 2 * kDkvRows) {
      advance();
      if (row0 + kDkvRows < end_row) fetch(row0 + kDkvRows, tiles[1]);
      step(tiles[0][0], tiles[0][1], words[0], careful);
      store_words(words[1]);
      end_of_step();
      if (row0 + kDkvRows >= end_row) break;
      advance();
      if (row0 + 2 * kDkvRows < end_row) fetch(row0 + 2 * kDkvRows, tiles[0]);
      step(tiles[1][0], tiles[1][1], words[1], careful);
      store_words(words[0]);
      end_of_step();
    }
  };
  pass(std::false_type{});
  if (__syncthreads_or(not_finite<D>(dk) || not_finite<D>(dv))) pass(std::true_type{});
  if (key >= s.n_k) return;
  if (a.row_parts > 1) {
    float* row = a.parts + ((part * a.n_k + s.k0 + key) * a.hkv + head) * (2 * D) + 4 * half;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        *(f32x4*)(row + 32 * db + 8 * i) = f32x4{dk[db][4 * i], dk[db][4 * i + 1], dk[db][4 * i + 2], dk[db][4 * i + 3]};
        *(f32x4*)(row + D + 32 * db + 8 * i) = f32x4{dv[db][4 * i], dv[db][4 * i + 1], dv[db][4 * i + 2], dv[db][4 * i + 3]};
      }
    return;
  }
  store_columns<D>(a.dk + (s.k0 + key) * a.dk_stride + head * D, dk, a.scale, lane);
  store_columns<D>(a.dv + (s.k0 + key) * a.dv_stride + head * D, dv, 1.f, lane);
}

// dk, dv of a tile's keys from the sums of its row_parts workgroups; kJoinKeys keys per workgroup, all loads of a sum under way at once
constexpr int kJoinKeys = 8, kMaxRowParts = 8;
template <int D>
__global__ void __launch_bounds__(256) attn_dkv_join_kernel(AttnArgs a) {
  int head, slot;
  head_and_slot(blockIdx.x, a.hkv, a.slots, head, slot);
  if (slot >= a.slots) return;
  int64_t first_slot;
  const Sequence s = sequence(a, sequence_of_slot(a.cu_k, a.n_seqs, a.n_k, 1, kDkvKeys, slot, &first_slot));
  const int tile_key = (int)(slot - first_slot) * kDkvKeys;
  if (slot < first_slot || tile_key >= s.n_k) return;
  constexpr int kFours = 2 * D / 4;              // of a key
  const int key0 = tile_key + blockIdx.y * kJoinKeys, n = (s.n_k - key0 < kJoinKeys ? s.n_k - key0 : kJoinKeys) * kFours;
  const int64_t part_stride = a.n_k * a.hkv * (2 * D);
  for (int i = threadIdx.x; i < n; i += 256) {
    const int64_t key = s.k0 + key0 + i / kFours;
    const int at = i % kFours * 4;
    const float* from = a.parts + (key * a.hkv + head) * (2 * D) + at;
    f32x4 x[kMaxRowParts], sum = {};
#pragma unroll
    for (int p = 0; p < kMaxRowParts; ++p) x[p] = p < a.row_parts ? *(const f32x4*)(from + p * part_stride) : f32x4{};
#pragma unroll
    for (int p = 0; p < kMaxRowParts; ++p) sum += x[p];
    if (at < D) *(bf16x4*)(a.dk + key * a.dk_stride + head * D + at) = __builtin_convertvector(sum * a.scale, bf16x4);
    else *(bf16x4*)(a.dv + key * a.dv_stride + head * D + at - D) = __builtin_convertvector(sum, bf16x4);
  }
}

bool misaligned(const void* p) { return ((uintptr_t)p & 15) != 0; }

// Checks of what forward and backward share; fills `a`.
nat_status attn_args(const nat_attn_params* p, const void* d_q, const void* d_k, const void* d_v, const int32_t* d_cu_q, const int32_t* d_cu_k,
                     AttnArgs* a) {
  if (!p) return NAT_INVALID_ARG;
  if (p->dtype != NAT_DTYPE_BF16) return NAT_UNSUPPORTED_DTYPE;
  if (p->n_seqs < 0 || p->n_q < 0 || p->n_k < 0 || p->n_q > INT32_MAX || p->n_k > INT32_MAX) return NAT_INVALID_ARG;
  if (!(p->scale > 0.f) || !(p->scale < INFINITY)) return NAT_INVALID_ARG;
  if (p->causal != 0 && p->causal != 1) return NAT_INVALID_ARG;
  if ((p->head_dim != 64 && p->head_dim != 128) || p->n_kv_heads <= 0 || p->n_q_heads <= 0 || p->n_q_heads % p->n_kv_heads != 0 ||
      p->n_q_heads > 4096)
    return NAT_BAD_SHAPE;
  const int64_t q_row = (int64_t)p->n_q_heads * p->head_dim, k_row = (int64_t)p->n_kv_heads * p->head_dim;
  const int group = p->n_q_heads / p->n_kv_heads;
  // rows of a group's matrix are counted in 32 bits, and a launch has to have room for the tile slots (grid_of adds up to 7 workgroups)
  constexpr int64_t kMostSlots = kMaxWorkItems / 256 - 7;
  if (p->n_q * group > INT32_MAX / 2 || (p->n_q * group / kRowTile + p->n_seqs) * p->n_kv_heads > kMostSlots ||
      (p->n_k / kDkvKeys + p->n_seqs) * p->n_kv_heads > kMostSlots)
    return NAT_BAD_SHAPE;
  auto stride_ok = [](int64_t s, int64_t row) { return s == 0 || (s >= row && s % 8 == 0 && s < kMaxStride); };
  if (!stride_ok(p->q_stride, q_row) || !stride_ok(p->out_stride, q_row) || !stride_ok(p->dout_stride, q_row) || !stride_ok(p->dq_stride, q_row) ||
      !stride_ok(p->k_stride, k_row) || !stride_ok(p->v_stride, k_row) || !stride_ok(p->dk_stride, k_row) || !stride_ok(p->dv_stride, k_row))
    return NAT_BAD_SHAPE;
  *a = AttnArgs{};
  a->n_seqs = p->n_seqs;
  if (p->n_seqs == 0) return NAT_OK;
  if (!d_cu_q || !d_cu_k || (p->n_q > 0 && !d_q) || (p->n_k > 0 && (!d_k || !d_v))) return NAT_INVALID_ARG;
  if (misaligned(d_q) || misaligned(d_k) || misaligned(d_v)) return NAT_INVALID_ARG;
  auto or_row = [](int64_t s, int64_t row) { return s ? s : row; };
  a->q = (const uint16_t*)d_q;
  a->k = (const uint16_t*)d_k;
  a->v = (const uint16_t*)d_v;
  a->cu_q = d_cu_q;
  a->cu_k = d_cu_k;
  a->hq = p->n_q_heads;
  a->hkv = p->n_kv_heads;
  a->group = group;
  a->group_inverse = (uint32_t)((1ull << 31) / group + 1);
  a->causal = p->causal;
  a->n_q = p->n_q;
  a->n_k = p->n_k;
  a->scale = p->scale;
  a->q_stride = or_row(p->q_stride, q_row);
  a->out_stride = or_row(p->out_stride, q_row);
  a->dout_stride = or_row(p->dout_stride, q_row);
  a->dq_stride = or_row(p->dq_stride, q_row);
  a->k_stride = or_row(p->k_stride, k_row);
  a->v_stride = or_row(p->v_stride, k_row);
  a->dk_stride = or_row(p->dk_stride, k_row);
  a->dv_stride = or_row(p->dv_stride, k_row);
  return NAT_OK;
}

// Workgroups per tile of keys: as many as make up for tiles of unequal length (causal) or fill the chip, with four steps each at least.  Backward in us, D = 128, 32 heads
// on 8, causal: 2048 tokens 332 with one, 190 with 3, 213 with 7; 4096 tokens 720, 557 with 3; all keys seen: 912, 899, 939 with 3.  D = 64, two workgroups at a time on a compute
// unit: 8192 tokens of 4 heads 271 with one, 203 with 3.
int row_parts_of(int64_t n_q, int64_t n_k, int64_t n_seqs, int64_t hkv, int64_t group, int head_dim, bool causal) {
  if (n_seqs <= 0 || n_q <= 0 || n_k <= 0) return 1;
  const int64_t blocks = (n_k / kDkvKeys + n_seqs) * hkv, steps = n_q * group / n_seqs / kDkvRows / (causal ? 2 : 1);
  int64_t p = (!causal ? 512 : head_dim == 128 ? 768 : 1024) / blocks;
  if (p > steps / 4) p = steps / 4;
  return (int)(p < 1 ? 1 : p > kMaxRowParts ? kMaxRowParts : p);
}
// Workgroups per tile of rows: where the tiles do not fill the chip, or, of unequal length (as many queries as keys, causal), fill it less than twice; 256 keys each at
// least, and more where there are many rows whose sums are written and read once more.  In us, D = 128, one workgroup per tile and so many: 16 rows behind 8000 (32 heads on 8) 147, 25 (15 parts); 8 x 5 behind 4000 77, 33; 256 behind 8000 152, 57; 8192 of 4 on 1
// 149, 102 (3 parts).  Twice as many for 6 x 350 behind 2000 (28 on 4): 121 instead of 84; two of 256 keys on
// average for 1024 (32 on 8): 43 instead of 29.
int key_parts_of(int64_t n_q, int64_t n_k, int64_t n_seqs, int64_t hkv, int64_t group, int head_dim, bool causal) {
  if (n_seqs <= 0 || n_q <= 0 || n_k <= 0) return 1;
  const int64_t part_keys = 256 + n_q * hkv * group / 64;
  const int64_t blocks = (n_q * group / kRowTile + n_seqs) * hkv, keys = (causal ? n_k - n_q / 2 : n_k) / n_seqs;
  int64_t p = (head_dim == 128 ? 512 : 768) * (causal && 2 * n_q > n_k ? 2 : 1) / blocks;
  if (p > keys / part_keys) p = keys / part_keys;
  return (int)(p < 1 ? 1 : p > kMaxKeyParts ? kMaxKeyParts : p);
}
size_t key_part_bytes(int64_t n_q, int64_t hq, int64_t head_dim) { return (size_t)n_q * hq * (head_dim + 2) * 4; }
// what the sizes of workspaces are computed from
bool counts_ok(const nat_attn_params* p) {
  return p && p->n_kv_heads > 0 && p->n_q_heads > 0 && p->n_q_heads <= 4096 && p->n_q_heads % p->n_kv_heads == 0 && p->n_q >= 0 && p->n_k >= 0 &&
         p->n_q <= INT32_MAX && p->n_k <= INT32_MAX && (p->head_dim == 64 || p->head_dim == 128);
}
size_t row_part_bytes(int64_t n_k, int64_t hkv, int64_t head_dim) { return (size_t)n_k * hkv * head_dim * 8; }

}  // namespace
}  // namespace nat

using namespace nat;

extern "C" size_t nat_attn_fwd_workspace_bytes(const nat_attn_params* p) {
  if (!counts_ok(p)) return 0;
  const int parts = key_parts_of(p->n_q, p->n_k, p->n_seqs, p->n_kv_heads, p->n_q_heads / p->n_kv_heads, p->head_dim, p->causal != 0);
  return parts > 1 ? (parts * key_part_bytes(p->n_q, p->n_q_heads, p->head_dim) + 255) / 256 * 256 : 0;
}

extern "C" nat_status nat_attn_fwd_split(const nat_attn_params* params, const void* d_q, const void* d_k, const void* d_v, const int32_t* d_cu_q,
                                         const int32_t* d_cu_k, void* d_out, float* d_lse, void* d_ws, size_t ws_bytes, void* stream) {
  AttnArgs a;
  const nat_status st = attn_args(params, d_q, d_k, d_v, d_cu_q, d_cu_k, &a);
  if (st != NAT_OK || a.n_seqs == 0 || a.n_q == 0) return st;
  if (!d_out || !d_lse || misaligned(d_out) || ((uintptr_t)d_ws & 255)) return NAT_INVALID_ARG;
  a.out = (uint16_t*)d_out;
  a.lse = d_lse;
  hipStream_t s = (hipStream_t)stream;
  ProfScope prof(PC_ATTN_FWD, s);
  a.slots = (int)(a.n_q * a.group / kRowTile + a.n_seqs);
  a.key_parts = key_parts_of(a.n_q, a.n_k, a.n_seqs, a.hkv, a.group, params->head_dim, a.causal != 0);
  const size_t part_bytes = key_part_bytes(a.n_q, a.hq, params->head_dim);
  while (a.key_parts > 1 && (!d_ws || ws_bytes < a.key_parts * part_bytes)) --a.key_parts;
  a.parts = (float*)d_ws;
  a.part_ml = a.parts + (size_t)a.key_parts * a.n_q * a.hq * params->head_dim;
  const unsigned blocks = grid_of(a.hkv, (int64_t)a.slots * a.key_parts);
  if (a.key_parts == 1) {
    if (params->head_dim == 128) attn_fwd_kernel<128, false><<<blocks, 256, 0, s>>>(a);
    else attn_fwd_kernel<64, false><<<blocks, 256, 0, s>>>(a);
    NAT_LAUNCH_CHECK();
  } else {
    if (params->head_dim == 128) attn_fwd_kernel<128, true><<<blocks, 256, 0, s>>>(a);
    else attn_fwd_kernel<64, true><<<blocks, 256, 0, s>>>(a);
    NAT_LAUNCH_CHECK();
    const dim3 joins(grid_of(a.hkv, a.slots), kRowTile / kJoinRows);
    if (params->head_dim == 128) attn_fwd_join_kernel<128><<<joins, 256, 0, s>>>(a);
    else attn_fwd_join_kernel<64><<<joins, 256, 0, s>>>(a);
    NAT_LAUNCH_CHECK();
  }
  return NAT_OK;
}

extern "C" nat_status nat_attn_fwd(const nat_attn_params* params, const void* d_q, const void* d_k, const void* d_v, const int32_t* d_cu_q,
                                   const int32_t* d_cu_k, void* d_out, float* d_lse, void* stream) {
  return nat_attn_fwd_split(params, d_q, d_k, d_v, d_cu_q, d_cu_k, d_out, d_lse, nullptr, 0, stream);
}

extern "C" size_t nat_attn_bwd_workspace_bytes(int64_t n_q, int32_t n_q_heads) {
  if (n_q <= 0 || n_q_heads <= 0 || n_q > INT32_MAX || n_q_heads > 4096) return 0;
  return ((size_t)n_q * (size_t)n_q_heads * 4 + 255) / 256 * 256;
}

extern "C" size_t nat_attn_bwd_workspace_full_bytes(const nat_attn_params* p) {
  if (!counts_ok(p)) return 0;
  const size_t least = nat_attn_bwd_workspace_bytes(p->n_q, p->n_q_heads);
  const int parts = row_parts_of(p->n_q, p->n_k, p->n_seqs, p->n_kv_heads, p->n_q_heads / p->n_kv_heads, p->head_dim, p->causal != 0);
  return parts > 1 ? least + parts * row_part_bytes(p->n_k, p->n_kv_heads, p->head_dim) : least;
}

extern "C" nat_status nat_attn_bwd(const nat_attn_params* params, const void* d_q, const void* d_k, const void* d_v, const void* d_out,
                                   const float* d_lse, const void* d_dout, const int32_t* d_cu_q, const int32_t* d_cu_k, void* d_dq, void* d_dk,
                                   void* d_dv, void* d_ws, size_t ws_bytes, void* stream) {
  AttnArgs a;
  const nat_status st = attn_args(params, d_q, d_k, d_v, d_cu_q, d_cu_k, &a);
  if (st != NAT_OK || a.n_seqs == 0) return st;
  if (a.n_q > 0 && (!d_out || !d_lse || !d_dout || !d_dq)) return NAT_INVALID_ARG;
  if (a.n_k > 0 && (!d_dk || !d_dv)) return NAT_INVALID_ARG;
  if (misaligned(d_out) || misaligned(d_dout) || misaligned(d_dq) || misaligned(d_dk) || misaligned(d_dv)) return NAT_INVALID_ARG;
  if (a.n_q > 0 && (!d_ws || ws_bytes < nat_attn_bwd_workspace_bytes(a.n_q, a.hq))) return NAT_WORKSPACE_TOO_SMALL;
  if ((uintptr_t)d_ws & 255) return NAT_INVALID_ARG;
  a.out = (uint16_t*)const_cast<void*>(d_out);
  a.lse = const_cast<float*>(d_lse);
  a.dout = (const uint16_t*)d_dout;
  a.delta = (float*)d_ws;
  a.dq = (uint16_t*)d_dq;
  a.dk = (uint16_t*)d_dk;
  a.dv = (uint16_t*)d_dv;
  hipStream_t s = (hipStream_t)stream;
  if (a.n_q > 0) {
    ProfScope prof(PC_ATTN_BWD, s);
    a.slots = (int)(a.n_q * a.group / kRowTile + a.n_seqs);
    if (params->head_dim == 128) attn_dq_kernel<128><<<grid_of(a.hkv, a.slots), 256, 0, s>>>(a);
    else attn_dq_kernel<64><<<grid_of(a.hkv, a.slots), 256, 0, s>>>(a);
    NAT_LAUNCH_CHECK();
  }
  if (a.n_k > 0) {
    ProfScope prof(PC_ATTN_BWD, s);
    a.slots = (int)(a.n_k / kDkvKeys + a.n_seqs);
    a.row_parts = row_parts_of(a.n_q, a.n_k, a.n_seqs, a.hkv, a.group, params->head_dim, a.causal != 0);
    const size_t least = nat_attn_bwd_workspace_bytes(a.n_q, a.hq), slab = row_part_bytes(a.n_k, a.hkv, params->head_dim);
    while (a.row_parts > 1 && ws_bytes < least + a.row_parts * slab) --a.row_parts;
    a.parts = (float*)((char*)d_ws + least);
    const unsigned blocks = grid_of(a.hkv, (int64_t)a.slots * a.row_parts);
    if (params->head_dim == 128) attn_dkv_kernel<128><<<blocks, 256, 0, s>>>(a);
    else attn_dkv_kernel<64><<<blocks, 256, 0, s>>>(a);
    NAT_LAUNCH_CHECK();
    if (a.row_parts > 1) {
      if (params->head_dim == 128) attn_dkv_join_kernel<128><<<dim3(grid_of(a.hkv, a.slots), kDkvKeys / kJoinKeys), 256, 0, s>>>(a);
      else attn_dkv_join_kernel<64><<<dim3(grid_of(a.hkv, a.slots), kDkvKeys / kJoinKeys), 256, 0, s>>>(a);
      NAT_LAUNCH_CHECK();
    }
  }
  return NAT_OK;
}
