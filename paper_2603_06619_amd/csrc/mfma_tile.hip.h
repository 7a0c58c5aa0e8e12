// Tiles of bf16 rows in LDS and the fragments that the matrix core takes from them: what the attention kernels share.
//
// Products are 32 x 32 x 16, C[m][n] += sum_k A[m][k] B[k][n] with, in lane l (c = l % 32, h = l / 32),
//   A: row m = c, k = 8 h + j, j = 0..7;   B: column n = c, k = 8 h + j;   C: column n = c, rows m = 8 (i / 4) + 4 h + i % 4, i = 0..15.
// A product's result in bf16 is the B operand of the next one as it lies in the registers: of 16 rows from 16 s on, lane l holds
// rows 16 s + 4 h .. + 3 and 16 s + 8 + 4 h .. + 3.  Those eight are taken as its k = 8 h .. + 7, and the A operand is read with the
// same order of k (transposed_fragment).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace nat {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// row of the result that element i of a lane of half h holds
__host__ __device__ constexpr int result_row(int i, int h) { return 8 * (i >> 2) + 4 * h + (i & 3); }

// Eight results, elements 8 s .. + 7, as the fragment of 16 k's of the next product's B.
__device__ __forceinline__ bf16x8 fragment_of_result(const f32x16& c, int s) {
  typedef float f32x8 __attribute__((ext_vector_type(8)));
  const f32x8 x = {c[8 * s], c[8 * s + 1], c[8 * s + 2], c[8 * s + 3], c[8 * s + 4], c[8 * s + 5], c[8 * s + 6], c[8 * s + 7]};
  return __builtin_convertvector(x, bf16x8);
}

// A tile of rows of D elements.  The 16-byte chunks of a row lie permuted, chunk c of row r at c ^ swizzle(r), so that neither kind of
// read has bank conflicts.  LDS has 64 banks of 4 bytes.  A fragment along the row is read 16 bytes per lane, 16 lanes at a time (0-3, 12-15,
// 20-27, then 4-11, 16-19, 28-31) at one chunk of as many rows: of a 256-byte row they want 16 permutations that differ, of
// 128-byte rows, two to a line of banks, 8 among the even and 8 among the odd ones.  The transposing read takes 64 bytes of four consecutive rows at a
// time, which want to lie in different quarters of the banks, or (16 x 16 products) 32 bytes of eight, in different eighths.
template <int D>
struct RowTile {
  static_assert(D == 64 || D == 128, "rows are one or two half lines of banks");
  static constexpr int kChunks = D / 8;
  __host__ __device__ static constexpr int swizzle(int row) {
    return D == 128 ? ((row & 3) << 2) | (((row >> 2) & 1) << 1) | ((row >> 3) & 1)
                    : (((row >> 1) & 1) << 2) | (((row >> 2) & 1) << 1) | ((row >> 3) & 1);
  }
  // byte offset of chunk c of row r
  __host__ __device__ static constexpr int chunk_at(int row, int chunk) { return row * (2 * D) + ((chunk ^ swizzle(row)) << 4); }
  // Fragment of rows 32 rb .. + 31 (m or n) and elements 16 s .. + 15 (k)
  __host__ __device__ static constexpr int fragment_at(int lane, int rb, int s) { return chunk_at(32 * rb + (lane & 31), 2 * s + (lane >> 5)); }
  // Fragment of elements 32 db .. + 31 (m) and rows 16 s .. + 15 (k, in the order of a result): two transposing reads, part = 0, 1
  __host__ __device__ static constexpr int transposed_at(int lane, int db, int s, int part) {
    const int i = lane & 15, row = 16 * s + 8 * part + 4 * (lane >> 5) + (i >> 2);
    return chunk_at(row, 4 * db + 2 * ((lane >> 4) & 1) + ((i & 3) >> 1)) + 8 * (i & 1);
  }
};

template <int D>
__device__ __forceinline__ bf16x8 row_fragment(const char* tile, int lane, int rb, int s) {
  return *(const bf16x8*)(tile + RowTile<D>::fragment_at(lane, rb, s));
}

// The transposing read works on groups of 16 lanes: lane i supplies the address of 4 consecutive elements and receives element i % 4 of those
// of lanes i / 4, i / 4 + 4, i / 4 + 8 and i / 4 + 12.
__device__ __forceinline__ s16x4 lds_transposed(const char* p) {
  typedef __attribute__((address_space(3))) s16x4* lds_ptr;
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(p));
}

template <int D>
__device__ __forceinline__ bf16x8 transposed_fragment(const char* tile, int lane, int db, int s) {
  typedef short s16x8 __attribute__((ext_vector_type(8)));
  const s16x4 a = lds_transposed(tile + RowTile<D>::transposed_at(lane, db, s, 0)), b = lds_transposed(tile + RowTile<D>::transposed_at(lane, db, s, 1));
  const s16x8 both = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
  return __builtin_bit_cast(bf16x8, both);
}

// Sum and maximum of a value over the two halves of the wavefront (lanes l and l ^ 32): the swap gives every lane both halves' values.
__device__ __forceinline__ float sum_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
  return __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
}
__device__ __forceinline__ float max_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
  return fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }      // one instruction; results below 2^-126 are 0

}  // namespace nat
