// What the attention kernels of one token per request share: reductions over the lanes of a
// 16x16 MFMA result, and how pages lie in LDS.
#pragma once
#include "common.hpp"

namespace ca {

template <typename T>
__device__ __forceinline__ T uniform(T v) {
  static_assert(sizeof(T) == 4, "");
  return __builtin_bit_cast(T, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, v)));
}

__device__ __forceinline__ float max2(float a, float b) {
  return __builtin_elementwise_maximum(a, b);   // a NaN stays
}

// Over the 4 lane groups that hold the same column.
__device__ __forceinline__ float groups_max(float x) {
  uint32_t u = __float_as_uint(x);
  auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  u = __float_as_uint(max2(__uint_as_float(r[0]), __uint_as_float(r[1])));
  r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return max2(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float groups_sum(float x) {
  uint32_t u = __float_as_uint(x);
  auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  u = __float_as_uint(__uint_as_float(r[0]) + __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// 2^x, and the maxima in log2 units: exp2 of -inf is 0.
__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i16x4 lds_i16x4;

// Key that row r of 16-key tile kt of a page stands for: lane group g, which the
// 16x16 result gives rows 4g .. 4g+3, then holds keys 32p + 8g .. 32p + 8g + 7
// of the 32-key step p (tiles 2p, 2p + 1).
__host__ __device__ constexpr int key_of(int kt, int r) {
  return 32 * (kt >> 1) + 8 * (r >> 2) + 4 * (kt & 1) + (r & 3);
}
// A page, or half of one, in LDS: rows of D are keys of K or token-major V, rows of 64
// keys the dimensions of a transposed V page.  16-byte chunk where chunk c of row r lies, so
// that operand reads meet no bank twice:
//   K: 16 lanes read 16 bytes each, of rows that differ in bits 0, 1, 3 and 4;
//   token-major V: 32 lanes of a transpose read cover rows {0..3, 8..11} (+
//     multiples) x 32 bytes, so bits 0, 1 and 3 pick the 32-byte pair;
//   transposed V: 16 lanes read 16 bytes each, of 16 rows in a row.
// Where rows are 128 bytes, two share the 256 bytes of all banks, by bit 0.
enum Half { kHalfK, kHalfV, kHalfVT };
template <int D, Half H>
__device__ __forceinline__ int swizzle(int r, int c) {
  if (H == kHalfVT) return c ^ ((r >> 1) & 7);
  if (H == kHalfK)
    return D == 128 ? (c ^ ((r & 3) | (((r >> 3) & 3) << 2)))
                    : (c ^ (((r >> 1) & 1) | (((r >> 3) & 3) << 1)));
  return D == 128 ? (c ^ (((r & 3) | (((r >> 3) & 1) << 2)) << 1))
                  : (c ^ ((((r >> 1) & 1) | (((r >> 3) & 1) << 1)) << 1));
}

}  // namespace ca
