// The layout of 4-bit weights (internal).
//
// Codes 0 .. 15 lie in tiles of 16 rows x 64 columns, 512 bytes: u32 [row tiles][column tiles][32 lanes][4].
// Lane 4 g + t (g = 0 .. 7, t = 0 .. 3) holds rows g and g + 8 of the tile; its word j columns
// w4_column(t, j) + i, i = 0 .. 3: row g's codes in bits 0, 16, 8, 24 and up, row g + 8's four bits above each.
// So a lane's four words are what four m16n8k16 steps want of it in the matrix operand (the columns of a step,
// in any order, only have to be the same as the rows' that they meet), a pair of neighbouring columns
// becomes two 16-bit values with one mask, and words 0, 1 and 2, 3 each cover 32 neighbouring columns,
// the smallest group.
#pragma once
#include "rows.cuh"

namespace xnor {

__host__ __device__ __forceinline__ int w4_column(int t, int j) { return 32 * (j >> 1) + 8 * t + 4 * (j & 1); }

// The part of a word that the four codes of one row make (for row g + 8: shifted up by four).
__device__ __forceinline__ uint32_t w4_spread(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3) {
  return c0 | c1 << 16 | c2 << 8 | c3 << 24;
}

// Two values of a word as 16-bit numbers code - zero, exact: pair 0, 1: columns 0 and 1 of rows g, g + 8; pair
// 2, 3: columns 2 and 3.  A code put into the mantissa of 2^k is 2^k + code; `zero` holds (2^k + zero) twice.
__device__ __forceinline__ uint32_t w4_pair(uint32_t w, int pair, __nv_bfloat16, uint32_t zero) {
  const uint32_t v = ((w >> (4 * pair)) & 0x000F000Fu) | 0x43004300u;                    // 128 + code
  const __nv_bfloat162 r = __hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&v), *reinterpret_cast<const __nv_bfloat162 *>(&zero));
  return *reinterpret_cast<const uint32_t *>(&r);
}
__device__ __forceinline__ uint32_t w4_pair(uint32_t w, int pair, __half, uint32_t zero) {
  const uint32_t v = ((w >> (4 * pair)) & 0x000F000Fu) | 0x64006400u;                    // 1024 + code
  const __half2 r = __hsub2(*reinterpret_cast<const __half2 *>(&v), *reinterpret_cast<const __half2 *>(&zero));
  return *reinterpret_cast<const uint32_t *>(&r);
}
__device__ __forceinline__ uint32_t w4_zero(uint32_t z, __nv_bfloat16) { return (0x4300u | z) * 0x00010001u; }
__device__ __forceinline__ uint32_t w4_zero(uint32_t z, __half) { return (0x6400u | z) * 0x00010001u; }

// Eight values of a row in 8 bits as 16-bit numbers, exact.  The code of an int8 with its sign bit turned is
// 128 + value; in the mantissa of 1024 it is 1152 + value.
__device__ __forceinline__ uint32_t i8_pair(uint32_t four, int pair) {
  const uint32_t v = __byte_perm(four ^ 0x80808080u, 0x64646464u, pair == 0 ? 0x4140 : 0x4342);
  const __half2 r = __hsub2(*reinterpret_cast<const __half2 *>(&v), __half2half2(__ushort_as_half(0x6480)));   // 1152
  return *reinterpret_cast<const uint32_t *>(&r);
}
__device__ __forceinline__ uint32_t e4m3_pair(uint32_t two) {
  const __half2_raw r = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)two, __NV_E4M3);
  return (uint32_t)r.x | (uint32_t)r.y << 16;
}

}  // namespace xnor
