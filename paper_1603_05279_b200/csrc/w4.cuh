// The layout of 4-bit weights (internal).
//
// Codes 0 .. 15 lie in tiles of 16 rows x 64 columns, 512 bytes, the tiles of 128 rows together:
// u32 [panels of 8 row tiles][column tiles][8][32 places][4].
// A word holds eight neighbouring columns of one row, column 2 i + h in bits 4 i + 16 h and up: a mask brings two
// neighbouring columns to where two 16-bit values have them.  Place 4 g + (t ^ (g >> 1 & 3)) of a tile (g = 0 .. 7,
// t = 0 .. 3) holds, of row g, columns 8 t .. and 32 + 8 t .., then the same of row g + 8.  So its four words are
// what four m16n8k16 steps want of a lane in the matrix operand (the columns of a step, in any order, only have
// to be the same as those of the rows that they meet), two steps each for 32 neighbouring columns, the smallest
// group.  And threads that read a whole row each, from shared memory, meet in no bank: that is what t is turned
// for.
#pragma once
#include "rows.cuh"

namespace xnor {

// Place and word of the tile that hold row r, columns c .. c + 7 (c a multiple of 8).
__host__ __device__ __forceinline__ int w4_place(int r, int c) { return 4 * (r & 7) + (((c & 31) >> 3) ^ ((r >> 1) & 3)); }
__host__ __device__ __forceinline__ int w4_word(int r, int c) { return 2 * ((r >> 3) & 1) + (c >> 5); }

// The tile of 16 rows `rt`, of column tile 0; the next column's is kW4Panel tiles on (a tile: 32 uint4).
__host__ __device__ __forceinline__ size_t w4_tile(int rt, int col_tiles) { return ((size_t)(rt / kW4Panel) * col_tiles) * kW4Panel + rt % kW4Panel; }

__host__ __device__ __forceinline__ int w4_bit(int column) { return 4 * (column >> 1) + 16 * (column & 1); }

// The eight values of a word, code - zero, as four pairs of 16-bit numbers, exact.  Conversions of small whole numbers by way of
// the mantissa are a known method: a code put into that of 2^k is 2^k + code.  `magic` is kW4Magic of the type, but as a variable that the compiler does not know (a kernel's
// argument): a mask and an OR are one instruction if only one of them is a constant in it.  (One row times
// 16384x8192: 24.0 -> 20.2 us.)
template <class T>
struct W4Type;
template <>
struct W4Type<__nv_bfloat16> {
  static constexpr uint32_t kMagic = 0x43004300u;                            // 128
  struct Zero { uint32_t a; };
  __device__ static __forceinline__ Zero zero(uint32_t z) { return {(0x4300u | z) * 0x00010001u}; }
  __device__ static __forceinline__ void expand(uint32_t w, const Zero &z, uint32_t magic, uint32_t (&v)[4]) {
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const uint32_t u = ((w >> (4 * p)) & 0x000F000Fu) | magic;
      const __nv_bfloat162 r = __hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&u), *reinterpret_cast<const __nv_bfloat162 *>(&z.a));
      v[p] = *reinterpret_cast<const uint32_t *>(&r);
    }
  }
};
template <>
struct W4Type<__half> {
  static constexpr uint32_t kMagic = 0x64006400u;                            // 1024
  struct Zero { uint32_t a, b; };                                            // 1024 + zero, -(64 + zero)
  __device__ static __forceinline__ Zero zero(uint32_t z) { return {(0x6400u | z) * 0x00010001u, (0xD400u | z << 4) * 0x00010001u}; }
  __device__ static __forceinline__ void expand(uint32_t w, const Zero &z, uint32_t magic, uint32_t (&v)[4]) {
    const uint32_t sixteenth = 0x2C002C00u;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t lo = ((w >> (8 * h)) & 0x000F000Fu) | magic, hi = ((w >> (8 * h)) & 0x00F000F0u) | magic;      // 1024 + 16 code
      const __half2 r0 = __hsub2(*reinterpret_cast<const __half2 *>(&lo), *reinterpret_cast<const __half2 *>(&z.a));
      const __half2 r1 = __hfma2(*reinterpret_cast<const __half2 *>(&hi), *reinterpret_cast<const __half2 *>(&sixteenth), *reinterpret_cast<const __half2 *>(&z.b));
      v[2 * h] = *reinterpret_cast<const uint32_t *>(&r0);
      v[2 * h + 1] = *reinterpret_cast<const uint32_t *>(&r1);
    }
  }
};

// w / s to the nearest whole number, ties to even, of the exact quotient (|w / s| below 2^20).  A first guess is off by one
// at most, where the quotient lies next to a border, and the rest w - q s is exact in 32 bits.
__device__ __forceinline__ float mend_quotient(float q, float w, float s) {
  const float r = fmaf(-q, s, w), twice = 2.0f * fabsf(r);
  return twice > s || (twice == s && ((int)q & 1)) ? q + (r > 0.0f ? 1.0f : -1.0f) : q;
}
__device__ __forceinline__ float round_quotient(float w, float s) { return mend_quotient(rintf(w / s), w, s); }

// The same of kN values.  With the reciprocal the guess is within 2e-6 of the quotient (at most 16), so only guesses that
// close to a border can be wrong; all are mended then.  (inv = 0: it would overflow.  Such a scale may be a few units of
// fp32's least number, so far from a seventh or a 15th that quotients leave the codes' range: -zero .. 15 - zero.)
template <int kN>
__device__ __forceinline__ void round_quotients(const float (&w)[kN], float s, float inv, float zero, float (&q)[kN]) {
  if (inv == 0.0f) {
#pragma unroll 1
    for (int i = 0; i < kN; ++i) q[i] = fminf(15.0f - zero, fmaxf(-zero, round_quotient(w[i], s)));
    return;
  }
  float far = 0.0f;
#pragma unroll
  for (int i = 0; i < kN; ++i) {
    const float t = w[i] * inv;
    q[i] = __fadd_rn(__fadd_rn(t, 12582912.0f), -12582912.0f);          // 1.5 2^23: rounds to a whole number
    far = fmaxf(far, fabsf(t - q[i]));
  }
  if (far > 0.49999f) {
#pragma unroll
    for (int i = 0; i < kN; ++i) q[i] = mend_quotient(q[i], w[i], s);
  }
}

// Four codes c0 .. c3 as c0 + 16 c1 + 256 c2 + 4096 c3, which 32-bit floats hold exactly; in the mantissa of 2^23 they
// lie as a word has them.  (With a conversion, a shift and an OR for each code 4096x4096 bf16 took
// 24.3 us, 18 to 20 so; what is left is 26 instructions a value, a third of them where quotients lie next to borders, as
// those of bf16 weights often do, at 2.6 a clock: blocks that load, wait, compute and store, half of the warps an SM can have.)
__device__ __forceinline__ float four_codes(float first, float c1, float c2, float c3) {
  return fmaf(c3, 4096.0f, fmaf(c2, 256.0f, fmaf(c1, 16.0f, first)));
}

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

// Eight values of x as four 16-bit pairs.  Bytes: int8 and e4m3 become 16-bit floats, exactly.
template <int kType>
struct RowsOf {
  using T = __half;                       // the products' type
  static constexpr int kBytes = 1;
};
template <> struct RowsOf<XNOR_BF16> { using T = __nv_bfloat16; static constexpr int kBytes = 2; };
template <> struct RowsOf<XNOR_F16> { using T = __half; static constexpr int kBytes = 2; };

// Two of four values in 8 bits.
template <int kType>
__device__ __forceinline__ uint32_t x_pair(uint32_t four, int pair) {
  if constexpr (kType == XNOR_I8) return i8_pair(four, pair);
  else return e4m3_pair((four >> (16 * pair)) & 0xFFFFu);
}
// As four pairs; `raw` is what lies in memory.
template <int kType>
__device__ __forceinline__ void x8_pairs(const uint32_t (&raw)[2 * RowsOf<kType>::kBytes], uint32_t (&v)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (RowsOf<kType>::kBytes == 2) v[i] = raw[i];
    else v[i] = x_pair<kType>(raw[i / 2], i & 1);
  }
}
// Columns k .. k + 7 of a row of K as they lie in memory; some may not exist (zeros) or lie anywhere.
template <int kType>
__device__ __forceinline__ void load_x8_raw(const uint8_t *row, int k, int K, bool pieces, uint32_t (&raw)[2 * RowsOf<kType>::kBytes]) {
  constexpr int kB = RowsOf<kType>::kBytes;
  const uint8_t *p = row + (size_t)k * kB;
  if (pieces && k + 8 <= K) {
    if constexpr (kB == 2) {
      const uint4 q = load_global(reinterpret_cast<const uint4 *>(p));
      raw[0] = q.x; raw[1] = q.y; raw[2] = q.z; raw[3] = q.w;
    } else {
      const uint2 q = load_global(reinterpret_cast<const uint2 *>(p));
      raw[0] = q.x; raw[1] = q.y;
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 2 * kB; ++i) raw[i] = 0u;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (k + i >= K) continue;
    if constexpr (kB == 2) raw[i / 2] |= (uint32_t)load_global(reinterpret_cast<const uint16_t *>(p) + i) << (16 * (i & 1));
    else raw[i / 4] |= (uint32_t)load_global(p + i) << (8 * (i & 3));
  }
}

}  // namespace xnor
