// Rows of 32-, 16- and 8-bit values in chunks of eight columns, as the norm and the 4-bit products read
// and write them (internal).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "common.cuh"

namespace xnor {

// Where rows and their number of columns allow it, a chunk moves as 16-byte pieces; else element by element.
__host__ inline bool rows_in_pieces(const void *p, long long stride, int cols, size_t elem) {
  return p == nullptr ||
         ((reinterpret_cast<uintptr_t>(p) & 15u) == 0 && (stride * (long long)elem) % 16 == 0 && cols % 8 == 0);
}

__device__ __forceinline__ uint4 load_global(const uint4 *p) {
  uint4 v;
  asm volatile("ld.global.v4.b32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(__cvta_generic_to_global(p)));
  return v;
}
__device__ __forceinline__ uint16_t load_global(const uint16_t *p) {
  uint16_t v;
  asm volatile("ld.global.b16 %0, [%1];" : "=h"(v) : "l"(__cvta_generic_to_global(p)));
  return v;
}
__device__ __forceinline__ uint8_t load_global(const uint8_t *p) {
  uint32_t v;
  asm volatile("ld.global.u8 %0, [%1];" : "=r"(v) : "l"(__cvta_generic_to_global(p)));
  return (uint8_t)v;
}

__device__ __forceinline__ float2 pair_to_float(uint32_t w, __nv_bfloat16) {
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));      // (one instruction each)
}
__device__ __forceinline__ float2 pair_to_float(uint32_t w, __half) {
  return __half22float2(*reinterpret_cast<const __half2 *>(&w));
}
__device__ __forceinline__ uint32_t float_to_pair(float a, float b, __nv_bfloat16) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ uint32_t float_to_pair(float a, float b, __half) {
  const __half2 v = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t *>(&v);
}

// Eight values as they lie in memory.
template <class T>
struct Chunk {
  static constexpr int kWords = (int)sizeof(T) * 2;
  uint32_t w[kWords];

  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = 0u;
  }
  // p: the chunk's first element; in: how many of its eight columns exist
  __device__ __forceinline__ void load(const T *p, bool pieces, int in) {
    if (pieces) {
      if (in > 0) {
#pragma unroll
        for (int i = 0; i < kWords / 4; ++i) {
          const uint4 v = load_global(reinterpret_cast<const uint4 *>(p) + i);
          w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
        }
      } else {
        zero();
      }
      return;
    }
    zero();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (i >= in) continue;
      if constexpr (sizeof(T) == 4) w[i] = load_global(reinterpret_cast<const uint32_t *>(p) + i);
      else w[i / 2] |= (uint32_t)load_global(reinterpret_cast<const uint16_t *>(p) + i) << (16 * (i & 1));
    }
  }
  __device__ __forceinline__ void store(T *p, bool pieces, int in) const {
    if (pieces) {
      if (in > 0) {
#pragma unroll
        for (int i = 0; i < kWords / 4; ++i)
          reinterpret_cast<uint4 *>(p)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
      }
      return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (i >= in) continue;
      if constexpr (sizeof(T) == 4) reinterpret_cast<uint32_t *>(p)[i] = w[i];
      else reinterpret_cast<uint16_t *>(p)[i] = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
    }
  }
  __device__ __forceinline__ void to_float(float v[8]) const {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 f = pair_to_float(w[i], T());
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
      }
    }
  }
  __device__ __forceinline__ void from_float(const float v[8]) {      // to nearest even
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(v[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = float_to_pair(v[2 * i], v[2 * i + 1], T());
    }
  }
};

// Root-mean-square norm (xnor_rmsnorm and its kin).
struct NormArgs {
  const void *x, *residual, *weight;
  void *sum, *y;
  float *rstd;
  void *q;                    // 8-bit output and its scales
  float *scales;
  int q_type, group;          // group 0: the whole row
  xnor_norm_desc d;
  float per_col;              // 1 / cols
};
cudaError_t launch_rmsnorm(const NormArgs &a, cudaStream_t st);
struct NormBackwardArgs {
  const void *dy, *dsum, *h, *weight;
  const float *rstd;
  void *dx;
  float *dweight, *work;
  xnor_norm_desc d;
  float per_col;
};
cudaError_t launch_rmsnorm_backward(const NormBackwardArgs &a, cudaStream_t st);
cudaError_t read_status_norm(int *status);
int rmsnorm_parts(int rows, int cols);     // rows of partial sums in the workspace
constexpr int kNormMaxCols = 32768;

// 4-bit weights.
constexpr int kW4Rows = 16, kW4Cols = 64;  // a tile: 16 rows of 64 columns, 512 bytes
constexpr int kW4Panel = 8;                // row tiles whose tiles of a column lie together
inline int w4_row_tiles(const xnor_w4_desc &d) { return d.N / kW4Rows + (d.N % kW4Rows != 0); }
inline int w4_panels(const xnor_w4_desc &d) { return (w4_row_tiles(d) + kW4Panel - 1) / kW4Panel; }
inline int w4_col_tiles(const xnor_w4_desc &d) { return d.K / kW4Cols + (d.K % kW4Cols != 0); }
cudaError_t launch_w4_quantize(const void *w, int type, const xnor_w4_desc &d, uint32_t *w_packed, float *scales,
                               uint8_t *zeros, cudaStream_t st);
cudaError_t launch_w4_pack(const uint8_t *codes, const xnor_w4_desc &d, uint32_t *w_packed, cudaStream_t st);
cudaError_t launch_w4_dequantize(const uint32_t *w_packed, const float *scales, const uint8_t *zeros,
                                 const xnor_w4_desc &d, int type, void *w, cudaStream_t st);
struct W4Args {
  const void *x;
  const float *x_scales;
  const uint32_t *w;
  const float *scales;
  const uint8_t *zeros;
  void *out;
  xnor_w4_desc d;
  xnor_w4_rows r;
};
cudaError_t launch_w4_few_rows(const W4Args &a, cudaStream_t st);
cudaError_t launch_w4_many_rows(const W4Args &a, cudaStream_t st);
cudaError_t read_status_w4(int *status);   // of the kernel for many rows, as the others'
// Which kernel: up to 8 rows the one for few rows is never slower (8 rows times 16384x4096 12.0 us, 15.9 in the other); 9 to
// 16 take it two passes' worth of registers, which pays for matrices that take a few microseconds only (12 rows times
// 4096x4096 6.9 against 8.9, times 8192x4096 12.3 against 11.3).
inline bool w4_few_rows(const xnor_w4_desc &d, int rows) { return rows <= 8 || (rows <= 16 && (long long)d.N * d.K <= 24ll << 20); }

}  // namespace xnor
