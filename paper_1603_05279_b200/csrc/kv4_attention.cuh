// What the kernels of attention over the cache in 4 bits have in common (internal).
#pragma once
#include "kv4.cuh"
#include "umma_common.cuh"

namespace xnor {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// A row's maximum is left behind by 2^8 at most: then P, up to 2^8 times a value's scale, is rounded to F16, relative to a
// power of two 2^e above the largest scale so far that the row sees and times 2^7.  That is at most 2^15, and has all 11 bits
// down to 2^-21 of that scale.  (As bfloat16 it gave outputs in bfloat16 half as much again of error.)  Outputs in F16 would show it: there
// what the rounding left is a second operand, and 22 bits are kept (16 sequences of 2000 tokens, five new: error 0.0003 -> 0.0002, which is
// the output's own rounding, 20.2 -> 21.2 us; prompts of 2000, 1000 and 333 tokens, 40 heads of 128 on 8, 115 -> 135 us).
constexpr float kRaise = 8.0f;
constexpr int kLift = 7;
template <class T> constexpr bool kTwoParts = false;
template <> constexpr bool kTwoParts<__half> = true;

// (a wait that gave up is the graver: that is written over this, and this not over that)
__device__ __forceinline__ void record_bounds(int *status) { atomicCAS(status, 0, (int)XNOR_ERR_BOUNDS); }

struct Sequence;
// How a call's rows are cut: tiles of `rows` queries of a head's group, units of `tokens`; of sequences with more than
// `least` and at most `most` rows.
struct Tiling {
  int group, rows, tokens, total_rows;
  int least, most;
  // Records lengths that the table has no room for; for all threads of a warp.
  __device__ __forceinline__ void check_lengths(const Kv4Where &W, int lane, int *status) const;
};

// A sequence of n new tokens and L in all has kv_heads x ceil(n group / rows) items of max(1, ceil(L / tokens)) units.
struct Sequence {
  int start, n, len;           // first row, rows (0: not of this kernel's), tokens that the table has room for
  int lead;                    // a row's last visible token, less the row
  int tiles, units;            // units: of an item
  bool cut;                    // longer than the table has room for
  __device__ __forceinline__ void load(const Kv4Where &W, const Tiling &T, int b) {
    const int end = load_int(W.starts + b + 1), all = load_int(W.lens + b);
    start = max(0, load_int(W.starts + b));
    n = max(0, min(T.total_rows, end) - start);
    const long long r = (long long)n * T.group;
    if (r <= T.least || r > T.most) n = 0;
    len = (int)min((long long)max(0, all), (long long)W.d.table_cols * W.d.page);
    lead = max(0, all) - end;
    cut = n > 0 && all > len;
    tiles = n > 0 ? (int)((r + T.rows - 1) / T.rows) : 0;
    units = max(1, (len + T.tokens - 1) / T.tokens);
  }
  // What thread `lane` of the warp has.
  __device__ __forceinline__ Sequence of(int lane) const {
    Sequence r = *this;
    r.start = __shfl_sync(0xffffffffu, start, lane);
    r.n = __shfl_sync(0xffffffffu, n, lane);
    r.len = __shfl_sync(0xffffffffu, len, lane);
    r.lead = __shfl_sync(0xffffffffu, lead, lane);
    r.tiles = __shfl_sync(0xffffffffu, tiles, lane);
    r.units = __shfl_sync(0xffffffffu, units, lane);
    return r;
  }
  __device__ __forceinline__ long long all(int kv_heads) const { return (long long)kv_heads * tiles * units; }
};

__device__ __forceinline__ void Tiling::check_lengths(const Kv4Where &W, int lane, int *status) const {
  bool cut = false;
  for (int b = (int)blockIdx.x * 32 + lane; b < W.d.seqs; b += (int)gridDim.x * 32) {
    Sequence s;
    s.load(W, *this, b);
    cut = cut || s.cut;
  }
  if (cut) record_bounds(status);
}

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// 2^i; 0 below fp32's normal numbers.
__device__ __forceinline__ float power_of_two(int i) { return i < -126 ? 0.0f : __uint_as_float((uint32_t)(i + 127) << 23); }
// 1 / 2^i, of a normal number whose inverse is one.
__device__ __forceinline__ float inverse_power(float v) { return __uint_as_float((254u << 23) - __float_as_uint(v)); }
// The power of two above a scale, within limits that keep all its uses normal numbers.  Infinity and NaN do not count.
constexpr int kLeastScale = -100, kMostScale = 127;
__device__ __forceinline__ int scale_above(float s) {
  const int i = (int)(__float_as_uint(s) >> 23) & 255;
  return i == 255 ? kLeastScale : min(kMostScale, max(kLeastScale, i - 126));
}

template <class K>
cudaError_t allow_shared(K *kernel, size_t bytes, bool (&flags)[64]) {
  bool &set = attr_done_for_current_device(flags);
  if (set) return cudaSuccess;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  if (e != cudaSuccess) (void)cudaGetLastError();
  set = e == cudaSuccess;
  return e;
}

}  // namespace xnor
