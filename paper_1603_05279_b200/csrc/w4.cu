// 4-bit weights with a scale for each group of columns: quantised from real weights, laid out from given
// codes, dequantised, and multiplied with a few rows.
#include <algorithm>
#include <climits>
#include <type_traits>

#include "umma_common.cuh"
#include "w4.cuh"

namespace xnor {

namespace {

// ---- layout -------------------------------------------------------------------------------
// A block: 16 rows x 256 columns, two steps of 128 columns (the largest group) whose loads are under way together; a
// thread: 16 columns of a row in each.
constexpr int kLayThreads = 128, kLaySteps = 2;
constexpr int kStepCols = 2 * kW4Cols, kLayCols = kLaySteps * kStepCols;
constexpr int kOctets = kStepCols / 8;
using LayWords = uint32_t[kLaySteps][kW4Rows][kOctets + 1];     // [steps][rows][groups of eight columns]

// Words of the block to the packed tiles: a warp, a tile.
__device__ __forceinline__ void write_tiles(const LayWords &words, int row_tile, int col_tile0, int col_tiles, uint32_t *w) {
  const int tile = threadIdx.x / 32, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  if (col_tile0 + tile >= col_tiles) return;
  const uint32_t (&s)[kW4Rows][kOctets + 1] = words[tile / 2];
  const int c = 8 * (tile & 1) + (t ^ ((g >> 1) & 3));      // this place's columns
  reinterpret_cast<uint4 *>(w)[(w4_tile(row_tile, col_tiles) + (size_t)(col_tile0 + tile) * kW4Panel) * 32 + lane] =
      make_uint4(s[g][c], s[g][c + 4], s[g + 8][c], s[g + 8][c + 4]);
}

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

// Thread (row r, 16 columns c ..): the scale of its group over 2, 4 or 8 neighbouring threads, then its codes.  A group
// is 2^lg columns.  NaN and infinity make its scale such, and its codes those of zero.
template <class T, bool kZeros>
__global__ void __launch_bounds__(kLayThreads)
w4_quantize_kernel(const T *w, const xnor_w4_desc d, int lg, int pieces, uint32_t *w_packed, float *scales, uint8_t *zeros) {
  __shared__ LayWords words;
  stream_order();
  const int r = threadIdx.x / 8, c = threadIdx.x % 8;
  const int n = blockIdx.y * kW4Rows + r;
  Chunk<T> in[kLaySteps][2];
  {
    const T *from = w + (size_t)min(n, d.N - 1) * d.K;
#pragma unroll
    for (int step = 0; step < kLaySteps; ++step)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int k = blockIdx.x * kLayCols + step * kStepCols + 16 * c + 8 * i;
        in[step][i].load(from + k, pieces, n < d.N ? min(8, max(0, d.K - k)) : 0);
      }
  }
#pragma unroll
  for (int step = 0; step < kLaySteps; ++step) {
    const int k = blockIdx.x * kLayCols + step * kStepCols + 16 * c;
    float v[16];
#pragma unroll
    for (int i = 0; i < 2; ++i) in[step][i].to_float(*reinterpret_cast<float (*)[8]>(v + 8 * i));
    const int lanes = 1 << (lg - 4);
    float s, z = 8.0f, lo = 0.0f, q[16];
    if constexpr (kZeros) {
      float hi = 0.0f, odd = 0.0f;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        lo = fminf(lo, v[i]);
        hi = fmaxf(hi, v[i]);
        odd = fmaf(v[i], 0.0f, odd);                     // NaN if any is NaN or infinite
      }
#pragma unroll
      for (int o = 1; o < 8; o *= 2) {
        const float ol = __shfl_xor_sync(0xffffffffu, lo, o), oh = __shfl_xor_sync(0xffffffffu, hi, o), oo = __shfl_xor_sync(0xffffffffu, odd, o);
        if (o < lanes) { lo = fminf(lo, ol); hi = fmaxf(hi, oh); odd += oo; }
      }
      s = (float)(((double)hi - (double)lo) / 15.0);
      if (odd != 0.0f && s <= 3.402823466e38f) s = odd;  // (infinite extremes have made it such)
    } else {
      uint32_t m = 0u;                                   // of bit patterns of magnitudes: a NaN is above every number
#pragma unroll
      for (int i = 0; i < 16; ++i) m = max(m, __float_as_uint(v[i]) & 0x7FFFFFFFu);
#pragma unroll
      for (int o = 1; o < 8; o *= 2) {
        const uint32_t om = __shfl_xor_sync(0xffffffffu, m, o);
        if (o < lanes) m = max(m, om);
      }
      s = __fdiv_rn(__uint_as_float(m), 7.0f);
    }
    const bool sound = s > 0.0f && s <= 3.402823466e38f;
    const float inv = sound && s > 1e-37f ? 1.0f / s : 0.0f;      // 0: it would overflow
    if (kZeros && sound) z = fminf(15.0f, fmaxf(0.0f, round_quotient(-lo, s)));
    if (sound) {
      round_quotients(v, s, inv, z, q);
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) q[i] = 0.0f;
    }
    if constexpr (kZeros) {
#pragma unroll
      for (int i = 0; i < 16; ++i) q[i] = fminf(q[i] + z, 15.0f);          // (at least 0: z rounds as the least value does, or the quotient is cut)
    }
    const float base = kZeros ? 8388608.0f : 8388608.0f + 8.0f * 4369.0f;  // 2^23, and a zero point of 8 in every code
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float *u = q + 8 * h;
      const uint32_t even = __float_as_uint(four_codes(u[0] + base, u[2], u[4], u[6])), odd = __float_as_uint(four_codes(u[1] + base, u[3], u[5], u[7]));
      words[step][r][2 * c + h] = __byte_perm(even, odd, 0x5410);
    }
    if (n < d.N && k < d.K && (c & (lanes - 1)) == 0) {
      const size_t at = (size_t)(k >> lg) * d.N + n;
      scales[at] = s;
      if constexpr (kZeros) zeros[at] = (uint8_t)z;
    }
  }
  __syncthreads();
  write_tiles(words, blockIdx.y, blockIdx.x * (kLayCols / kW4Cols), (d.K + kW4Cols - 1) / kW4Cols, w_packed);
}

__global__ void __launch_bounds__(kLayThreads)
w4_pack_kernel(const uint8_t *codes, const xnor_w4_desc d, uint32_t *w_packed) {
  __shared__ LayWords words;
  stream_order();
  const int r = threadIdx.x / 8, c = threadIdx.x % 8;
  const int n = blockIdx.y * kW4Rows + r;
  const bool pieces = d.K % 8 == 0;
#pragma unroll
  for (int q = 0; q < 2 * kLaySteps; ++q) {
    const int k = blockIdx.x * kLayCols + (q / 2) * kStepCols + 16 * c + 8 * (q & 1);
    uint32_t word = 0x88888888u;
    if (n < d.N && k < d.K) {
      const uint8_t *from = codes + (size_t)n * d.K + k;
      if (pieces) {
        const uint2 v = load_global(reinterpret_cast<const uint2 *>(from));
        const uint32_t a = v.x & 0x0F0F0F0Fu, b = v.y & 0x0F0F0F0Fu;         // codes 0 .. 3 and 4 .. 7, one in each byte
        const uint32_t even = __byte_perm(a, b, 0x6420), odd = __byte_perm(a, b, 0x7531);
        word = __byte_perm(even | even >> 4, odd | odd >> 4, 0x6420);
      } else {
        word = 0u;
#pragma unroll
        for (int i = 0; i < 8; ++i) word |= (k + i < d.K ? load_global(from + i) & 15u : 8u) << w4_bit(i);
      }
    }
    words[q / 2][r][2 * c + (q & 1)] = word;
  }
  __syncthreads();
  write_tiles(words, blockIdx.y, blockIdx.x * (kLayCols / kW4Cols), (d.K + kW4Cols - 1) / kW4Cols, w_packed);
}

template <class T>
__global__ void __launch_bounds__(kLayThreads)
w4_dequantize_kernel(const uint32_t *w_packed, const float *scales, const uint8_t *zeros, const xnor_w4_desc d,
                     int lg, int pieces, uint32_t magic, T *w) {
  __shared__ uint32_t words[kLayCols / kW4Cols][32][5];
  stream_order();
  const int col_tiles = (d.K + kW4Cols - 1) / kW4Cols;
  {
    const int tile = threadIdx.x / 32, lane = threadIdx.x & 31, ct = blockIdx.x * (kLayCols / kW4Cols) + tile;
    if (ct < col_tiles) {
      const uint4 v = load_global(reinterpret_cast<const uint4 *>(w_packed) + (w4_tile(blockIdx.y, col_tiles) + (size_t)ct * kW4Panel) * 32 + lane);
      words[tile][lane][0] = v.x; words[tile][lane][1] = v.y; words[tile][lane][2] = v.z; words[tile][lane][3] = v.w;
    }
  }
  const int r = threadIdx.x / 8, c = threadIdx.x % 8, n = blockIdx.y * kW4Rows + r;
  float s[kLaySteps];
  uint32_t z[kLaySteps];
#pragma unroll
  for (int step = 0; step < kLaySteps; ++step) {
    const int k = blockIdx.x * kLayCols + step * kStepCols + 16 * c;
    const bool in = n < d.N && k < d.K;
    const size_t at = in ? (size_t)(k >> lg) * d.N + n : 0;  // 16 columns lie in one group
    s[step] = load_global(scales + at);
    z[step] = zeros ? load_global(zeros + at) : 8u;
  }
  __syncthreads();
  if (n >= d.N) return;
#pragma unroll
  for (int step = 0; step < kLaySteps; ++step) {
    const int k = blockIdx.x * kLayCols + step * kStepCols + 16 * c;
    if (k >= d.K) return;
    const W4Type<__nv_bfloat16>::Zero zero = W4Type<__nv_bfloat16>::zero(z[step]);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int col = 16 * (c & 3) + 8 * h;
      uint32_t pair[4];
      W4Type<__nv_bfloat16>::expand(words[2 * step + c / 4][w4_place(r, col)][w4_word(r, col)], zero, magic, pair);
      float v[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 f = pair_to_float(pair[i], __nv_bfloat16());
        v[2 * i] = f.x * s[step];
        v[2 * i + 1] = f.y * s[step];
      }
      Chunk<T> a;
      a.from_float(v);
      a.store(w + (size_t)n * d.K + k + 8 * h, pieces, min(8, max(0, d.K - (k + 8 * h))));
    }
  }
}

// ---- a few rows ---------------------------------------------------------------------------
// out[t][n] = x_scale[t] sum over groups of scale[g][n] sum over the group of (code - zero)[n][k] x[t][k].
// Codes minus zeros and the rows' values are exact 16-bit operands of m16n8k16 products summed in 32 bits: 16
// weight rows against 8 rows of x per step, whatever few of those exist (no extra traffic: the lanes of missing
// rows read the last one).  Bound by the weights' bytes.  A warp multiplies kR tiles of 16 weight rows with the
// same rows of x in its registers; the warps of a block and the blocks of its cluster divide the columns, and
// add their sums in shared memory in a fixed order.
constexpr int kFewThreads = 256, kFewWarps = kFewThreads / 32;
constexpr int kMaxSplit = 8;

// d = a b + c
template <class T>
__device__ __forceinline__ void mma_16x8x16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, const float *c) {
  if constexpr (std::is_same<T, __half>::value)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %12, %13};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %12, %13};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
}

// kN: blocks of eight rows of x; kR: tiles of weight rows; kGroup, kZeros: as the weights have them; kU: column
// tiles of a stage (a group of 128 stays in one: 2).
template <int kType, int kN, int kR, int kGroup, bool kZeros>
__global__ void __launch_bounds__(kFewThreads, kN == 1 ? 2 : 1)
w4_few_rows_kernel(const W4Args A, int pieces, uint32_t magic) {
  using T = typename RowsOf<kType>::T;
  constexpr int kB = RowsOf<kType>::kBytes, kU = 2, kCols = kU * kW4Cols, kS = kCols / kGroup;
  constexpr int kTok = 8 * kN, kOut = kW4Rows * kR;
  extern __shared__ float shared[];
  float *part = shared;                                     // [warps][kTok][kOut + 1]
  float *sums = shared + kFewWarps * kTok * (kOut + 1);     // [kTok][kOut]
  stream_order();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const int N = A.d.N, K = A.d.K;
  const int col_tiles = (K + kW4Cols - 1) / kW4Cols, row_tiles = (N + kW4Rows - 1) / kW4Rows, groups = (K + kGroup - 1) / kGroup;
  const int split = gridDim.x, rank = blockIdx.x;           // blocks of the cluster
  const int n0 = blockIdx.y * kOut;
  // stages of two column tiles: this warp's
  const unsigned stages = (unsigned)(col_tiles + kU - 1) / kU, slice = (unsigned)(rank * kFewWarps + warp);
  const int lg = 31 - __clz(split * kFewWarps);             // a power of two of slices; fewer than 2^18 stages
  const int st0 = (int)((stages * slice) >> lg), st1 = (int)((stages * (slice + 1)) >> lg);
  const uint8_t *x[kN];
#pragma unroll
  for (int i = 0; i < kN; ++i)
    x[i] = static_cast<const uint8_t *>(A.x) + (long long)min(8 * i + g, A.r.rows - 1) * A.r.x_stride * kB;
  const uint4 *w[kR];
  int na[kR], nb[kR];                                       // this lane's weight rows, inside the matrix
#pragma unroll
  for (int i = 0; i < kR; ++i) {
    w[i] = reinterpret_cast<const uint4 *>(A.w) + w4_tile(min((int)blockIdx.y * kR + i, row_tiles - 1), col_tiles) * 32 + w4_place(g, 8 * t);
    na[i] = min(n0 + kW4Rows * i + g, N - 1);
    nb[i] = min(n0 + kW4Rows * i + g + 8, N - 1);
  }
  const bool x_groups = kB == 1 && A.r.x_group != 0;
  float total[kR][kN][4] = {};

  struct Stage {
    uint4 w[kR][kU];
    uint32_t x[kN][2 * kU][2 * kB];         // as they lie in memory: a conversion would wait for its load
    float sa[kR][kS], sb[kR][kS];
    uint32_t za[kR][kS], zb[kR][kS];
  };
  // this lane's part of stage 0; a stage is one multiply-add from there
  const float *pa[kR], *pb[kR];
  const uint8_t *qa[kR], *qb[kR];
#pragma unroll
  for (int i = 0; i < kR; ++i) {
    pa[i] = A.scales + na[i];
    pb[i] = A.scales + nb[i];
    qa[i] = A.zeros + (kZeros ? na[i] : 0);
    qb[i] = A.zeros + (kZeros ? nb[i] : 0);
  }
#pragma unroll
  for (int i = 0; i < kN; ++i) x[i] += 8 * t * kB;
  // stages that lie inside the rows, at addresses that allow whole pieces
  const int sound = pieces ? min(st1, K / kCols) : st0;
  auto load = [&](int st, Stage &s) {
    if (st >= sound) return;
#pragma unroll
    for (int i = 0; i < kR; ++i) {
      const uint4 *p = w[i] + (long long)st * (kU * kW4Panel * 32);
#pragma unroll
      for (int u = 0; u < kU; ++u) s.w[i][u] = load_global(p + u * kW4Panel * 32);
    }
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const uint8_t *p = x[i] + (long long)st * (kCols * kB);
#pragma unroll
      for (int h = 0; h < 2 * kU; ++h) load_x8_raw<kType>(p, 32 * h, INT_MAX, true, s.x[i][h]);
    }
#pragma unroll
    for (int h = 0; h < kS; ++h) {
      const long long at = (long long)st * (kS * N) + h * N;
#pragma unroll
      for (int i = 0; i < kR; ++i) {
        s.sa[i][h] = load_global(pa[i] + at);
        s.sb[i][h] = load_global(pb[i] + at);
        s.za[i][h] = kZeros ? load_global(qa[i] + at) : 8u;
        s.zb[i][h] = kZeros ? load_global(qb[i] + at) : 8u;
      }
    }
  };
  auto load_any = [&](int st, Stage &s) {
#pragma unroll
    for (int i = 0; i < kR; ++i)
#pragma unroll
      for (int u = 0; u < kU; ++u) s.w[i][u] = load_global(w[i] + (size_t)min(st * kU + u, col_tiles - 1) * (kW4Panel * 32));
#pragma unroll
    for (int i = 0; i < kN; ++i)
#pragma unroll
      for (int h = 0; h < 2 * kU; ++h) load_x8_raw<kType>(x[i], st * kCols + 32 * h, K - 8 * t, pieces, s.x[i][h]);
#pragma unroll
    for (int h = 0; h < kS; ++h) {
      // a group that does not exist counts nothing: its columns of x are zeros, and so is its scale
      const bool there = st * kS + h < groups;
      const long long at = there ? (long long)(st * kS + h) * N : 0;
#pragma unroll
      for (int i = 0; i < kR; ++i) {
        s.sa[i][h] = there ? load_global(pa[i] + at) : 0.0f;
        s.sb[i][h] = there ? load_global(pb[i] + at) : 0.0f;
        s.za[i][h] = kZeros ? load_global(qa[i] + at) : 8u;
        s.zb[i][h] = kZeros ? load_global(qb[i] + at) : 8u;
      }
    }
  };
  auto multiply = [&](int st, const Stage &s) {
    const float none[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    uint32_t xv[kN][2 * kU][4];
#pragma unroll
    for (int n = 0; n < kN; ++n)
#pragma unroll
      for (int h = 0; h < 2 * kU; ++h) x8_pairs<kType>(s.x[n][h], xv[n][h]);
#pragma unroll
    for (int i = 0; i < kR; ++i) {
      float acc[kN][4];
#pragma unroll
      for (int h = 0; h < 2 * kU; ++h) {                    // 32 columns
        const int grp = 32 * h / kGroup;
        const uint4 q = s.w[i][h / 2];
        const uint32_t va = h % 2 ? q.y : q.x, vb = h % 2 ? q.w : q.z;
        uint32_t ra[4], rb[4];
        W4Type<T>::expand(va, W4Type<T>::zero(s.za[i][grp]), magic, ra);
        W4Type<T>::expand(vb, W4Type<T>::zero(s.zb[i][grp]), magic, rb);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const uint32_t a[4] = {ra[2 * j], rb[2 * j], ra[2 * j + 1], rb[2 * j + 1]};
#pragma unroll
          for (int n = 0; n < kN; ++n)
            mma_16x8x16<T>(acc[n], a, xv[n][h][2 * j], xv[n][h][2 * j + 1], 32 * h % kGroup == 0 && j == 0 ? none : acc[n]);
        }
        if ((32 * h + 32) % kGroup != 0) continue;          // the group goes on
        const float sa = s.sa[i][grp], sb = s.sb[i][grp];
#pragma unroll
        for (int n = 0; n < kN; ++n) {
          if (kB == 1 && x_groups) {
            const long long t0 = min(8 * n + 2 * t, A.r.rows - 1), t1 = min(8 * n + 2 * t + 1, A.r.rows - 1);
            const int at = min(st * kS + grp, groups - 1);
            const float s0 = load_global(A.x_scales + t0 * groups + at), s1 = load_global(A.x_scales + t1 * groups + at);
            acc[n][0] *= s0; acc[n][1] *= s1; acc[n][2] *= s0; acc[n][3] *= s1;
          }
          total[i][n][0] = fmaf(acc[n][0], sa, total[i][n][0]);
          total[i][n][1] = fmaf(acc[n][1], sa, total[i][n][1]);
          total[i][n][2] = fmaf(acc[n][2], sb, total[i][n][2]);
          total[i][n][3] = fmaf(acc[n][3], sb, total[i][n][3]);
        }
      }
    }
  };
  // stages come in two ahead, by name (moving one to the other would wait for its loads)
  Stage s0, s1;
  load(st0, s0);
  load(st0 + 1, s1);
#pragma unroll 1
  for (int st = st0; st < sound; st += 2) {
    multiply(st, s0);
    load(st + 2, s0);
    if (st + 1 >= sound) break;
    multiply(st + 1, s1);
    load(st + 3, s1);
  }
  // what is left: the ragged end of the rows, or all of them
#pragma unroll 1
  for (int st = max(st0, sound); st < st1; ++st) {
    load_any(st, s0);
    multiply(st, s0);
  }
#pragma unroll
  for (int i = 0; i < kR; ++i)
#pragma unroll
    for (int n = 0; n < kN; ++n) {
      float *p = part + (warp * kTok + 8 * n + 2 * t) * (kOut + 1) + kW4Rows * i + g;
      p[0] = total[i][n][0];
      p[kOut + 1] = total[i][n][1];
      p[8] = total[i][n][2];
      p[kOut + 1 + 8] = total[i][n][3];
    }
  __syncthreads();
  const int toks = A.r.rows;
  for (int e = threadIdx.x; e < toks * kOut; e += kFewThreads) {
    const int n = e % kOut, tok = e / kOut;
    float s = part[tok * (kOut + 1) + n];
#pragma unroll
    for (int i = 1; i < kFewWarps; ++i) s += part[(i * kTok + tok) * (kOut + 1) + n];
    sums[e] = s;
  }
  if (split > 1) umma::cluster_sync();
  // (without a cluster every thread reads what it wrote itself)
  // the cluster's blocks write the outputs in turn; each adds the blocks' sums in the same order
  for (int e = rank * kFewThreads + threadIdx.x; e < toks * kOut; e += split * kFewThreads) {
    const int n = e % kOut;
    float s = 0.0f;
    if (split == 1) s = sums[e];
    else
      for (int i = 0; i < split; ++i) {
        uint32_t a;
        float v;
        asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"((uint32_t)__cvta_generic_to_shared(sums + e)), "r"(i));
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
        s += v;
      }
    if (n0 + n >= N) continue;
    const long long row = e / kOut;
    if (A.x_scales != nullptr && !x_groups) s *= load_global(A.x_scales + row);
    const size_t at = (size_t)(row * A.r.out_stride) + n0 + n;
    if (A.r.out_type == XNOR_F32) static_cast<float *>(A.out)[at] = s;
    else if (A.r.out_type == XNOR_BF16) static_cast<__nv_bfloat16 *>(A.out)[at] = __float2bfloat16_rn(s);
    else static_cast<__half *>(A.out)[at] = __float2half_rn(s);
  }
  if (split > 1) umma::cluster_sync();
}

template <int kType, int kN, int kR, int kGroup, bool kZeros>
cudaError_t few_rows(const W4Args &a, cudaStream_t st) {
  constexpr int kTok = 8 * kN, kOut = kW4Rows * kR;        // rows of x: kTok at most
  constexpr size_t kSmem = (size_t)(kFewWarps * kTok * (kOut + 1) + kTok * kOut) * sizeof(float);
  static_assert(kSmem <= 48 * 1024, "shared memory");
  const int blocks = (w4_row_tiles(a.d) + kR - 1) / kR, col_tiles = w4_col_tiles(a.d);
  // blocks of a cluster divide the columns while the blocks are fewer than the GPU has SMs and every warp
  // keeps two tiles
  int split = 1;
  while (split < kMaxSplit && blocks * split < sm_count_of_current_device() && col_tiles >= 4 * split * kFewWarps) split *= 2;
  const int pieces = rows_in_pieces(a.x, a.r.x_stride, 8, RowsOf<kType>::kBytes);
  const dim3 grid((unsigned)split, (unsigned)blocks);
  return launch_kernel(w4_few_rows_kernel<kType, kN, kR, kGroup, kZeros>, grid, kFewThreads, kSmem, st, (unsigned)split, a, pieces,
                       W4Type<typename RowsOf<kType>::T>::kMagic);
}
// Two tiles of weight rows share the rows of x in registers, where two stages of them fit (small groups and zero points
// take registers too).
template <int kType, int kN, int kGroup>
cudaError_t few_rows(const W4Args &a, cudaStream_t st) {
  if (a.zeros) return few_rows<kType, kN, 1, kGroup, true>(a, st);
  return few_rows<kType, kN, kGroup == 32 || kN == 2 ? 1 : 2, kGroup, false>(a, st);
}
template <int kType, int kN>
cudaError_t few_rows(const W4Args &a, cudaStream_t st) {
  return a.d.group == 32 ? few_rows<kType, kN, 32>(a, st) : a.d.group == 64 ? few_rows<kType, kN, 64>(a, st) : few_rows<kType, kN, 128>(a, st);
}
template <int kType>
cudaError_t few_rows(const W4Args &a, cudaStream_t st) {
  return a.r.rows <= 8 ? few_rows<kType, 1>(a, st) : few_rows<kType, 2>(a, st);
}

dim3 lay_grid(const xnor_w4_desc &d) { return dim3((unsigned)((d.K + kLayCols - 1) / kLayCols), (unsigned)w4_row_tiles(d)); }
// ... of every row tile of the panels
dim3 fill_grid(const xnor_w4_desc &d) { return dim3(lay_grid(d).x, (unsigned)(w4_panels(d) * kW4Panel)); }

}  // namespace

namespace {

int log2_of(int group) { return group == 32 ? 5 : group == 64 ? 6 : 7; }

template <class T>
cudaError_t quantize(const void *w, const xnor_w4_desc &d, uint32_t *w_packed, float *scales, uint8_t *zeros, cudaStream_t st) {
  const int lg = log2_of(d.group), pieces = d.K % 8 == 0;
  if (zeros) return launch_kernel(w4_quantize_kernel<T, true>, fill_grid(d), kLayThreads, 0, st, 1, (const T *)w, d, lg, pieces, w_packed, scales, zeros);
  return launch_kernel(w4_quantize_kernel<T, false>, fill_grid(d), kLayThreads, 0, st, 1, (const T *)w, d, lg, pieces, w_packed, scales, zeros);
}

template <class T>
cudaError_t dequantize(const uint32_t *w_packed, const float *scales, const uint8_t *zeros, const xnor_w4_desc &d, void *w, cudaStream_t st) {
  return launch_kernel(w4_dequantize_kernel<T>, lay_grid(d), kLayThreads, 0, st, 1, w_packed, scales, zeros, d, log2_of(d.group), (int)(d.K % 8 == 0),
                       W4Type<__nv_bfloat16>::kMagic, (T *)w);
}

}  // namespace

cudaError_t launch_w4_quantize(const void *w, int type, const xnor_w4_desc &d, uint32_t *w_packed, float *scales,
                               uint8_t *zeros, cudaStream_t st) {
  if (type == XNOR_F32) return quantize<float>(w, d, w_packed, scales, zeros, st);
  return type == XNOR_BF16 ? quantize<__nv_bfloat16>(w, d, w_packed, scales, zeros, st) : quantize<__half>(w, d, w_packed, scales, zeros, st);
}

cudaError_t launch_w4_pack(const uint8_t *codes, const xnor_w4_desc &d, uint32_t *w_packed, cudaStream_t st) {
  return launch_kernel(w4_pack_kernel, fill_grid(d), kLayThreads, 0, st, 1, codes, d, w_packed);
}

cudaError_t launch_w4_dequantize(const uint32_t *w_packed, const float *scales, const uint8_t *zeros,
                                 const xnor_w4_desc &d, int type, void *w, cudaStream_t st) {
  if (type == XNOR_F32) return dequantize<float>(w_packed, scales, zeros, d, w, st);
  return type == XNOR_BF16 ? dequantize<__nv_bfloat16>(w_packed, scales, zeros, d, w, st) : dequantize<__half>(w_packed, scales, zeros, d, w, st);
}

cudaError_t launch_w4_few_rows(const W4Args &a, cudaStream_t st) {
  if (a.r.rows == 0) return cudaSuccess;
  switch (a.r.x_type) {
    case XNOR_BF16: return few_rows<XNOR_BF16>(a, st);
    case XNOR_F16: return few_rows<XNOR_F16>(a, st);
    case XNOR_I8: return few_rows<XNOR_I8>(a, st);
    default: return few_rows<XNOR_E4M3>(a, st);
  }
}

}  // namespace xnor
