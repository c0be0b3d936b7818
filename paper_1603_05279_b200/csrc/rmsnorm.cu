// Root-mean-square norm of rows with the residual's addition, in the rows' type or in 8 bits with scales, and
// its backward pass.  Every row is read once: its values stay in the registers of a team of threads.
//
// HBM bounds them.  The forward pass gets there with enough loads under way in registers (8192x4096 bf16 with residual
// 43.7 us, 0.94 of the copy bandwidth); a ring of rows in shared memory, filled by bulk copies, took longer there (59:
// fewer warps for the same work).  The backward pass, which has the sums of the weight's gradient in its registers too,
// needs that ring for long rows in numbers (4096x4096 39 -> 34 us): persistent blocks, one row at a time.
#include <algorithm>
#include <type_traits>

#include "rows.cuh"
#include "umma_common.cuh"

namespace xnor {

__device__ int g_status_norm = 0;

namespace {

using namespace umma;

// ---- reductions over a team (a power of two of threads, 32 and more, of a block) ---------------
struct Team {
  int size, rank, first_warp, warps;
  __device__ __forceinline__ explicit Team(int size_) : size(size_) {
    rank = (int)threadIdx.x & (size - 1);
    first_warp = ((int)threadIdx.x - rank) >> 5;
    warps = size >> 5;
  }
  // Every thread of the block calls it; red: one word per warp, not in use by the call before.
  template <class V, class F>
  __device__ __forceinline__ V reduce(V v, V *red, F op) const {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, o));
    if (warps == 1) return v;
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
    __syncthreads();
    v = red[first_warp];
    for (int i = 1; i < warps; ++i) v = op(v, red[first_warp + i]);     // the same order in every thread
    return v;
  }
};

struct Add { __device__ __forceinline__ float operator()(float a, float b) const { return a + b; } };
// The larger of two, a NaN if either is one.
struct Max {
  __device__ __forceinline__ float operator()(float a, float b) const {
    float m;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(a), "f"(b));
    return m;
  }
};

// Eight weights: ones (kind 0), in 32 bits (1) or of the rows' type (2).
template <class T>
__device__ __forceinline__ void load_weights(const void *w, int kind, int c, int in, float (&v)[8]) {
  if (kind == 0) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 1.0f;
  } else if (kind == 1) {
    Chunk<float> a;
    a.load(static_cast<const float *>(w) + c, in == 8, in);
    a.to_float(v);
  } else {
    Chunk<T> a;
    a.load(static_cast<const T *>(w) + c, in == 8, in);
    a.to_float(v);
  }
}
template <class T>
int weight_kind(const void *w, const xnor_norm_desc &d) {
  return w == nullptr ? 0 : d.weight_type == XNOR_F32 ? 1 : 2;
}

// A row's root in two factors: the power of two that is in it, by which values are scaled without a rounding, and the rest,
// 1 to 2.  0, infinite and NaN roots are the first.
__device__ __forceinline__ float power_of(float rstd, float &rest) {
  const bool sound = rstd > 0.0f && rstd <= 3.402823466e38f;
  rest = sound ? __uint_as_float((__float_as_uint(rstd) & 0x007FFFFFu) | 0x3F800000u) : 1.0f;
  return sound ? __uint_as_float(__float_as_uint(rstd) & 0x7F800000u) : rstd;
}

// The values of a group as 8-bit outputs want them.  u = h weight times a power of two, m = max|u|: the row's root is in both, so
// that q is the rounding of top u / m.  16-bit h and weight often put that exactly between two outputs (243 of 2 M e4m3
// quotients of normal bf16 rows), where an approximate quotient would decide by chance.  So quotients are rounded to fp32 correctly, by
// Markstein's correction of an approximate one with its residual (1990), a multiply-add each.  Where top u has more than 24
// bits (all but bf16 rows with bf16 weights or none) its rest is added to the residual.  (2048x4096 bf16 to e4m3 17.6 us, 16.3
// with approximate quotients, 17.9 with the rest added throughout and the scale by an IEEE division.)
struct Quotients {
  float part, divisor, inv, scale;         // top and m, both 2^-9 of it; 1 / divisor
  bool tiny;                               // the scale loses bits, or is near to that: divided by as it is
  __device__ __forceinline__ Quotients(float m, float rest, bool i8) {
    const float over = i8 ? 512.0f / 127.0f : 512.0f / 448.0f;
    const bool sound = m > 0.0f && m <= 3.402823466e38f;                // else zeros (NaN)
    tiny = m > 0.0f && m < 0x1p-90f;
    part = (i8 ? 127.0f : 448.0f) * 0x1p-9f;
    divisor = sound ? m * 0x1p-9f : 0.0f;
    const float largest = divisor * rest, s = __fmul_rn(largest, over);
    scale = sound ? __fmaf_rn(__fmaf_rn(-s, part, largest), over, s) : m;
    if (tiny) scale = __fdiv_rn(m * rest, i8 ? 127.0f : 448.0f);
    float r;
    asm("rcp.approx.f32 %0, %1;" : "=f"(r) : "f"(divisor));
    inv = sound ? r : 0.0f;
  }
  __device__ __forceinline__ void divide(float (&u)[8], float rest, bool wide) const {
    if (tiny) {
#pragma unroll 1
      for (int i = 0; i < 8; ++i) u[i] = scale > 0.0f ? __fdiv_rn(u[i] * rest, scale) : 0.0f;
    } else if (wide) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float n = __fmul_rn(part, u[i]), t = __fmul_rn(n, inv);
        u[i] = __fmaf_rn(__fadd_rn(__fmaf_rn(-t, divisor, n), __fmaf_rn(part, u[i], -n)), inv, t);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float n = __fmul_rn(part, u[i]), t = __fmul_rn(n, inv);
        u[i] = __fmaf_rn(__fmaf_rn(-t, divisor, n), inv, t);
      }
    }
  }
};

__device__ __forceinline__ uint32_t pack_i8(float a, float b, float c, float d) {
  auto q = [](float v) { return (uint32_t)(uint8_t)(int8_t)min(127, max(-127, __float2int_rn(v))); };
  return q(a) | q(b) << 8 | q(c) << 16 | q(d) << 24;
}
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
  const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
  return lo | hi << 16;
}

// Forward: what follows the loads of a row.  Chunk c = rank + v * team of a row belongs to one thread; kV chunks per
// thread cover the row.
template <class T, int kV, bool kQuant>
__device__ __forceinline__ void finish_row(const NormArgs &A, const Team &team, long long row, bool real, const int (&in)[kV], Chunk<T> (&xc)[kV],
                                           const Chunk<T> (&rc)[kV], const float (&wc)[kV][8], int weights, int pieces, float *red,
                                           float *red_max) {
  const int D = A.d.cols;
  // (16-bit values stay packed and are converted twice: half the registers, so twice the rows under way)
  float ss = 0.0f;
#pragma unroll
  for (int v = 0; v < kV; ++v) {
    float h[8];
    xc[v].to_float(h);
    if (A.residual) {
      float r[8];
      rc[v].to_float(r);
#pragma unroll
      for (int i = 0; i < 8; ++i) h[i] += r[i];
      // the norm is of the sum as it is stored, which is what later layers and the backward pass read
      xc[v].from_float(h);
      xc[v].to_float(h);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) ss = fmaf(h[i], h[i], ss);
  }
  if (A.sum) {
    T *sum = static_cast<T *>(A.sum) + (real ? row * A.d.sum_stride : 0);
#pragma unroll
    for (int v = 0; v < kV; ++v) xc[v].store(sum + 8 * (team.rank + v * team.size), pieces, in[v]);
  }
  ss = team.reduce(ss, red, Add());
  const float rstd = __frsqrt_rn(fmaf(ss, A.per_col, A.d.eps));
  if (A.rstd && real && team.rank == 0) A.rstd[row] = rstd;
  float rest = 1.0f;                          // (8 bits: of the row's root)
  const float root = kQuant ? power_of(rstd, rest) : rstd;
  auto normed = [&](int v, float (&y)[8]) {
    xc[v].to_float(y);
    float late[8];
    if constexpr (kV > 2) load_weights<T>(A.weight, weights, 8 * (team.rank + v * team.size), in[v], late);     // (long rows: not held over the sum)
    const float *w = kV > 2 ? late : wc[v];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = y[i] * root * w[i];
  };
  if constexpr (!kQuant) {
    T *y = static_cast<T *>(A.y) + (real ? row * A.d.y_stride : 0);
#pragma unroll
    for (int v = 0; v < kV; ++v) {
      float u[8];
      normed(v, u);
      xc[v].from_float(u);
      xc[v].store(y + 8 * (team.rank + v * team.size), pieces, in[v]);
    }
  } else {
    const bool i8 = A.q_type == XNOR_I8;
    float u[kV <= 2 ? kV : 1][8];             // (many chunks: formed again)
    float m[kV];
#pragma unroll
    for (int v = 0; v < kV; ++v) {
      float (&y)[8] = u[kV <= 2 ? v : 0];
      normed(v, y);
      m[v] = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) m[v] = Max()(m[v], fabsf(y[i]));
    }
    const int lanes = A.group / 8, lg = 31 - __clz(max(A.group, 1));      // threads of a group: 4, 8 or 16, in one warp
    if (A.group == 0) {
      float all = m[0];
#pragma unroll
      for (int v = 1; v < kV; ++v) all = Max()(all, m[v]);
      all = team.reduce(all, red_max, Max());
#pragma unroll
      for (int v = 0; v < kV; ++v) m[v] = all;
    } else {
#pragma unroll
      for (int v = 0; v < kV; ++v)
#pragma unroll
        for (int o = 1; o < 16; o *= 2) {
          const float other = __shfl_xor_sync(0xffffffffu, m[v], o);
          if (o < lanes) m[v] = Max()(m[v], other);
        }
    }
    uint8_t *q = static_cast<uint8_t *>(A.q) + (real ? row * D : 0);
#pragma unroll
    for (int v = 0; v < kV; ++v) {
      const int chunk = team.rank + v * team.size;
      const Quotients of(m[v], rest, i8);
      if (A.group == 0) {
        if (v == 0 && team.rank == 0 && real) A.scales[row] = of.scale;
      } else if (in[v] > 0 && (chunk & (lanes - 1)) == 0) {
        A.scales[row * (D >> lg) + (chunk >> (lg - 3))] = of.scale;
      }
      float (&y)[8] = u[kV <= 2 ? v : 0];
      if constexpr (kV > 2) normed(v, y);
      of.divide(y, rest, !std::is_same<T, __nv_bfloat16>::value || weights == 1);
      const uint32_t lo = i8 ? pack_i8(y[0], y[1], y[2], y[3]) : pack_e4m3(y[0], y[1], y[2], y[3]);
      const uint32_t hi = i8 ? pack_i8(y[4], y[5], y[6], y[7]) : pack_e4m3(y[4], y[5], y[6], y[7]);
      if ((D & 7) == 0) {
        if (in[v] > 0) *reinterpret_cast<uint2 *>(q + 8 * chunk) = make_uint2(lo, hi);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i < in[v]) q[8 * chunk + i] = (uint8_t)((i < 4 ? lo : hi) >> (8 * (i & 3)));
      }
    }
  }
}

template <class T, int kV, int kMost, bool kQuant>
__global__ void __launch_bounds__(kMost, kMost <= 512 && sizeof(T) == 2 ? 2 : 1)
rmsnorm_kernel(const NormArgs A, int team_size, int weights, int pieces) {
  __shared__ float red[kMost / 32];
  __shared__ float red_max[kMost / 32];
  const Team team(team_size);
  const int D = A.d.cols;
  const long long row = (long long)blockIdx.x * ((int)blockDim.x / team_size) + ((int)threadIdx.x / team_size);
  const bool real = row < A.d.rows;
  const T *x = static_cast<const T *>(A.x) + (real ? row * A.d.x_stride : 0);
  const T *res = static_cast<const T *>(A.residual) + (real && A.residual ? row * A.d.residual_stride : 0);
  int in[kV];
#pragma unroll
  for (int v = 0; v < kV; ++v) in[v] = real ? min(8, max(0, D - 8 * (team.rank + v * team.size))) : 0;
  stream_order();
  Chunk<T> xc[kV], rc[kV];
  float wc[kV][8];
#pragma unroll
  for (int v = 0; v < kV; ++v) {
    const int c = 8 * (team.rank + v * team.size);
    xc[v].load(x + c, pieces, in[v]);
    if (A.residual) rc[v].load(res + c, pieces, in[v]);
  }
  if constexpr (kV <= 2) {
#pragma unroll
    for (int v = 0; v < kV; ++v) load_weights<T>(A.weight, weights, 8 * (team.rank + v * team.size), in[v], wc[v]);
  }
  finish_row<T, kV, kQuant>(A, team, row, real, in, xc, rc, wc, weights, pieces, red, red_max);
}

// ---- rows through a ring in shared memory -----------------------------------------------------
constexpr int kMaxStages = 8;
constexpr int kRingControl = 128;          // barriers and the abort flag

// Blocks take rows b, b + grid, ...; thread 0 copies each row's tensors, `tensors` of them, into a stage.
struct RowRing {
  uint32_t bars, data, row_bytes, stage_bytes, stages;
  volatile int *abort_flag;
  int count;                               // rows of this block

  __device__ __forceinline__ RowRing(uint8_t *smem, int rows, uint32_t row_bytes_, int tensors, int stages_)
      : bars(smem_u32(smem)), data(smem_u32(smem) + kRingControl), row_bytes(row_bytes_), stage_bytes(row_bytes_ * (uint32_t)tensors),
        stages((uint32_t)stages_), abort_flag(reinterpret_cast<volatile int *>(smem + 8 * kMaxStages)) {
    count = (int)blockIdx.x < rows ? (rows - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x : 0;
    if (threadIdx.x == 0) {
      for (uint32_t s = 0; s < stages; ++s) mbar_init(bars + 8u * s, 1);
      *abort_flag = 0;
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
  }
  __device__ __forceinline__ long long row(int i) const { return blockIdx.x + (long long)i * gridDim.x; }
  __device__ __forceinline__ uint32_t stage(int i) const { return data + ((uint32_t)i % stages) * stage_bytes; }
  __device__ __forceinline__ void expect(int i) const { mbar_arrive_expect_tx(bars + 8u * ((uint32_t)i % stages), stage_bytes); }
  __device__ __forceinline__ void copy(int i, int tensor, const void *from) const {
    bulk_copy_g2s(stage(i) + (uint32_t)tensor * row_bytes, from, row_bytes, bars + 8u * ((uint32_t)i % stages));
  }
  // Waits for row i of this block; false (for every thread): given up.
  __device__ __forceinline__ bool wait(int i) const {
    const bool ok = mbar_wait(bars + 8u * ((uint32_t)i % stages), ((uint32_t)i / stages) & 1u, abort_flag, &g_status_norm);
    return ok;
  }
  // After giving up at row i: the copies in flight must land before the block's shared memory is released.
  __device__ __forceinline__ void drain(int i) const {
    for (int k = i; k < count && k < i + (int)stages; ++k)
      for (int n = 0; n < (1 << 12) && !mbar_try(bars + 8u * ((uint32_t)k % stages), ((uint32_t)k / stages) & 1u); ++n) {}
  }
};

template <class T>
__device__ __forceinline__ void load_shared(Chunk<T> &c, uint32_t addr) {
#pragma unroll
  for (int i = 0; i < Chunk<T>::kWords / 4; ++i) {
    uint32_t v[4];
    lds128(addr + 16u * i, v);
    c.w[4 * i] = v[0]; c.w[4 * i + 1] = v[1]; c.w[4 * i + 2] = v[2]; c.w[4 * i + 3] = v[3];
  }
}

// Backward.  With u = w dy: dx = rstd (u - h (rstd^2 / D) sum(u h)) (+ dsum), dw = sum over rows of dy h rstd.
// Blocks take rows in turn; the sums of dw stay in registers and leave as one row of partial sums per block,
// which rmsnorm_dweight_kernel adds in the blocks' order.
template <class T>
__device__ __forceinline__ void add_chunk(const Chunk<T> &h, const Chunk<T> &y, const float (&w)[8], float rstd, float &dot, float (&dw)[8]) {
  float hv[8], yv[8];
  h.to_float(hv);
  y.to_float(yv);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float yh = yv[i] * hv[i];
    dot = fmaf(yh, w[i], dot);
    dw[i] = fmaf(yh, rstd, dw[i]);
  }
}
template <class T>
__device__ __forceinline__ Chunk<T> gradient_chunk(const Chunk<T> &h, const Chunk<T> &y, const Chunk<T> &s, bool add, const float (&w)[8],
                                                   float rstd, float k) {
  float hv[8], yv[8], sv[8], o[8];
  h.to_float(hv);
  y.to_float(yv);
#pragma unroll
  for (int i = 0; i < 8; ++i) o[i] = rstd * fmaf(-hv[i], k, yv[i] * w[i]);
  if (add) {
    s.to_float(sv);
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] += sv[i];
  }
  Chunk<T> c;
  c.from_float(o);
  return c;
}

// This block's partial sums of dw.
template <int kV>
__device__ __forceinline__ void store_partial(const NormBackwardArgs &A, const Team &team, const int (&in)[kV], const float (&dw)[kV][8]) {
  if (A.work == nullptr) return;
  float *part = A.work + (size_t)blockIdx.x * A.d.cols;
#pragma unroll
  for (int v = 0; v < kV; ++v) {
    Chunk<float> f;
    f.from_float(dw[v]);
    f.store(part + 8 * (team.rank + v * team.size), (A.d.cols & 7) == 0, in[v]);
  }
}

// Several teams share a block where rows are short; the first adds their sums of dw.
template <class T, int kV, int kMost>
__global__ void __launch_bounds__(kMost)
rmsnorm_backward_kernel(const NormBackwardArgs A, int team_size, int weights, int pieces) {
  __shared__ float red[2][kMost / 32];
  extern __shared__ float sums[];                    // [teams - 1][columns, rounded up to the teams' chunks]
  const Team team(team_size);
  const int D = A.d.cols, teams = (int)blockDim.x / team_size, which = (int)threadIdx.x / team_size;
  int in[kV];
#pragma unroll
  for (int v = 0; v < kV; ++v) in[v] = min(8, max(0, D - 8 * (team.rank + v * team.size)));
  stream_order();
  float wc[kV][8], dw[kV][8] = {};
#pragma unroll
  for (int v = 0; v < kV; ++v) load_weights<T>(A.weight, weights, 8 * (team.rank + v * team.size), in[v], wc[v]);
  int turn = 0;
#pragma unroll 1
  for (long long first = (long long)blockIdx.x * teams; first < A.d.rows; first += (long long)gridDim.x * teams, turn ^= 1) {
    const bool real = first + which < A.d.rows;
    const long long row = real ? first + which : 0;
    const T *h = static_cast<const T *>(A.h) + row * A.d.x_stride;
    const T *dy = static_cast<const T *>(A.dy) + row * A.d.y_stride;
    const T *ds = static_cast<const T *>(A.dsum) + (A.dsum ? row * A.d.residual_stride : 0);
    Chunk<T> hc[kV], yc[kV], sc[kV];
#pragma unroll
    for (int v = 0; v < kV; ++v) {
      const int c = 8 * (team.rank + v * team.size), n = real ? in[v] : 0;
      hc[v].load(h + c, pieces, n);
      yc[v].load(dy + c, pieces, n);
      if (A.dsum) sc[v].load(ds + c, pieces, n);
    }
    const float rstd = load_global_if(A.rstd + row, real);
    float dot = 0.0f;
#pragma unroll
    for (int v = 0; v < kV; ++v) add_chunk<T>(hc[v], yc[v], wc[v], rstd, dot, dw[v]);
    dot = team.reduce(dot, red[turn], Add());
    if (!real) continue;
    const float k = dot * (rstd * rstd * A.per_col);
    T *dx = static_cast<T *>(A.dx) + row * A.d.sum_stride;
#pragma unroll
    for (int v = 0; v < kV; ++v)
      gradient_chunk<T>(hc[v], yc[v], sc[v], A.dsum != nullptr, wc[v], rstd, k).store(dx + 8 * (team.rank + v * team.size), pieces, in[v]);
  }
  if (A.work == nullptr) return;
  if (teams > 1) {
    const int width = 8 * kV * team_size;
    if (which > 0) {
#pragma unroll
      for (int v = 0; v < kV; ++v)
#pragma unroll
        for (int i = 0; i < 8; ++i) sums[(which - 1) * width + (v * 8 + i) * team_size + team.rank] = dw[v][i];
    }
    __syncthreads();
    if (which > 0) return;
    for (int o = 0; o < teams - 1; ++o)
#pragma unroll
      for (int v = 0; v < kV; ++v)
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[v][i] += sums[o * width + (v * 8 + i) * team_size + team.rank];
  }
  store_partial<kV>(A, team, in, dw);
}

// Long rows through the ring.  Both passes over a row read it from there, so that registers hold the sums of dw and
// little else; a stage is free when the next row begins.
template <class T, int kV, int kMost>
__global__ void __launch_bounds__(kMost)
rmsnorm_backward_ring_kernel(const NormBackwardArgs A, int weights, int stages) {
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ float red[2][kMost / 32];
  const Team team((int)blockDim.x);
  const RowRing ring(smem, A.d.rows, (uint32_t)A.d.cols * sizeof(T), A.dsum ? 3 : 2, stages);
  int in[kV];
#pragma unroll
  for (int v = 0; v < kV; ++v) in[v] = min(8, max(0, A.d.cols - 8 * (team.rank + v * team.size)));
  stream_order();
  auto fetch = [&](int i) {
    if (threadIdx.x != 0 || i >= ring.count) return;
    ring.expect(i);
    ring.copy(i, 0, static_cast<const T *>(A.h) + ring.row(i) * A.d.x_stride);
    ring.copy(i, 1, static_cast<const T *>(A.dy) + ring.row(i) * A.d.y_stride);
    if (A.dsum) ring.copy(i, 2, static_cast<const T *>(A.dsum) + ring.row(i) * A.d.residual_stride);
  };
  for (int i = 0; i < stages; ++i) fetch(i);
  float wc[kV][8], dw[kV][8] = {};
#pragma unroll
  for (int v = 0; v < kV; ++v) load_weights<T>(A.weight, weights, 8 * (team.rank + v * team.size), in[v], wc[v]);
  float next = ring.count > 0 ? load_global(A.rstd + ring.row(0)) : 0.0f;
#pragma unroll 1
  for (int i = 0; i < ring.count; ++i) {
    const float rstd = next;
    if (i + 1 < ring.count) next = load_global(A.rstd + ring.row(i + 1));
    if (__syncthreads_or(!ring.wait(i))) {         // (all give up together)
      if (threadIdx.x == 0) ring.drain(i);
      return;
    }
    if (i > 0) fetch(i - 1 + stages);              // (every thread is done with row i - 1)
    const uint32_t at = ring.stage(i) + 8u * (uint32_t)sizeof(T) * (uint32_t)team.rank, step = 8u * (uint32_t)sizeof(T) * (uint32_t)team.size;
    float dot = 0.0f;
#pragma unroll
    for (int v = 0; v < kV; ++v) {
      if (in[v] == 0) continue;
      Chunk<T> h, y;
      load_shared(h, at + (uint32_t)v * step);
      load_shared(y, at + (uint32_t)v * step + ring.row_bytes);
      add_chunk<T>(h, y, wc[v], rstd, dot, dw[v]);
    }
    dot = team.reduce(dot, red[i & 1], Add());
    const float k = dot * (rstd * rstd * A.per_col);
    T *dx = static_cast<T *>(A.dx) + ring.row(i) * A.d.sum_stride;
#pragma unroll
    for (int v = 0; v < kV; ++v) {
      if (in[v] == 0) continue;
      Chunk<T> h, y, s;
      load_shared(h, at + (uint32_t)v * step);
      load_shared(y, at + (uint32_t)v * step + ring.row_bytes);
      if (A.dsum) load_shared(s, at + (uint32_t)v * step + 2u * ring.row_bytes);
      gradient_chunk<T>(h, y, s, A.dsum != nullptr, wc[v], rstd, k).store(dx + 8 * (team.rank + v * team.size), true, in[v]);
    }
  }
  store_partial<kV>(A, team, in, dw);
}

// dweight[c] = sum over the partial rows, in a fixed order: kSumWays threads of a column take every kSumWays-th row each,
// ten loads under way at a time (one at a time, with eight threads to a column, the whole backward pass took 35.3 us for
// 4096x4096 instead of 33.0 at the time, 15.6 instead of 14.4 for 20000x256).
constexpr int kSumCols = 32, kSumWays = 32, kSumLoads = 10;
__global__ void __launch_bounds__(kSumCols * kSumWays)
rmsnorm_dweight_kernel(const float *part, int parts, int D, float *__restrict__ dweight) {
  __shared__ float red[kSumWays][kSumCols + 1];
  stream_order();
  const int lane = threadIdx.x % kSumCols, way = threadIdx.x / kSumCols;
  const int c = blockIdx.x * kSumCols + lane;
  float s = 0.0f;
  for (int p = way; p < parts; p += kSumLoads * kSumWays) {
    float v[kSumLoads];
#pragma unroll
    for (int i = 0; i < kSumLoads; ++i) {
      const bool in = c < D && p + i * kSumWays < parts;
      v[i] = load_global_if(part + (in ? (size_t)(p + i * kSumWays) * D + c : 0), in);
    }
#pragma unroll
    for (int i = 0; i < kSumLoads; ++i) s += v[i];
  }
  red[way][lane] = s;
  __syncthreads();
  // warp w now has column w's sums in its lanes
  s = red[lane][way];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  const int col = blockIdx.x * kSumCols + way;
  if (lane == 0 && col < D) dweight[col] = s;
}

// How a row of `cols` columns is dealt out: chunks per thread, and the most threads that takes (which sets
// the registers each may have).
struct Deal {
  int per_thread, most, team;       // team: a power of two of whole warps
};
enum Pass { kForward, kQuantized, kBackward };
// Chunks per thread, measured: 8192x4096 with residual 59 us with one, 47 with two, 43.7 with four (32 bits, 4096x4096: 51,
// 43.6, 46.4); e4m3 2048x4096 23, 16.6, 19.2 (before its quotients were corrected); backward 4096x4096 50 with one, 34 with two.
Deal deal(int cols, Pass pass, size_t elem) {
  const int chunks = (cols + 7) / 8;
  Deal d;
  d.per_thread = chunks <= 256 ? 1 : chunks <= (pass == kForward && elem == 2 ? 256 : 1024) ? 2 : 4;
  d.most = chunks <= 2048 ? 512 : 1024;
  d.team = 32;
  while (d.team * d.per_thread < chunks) d.team *= 2;
  return d;
}

// The backward pass: threads per block (several teams of short rows), and at most so many blocks per SM.
int backward_threads(const Deal &l) { return std::max(l.team, 256); }
int most_per_sm(const Deal &l) { return std::max(1, (l.per_thread <= 2 ? 1024 : 512) / backward_threads(l)); }

// Its blocks, and the ring's stages.  0 stages: not for these rows (short ones, whose copies would be small, few of them, or
// two of their stages do not fit).  `tensors`: read per row.  More blocks are better down to two stages each (4096x4096
// bf16 31.7 us with four per SM, 34.8 with two; in 32 bits, where four leave one stage, 33.6 and 29.2).
struct BackwardPlan {
  int blocks, stages;
  size_t smem;
};
int blocks_of(int rows, const Deal &l, int per_sm) {
  const int teams = backward_threads(l) / l.team;
  return std::min((int)((rows + (long long)teams - 1) / teams), per_sm * (int)kSms);
}
BackwardPlan plan_backward(int rows, int cols, size_t elem, int tensors, bool pieces) {
  const size_t row = (size_t)cols * elem, stage = row * (size_t)tensors;
  const Deal l = deal(cols, kBackward, elem);
  int per_sm = most_per_sm(l);
  BackwardPlan p = {blocks_of(rows, l, per_sm), 0, 0};
  if (!pieces || row < 4096 || l.team != backward_threads(l) || l.most > 512 || rows < 4 * (int)kSms) return p;
  for (; per_sm >= 1; per_sm /= 2) {
    const int stages = (int)std::min<size_t>(kMaxStages, (200 * 1024 / (size_t)per_sm - 2048) / stage);
    if (stages >= 2) return {blocks_of(rows, l, per_sm), stages, kRingControl + (size_t)stages * stage};
  }
  return p;
}

template <class K>
cudaError_t allow_shared(K *kernel, bool (&flags)[64]) {
  bool &set = attr_done_for_current_device(flags);
  if (set) return cudaSuccess;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 220 * 1024);
  if (e != cudaSuccess) (void)cudaGetLastError();
  set = e == cudaSuccess;
  return e;
}

template <class T, int kV, int kMost, bool kQuant>
cudaError_t run(const NormArgs &a, const Deal &l, int pieces, cudaStream_t st) {
  const int w = weight_kind<T>(a.weight, a.d);
  const int threads = std::max(l.team, 128), per_block = threads / l.team;
  const dim3 grid((unsigned)((a.d.rows + (long long)per_block - 1) / per_block));
  return launch_kernel(rmsnorm_kernel<T, kV, kMost, kQuant>, grid, (unsigned)threads, 0, st, 1, a, l.team, w, pieces);
}

template <class T, int kV, int kMost>
cudaError_t run(const NormArgs &a, const Deal &l, cudaStream_t st) {
  const int pieces = rows_in_pieces(a.x, a.d.x_stride, a.d.cols, sizeof(T)) &&
                     rows_in_pieces(a.residual, a.d.residual_stride, a.d.cols, sizeof(T)) &&
                     rows_in_pieces(a.sum, a.d.sum_stride, a.d.cols, sizeof(T)) &&
                     rows_in_pieces(a.y, a.d.y_stride, a.d.cols, sizeof(T));
  return a.q ? run<T, kV, kMost, true>(a, l, pieces, st) : run<T, kV, kMost, false>(a, l, pieces, st);
}

template <class T, int kV, int kMost>
cudaError_t run(const NormBackwardArgs &a, const Deal &l, cudaStream_t st, int *blocks) {
  const int pieces = rows_in_pieces(a.h, a.d.x_stride, a.d.cols, sizeof(T)) &&
                     rows_in_pieces(a.dy, a.d.y_stride, a.d.cols, sizeof(T)) &&
                     rows_in_pieces(a.dsum, a.d.residual_stride, a.d.cols, sizeof(T)) &&
                     rows_in_pieces(a.dx, a.d.sum_stride, a.d.cols, sizeof(T));
  const int w = weight_kind<T>(a.weight, a.d);
  const BackwardPlan plan = plan_backward(a.d.rows, a.d.cols, sizeof(T), a.dsum ? 3 : 2, pieces);
  *blocks = plan.blocks;
  if constexpr (kMost <= 512) {
    if (plan.stages > 0) {
      static bool flags[64] = {};
      const cudaError_t e = allow_shared(rmsnorm_backward_ring_kernel<T, kV, kMost>, flags);
      if (e != cudaSuccess) return e;
      return launch_kernel(rmsnorm_backward_ring_kernel<T, kV, kMost>, dim3((unsigned)plan.blocks), (unsigned)l.team, plan.smem, st, 1, a, w,
                           plan.stages);
    }
  }
  const int threads = backward_threads(l), teams = threads / l.team;
  return launch_kernel(rmsnorm_backward_kernel<T, kV, kMost>, dim3((unsigned)plan.blocks), (unsigned)threads,
                       (size_t)(teams - 1) * 8 * kV * l.team * sizeof(float), st, 1, a, l.team, w, pieces);
}

Pass pass_of(const NormArgs &a) { return a.q ? kQuantized : kForward; }
Pass pass_of(const NormBackwardArgs &) { return kBackward; }

template <class T, class Args, class... More>
cudaError_t run_type(const Args &a, cudaStream_t st, More... more) {
  const Deal l = deal(a.d.cols, pass_of(a), sizeof(T));
  if (l.most > 512) return run<T, 4, 1024>(a, l, st, more...);
  return l.per_thread == 1 ? run<T, 1, 512>(a, l, st, more...) : l.per_thread == 2 ? run<T, 2, 512>(a, l, st, more...) : run<T, 4, 512>(a, l, st, more...);
}
template <class Args, class... More>
cudaError_t run_any(const Args &a, cudaStream_t st, More... more) {
  if (a.d.type == XNOR_F32) return run_type<float>(a, st, more...);
  return a.d.type == XNOR_BF16 ? run_type<__nv_bfloat16>(a, st, more...) : run_type<__half>(a, st, more...);
}

}  // namespace

// (Does not depend on the device.)
int rmsnorm_parts(int rows, int cols) {
  const Deal l = deal(cols, kBackward, 2);
  return blocks_of(rows, l, most_per_sm(l));
}

cudaError_t read_status_norm(int *status) {
  cudaError_t e = cudaMemcpyFromSymbol(status, g_status_norm, sizeof(int));
  if (e == cudaSuccess && *status != 0) {
    const int zero = 0;
    e = cudaMemcpyToSymbol(g_status_norm, &zero, sizeof(int));
  }
  return e;
}

cudaError_t launch_rmsnorm(const NormArgs &a, cudaStream_t st) { return a.d.rows == 0 ? cudaSuccess : run_any(a, st); }

cudaError_t launch_rmsnorm_backward(const NormBackwardArgs &args, cudaStream_t st) {
  NormBackwardArgs a = args;
  if (a.dweight == nullptr) a.work = nullptr;
  int blocks = 0;                              // and rows of partial sums
  const cudaError_t e = a.d.rows > 0 ? run_any(a, st, &blocks) : cudaSuccess;
  if (e != cudaSuccess || a.dweight == nullptr) return e;
  return launch_kernel(rmsnorm_dweight_kernel, dim3((unsigned)((a.d.cols + kSumCols - 1) / kSumCols)), kSumCols * kSumWays, 0, st, 1,
                       (const float *)a.work, blocks, a.d.cols, a.dweight);
}

}  // namespace xnor
