// Root-mean-square norm of rows with the residual's addition, in the rows' type or in 8 bits with scales, and
// its backward pass.  Every row is read once: its values stay in the registers of a team of threads.
#include <algorithm>

#include "rows.cuh"

namespace xnor {

namespace {

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
// Of bit patterns of magnitudes: a NaN is above every number and stays.
struct Max { __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const { return max(a, b); } };

__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// The weights of a chunk: none (1), 32 bits, or the rows' type.
template <class T>
struct Weights {
  Chunk<float> wide;
  Chunk<T> same;
  __device__ __forceinline__ void load(const void *w, int kind, int c, int in) {
    if (kind == 1) wide.load(static_cast<const float *>(w) + c, in == 8, in);
    else if (kind == 2) same.load(static_cast<const T *>(w) + c, in == 8, in);
  }
  __device__ __forceinline__ void to_float(int kind, float v[8]) const {
    if (kind == 1) wide.to_float(v);
    else if (kind == 2) same.to_float(v);
    else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = 1.0f;
    }
  }
};
template <class T>
int weight_kind(const void *w, const xnor_norm_desc &d) {
  return w == nullptr ? 0 : d.weight_type == XNOR_F32 ? 1 : 2;
}

// y / s to nearest even.  The reciprocal is within an ulp of the quotient's factor except where it overflows.
struct Divide {
  float s, inv;
  bool tiny;
  __device__ __forceinline__ explicit Divide(float s_) : s(s_) {
    tiny = s > 0.0f && s < 1e-37f;
    inv = s > 0.0f ? 1.0f / s : 0.0f;
  }
  __device__ __forceinline__ float operator()(float y) const { return tiny ? y / s : y * inv; }
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

// Forward.  Chunk c = rank + v * team of a row belongs to one thread; kV chunks per thread cover the row.
template <class T, int kV, int kMost, bool kQuant>
__global__ void __launch_bounds__(kMost)
rmsnorm_kernel(const NormArgs A, int team_size, int weights, int pieces) {
  __shared__ float red[kMost / 32];
  __shared__ uint32_t red_max[kMost / 32];
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
  Weights<T> wc[kV];
#pragma unroll
  for (int v = 0; v < kV; ++v) {
    const int c = 8 * (team.rank + v * team.size);
    xc[v].load(x + c, pieces, in[v]);
    if (A.residual) rc[v].load(res + c, pieces, in[v]);
  }
#pragma unroll
  for (int v = 0; v < kV; ++v) wc[v].load(A.weight, weights, 8 * (team.rank + v * team.size), in[v]);
  float h[kV][8], ss = 0.0f;
#pragma unroll
  for (int v = 0; v < kV; ++v) {
    xc[v].to_float(h[v]);
    if (A.residual) {
      float r[8];
      rc[v].to_float(r);
#pragma unroll
      for (int i = 0; i < 8; ++i) h[v][i] += r[i];
      // the norm is of the sum as it is stored, which is what later layers and the backward pass read
      xc[v].from_float(h[v]);
      xc[v].to_float(h[v]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) ss = fmaf(h[v][i], h[v][i], ss);
  }
  if (A.sum) {
    T *sum = static_cast<T *>(A.sum) + (real ? row * A.d.sum_stride : 0);
#pragma unroll
    for (int v = 0; v < kV; ++v) xc[v].store(sum + 8 * (team.rank + v * team.size), pieces, in[v]);
  }
  ss = team.reduce(ss, red, Add());
  const float rstd = 1.0f / sqrtf(ss / (float)D + A.d.eps);
  if (A.rstd && real && team.rank == 0) A.rstd[row] = rstd;
#pragma unroll
  for (int v = 0; v < kV; ++v) {
    float w[8];
    wc[v].to_float(weights, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) h[v][i] = h[v][i] * rstd * w[i];
  }
  if constexpr (!kQuant) {
    T *y = static_cast<T *>(A.y) + (real ? row * A.d.y_stride : 0);
#pragma unroll
    for (int v = 0; v < kV; ++v) {
      xc[v].from_float(h[v]);
      xc[v].store(y + 8 * (team.rank + v * team.size), pieces, in[v]);
    }
  } else {
    const float top = A.q_type == XNOR_I8 ? 127.0f : 448.0f;
    uint32_t m[kV];
#pragma unroll
    for (int v = 0; v < kV; ++v) {
      m[v] = 0u;
#pragma unroll
      for (int i = 0; i < 8; ++i) m[v] = max(m[v], magnitude(h[v][i]));
    }
    const int lanes = A.group / 8;            // threads of a group: 4, 8 or 16, in one warp
    if (A.group == 0) {
      uint32_t all = m[0];
#pragma unroll
      for (int v = 1; v < kV; ++v) all = max(all, m[v]);
      all = team.reduce(all, red_max, Max());
#pragma unroll
      for (int v = 0; v < kV; ++v) m[v] = all;
    } else {
#pragma unroll
      for (int v = 0; v < kV; ++v)
        for (int o = 1; o < lanes; o *= 2) m[v] = max(m[v], __shfl_xor_sync(0xffffffffu, m[v], o));
    }
    uint8_t *q = static_cast<uint8_t *>(A.q) + (real ? row * D : 0);
#pragma unroll
    for (int v = 0; v < kV; ++v) {
      const int chunk = team.rank + v * team.size;
      const float s = __fdiv_rn(__uint_as_float(m[v]), top);
      if (A.group == 0) {
        if (v == 0 && team.rank == 0 && real) A.scales[row] = s;
      } else if (in[v] > 0 && (chunk & (lanes - 1)) == 0) {
        A.scales[row * (D / A.group) + chunk / lanes] = s;
      }
      const Divide by(s);
      float u[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) u[i] = by(h[v][i]);
      const bool i8 = A.q_type == XNOR_I8;
      const uint32_t lo = i8 ? pack_i8(u[0], u[1], u[2], u[3]) : pack_e4m3(u[0], u[1], u[2], u[3]);
      const uint32_t hi = i8 ? pack_i8(u[4], u[5], u[6], u[7]) : pack_e4m3(u[4], u[5], u[6], u[7]);
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

// Backward.  With u = w dy: dx = rstd (u - h (rstd^2 / D) sum(u h)) (+ dsum), dw = sum over rows of dy h rstd.
// A block takes rows b, b + grid, ...; the sums of dw stay in registers and leave as one row of partial sums
// per block, which rmsnorm_dweight_kernel adds in the blocks' order.
template <class T, int kV, int kMost>
__global__ void __launch_bounds__(kMost)
rmsnorm_backward_kernel(const NormBackwardArgs A, int weights, int pieces) {
  __shared__ float red[2][kMost / 32];
  const Team team((int)blockDim.x);
  const int D = A.d.cols;
  int in[kV];
#pragma unroll
  for (int v = 0; v < kV; ++v) in[v] = min(8, max(0, D - 8 * (team.rank + v * team.size)));
  stream_order();
  Weights<T> wc[kV];
  float dw[kV][8];
#pragma unroll
  for (int v = 0; v < kV; ++v) {
    wc[v].load(A.weight, weights, 8 * (team.rank + v * team.size), in[v]);
#pragma unroll
    for (int i = 0; i < 8; ++i) dw[v][i] = 0.0f;
  }
  int turn = 0;
  for (long long row = blockIdx.x; row < A.d.rows; row += gridDim.x, turn ^= 1) {
    const T *h = static_cast<const T *>(A.h) + row * A.d.x_stride;
    const T *dy = static_cast<const T *>(A.dy) + row * A.d.y_stride;
    const T *ds = static_cast<const T *>(A.dsum) + (A.dsum ? row * A.d.residual_stride : 0);
    T *dx = static_cast<T *>(A.dx) + row * A.d.sum_stride;
    Chunk<T> hc[kV], yc[kV], sc[kV];
#pragma unroll
    for (int v = 0; v < kV; ++v) {
      const int c = 8 * (team.rank + v * team.size);
      hc[v].load(h + c, pieces, in[v]);
      yc[v].load(dy + c, pieces, in[v]);
      if (A.dsum) sc[v].load(ds + c, pieces, in[v]);
    }
    const float rstd = load_global(A.rstd + row);
    float dot = 0.0f;
#pragma unroll
    for (int v = 0; v < kV; ++v) {
      float hv[8], yv[8], w[8];
      hc[v].to_float(hv);
      yc[v].to_float(yv);
      wc[v].to_float(weights, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        dot = fmaf(yv[i] * w[i], hv[i], dot);
        dw[v][i] = fmaf(yv[i], hv[i] * rstd, dw[v][i]);
      }
    }
    dot = team.reduce(dot, red[turn], Add());
    const float k = dot * (rstd * rstd / (float)D);
#pragma unroll
    for (int v = 0; v < kV; ++v) {
      float hv[8], yv[8], w[8], sv[8], o[8];
      hc[v].to_float(hv);
      yc[v].to_float(yv);
      wc[v].to_float(weights, w);
      if (A.dsum) sc[v].to_float(sv);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        o[i] = rstd * fmaf(-hv[i], k, yv[i] * w[i]);
        if (A.dsum) o[i] += sv[i];
      }
      Chunk<T> oc;
      oc.from_float(o);
      oc.store(dx + 8 * (team.rank + v * team.size), pieces, in[v]);
    }
  }
  if (A.work == nullptr) return;
  float *part = A.work + (size_t)blockIdx.x * D;
#pragma unroll
  for (int v = 0; v < kV; ++v) {
    const int c = 8 * (team.rank + v * team.size);
    Chunk<float> f;
    f.from_float(dw[v]);
    f.store(part + c, (D & 7) == 0, in[v]);
  }
}

// dweight[c] = sum over the partial rows, in their order: eight threads of a column take every eighth row each.
constexpr int kSumCols = 32, kSumWays = 8;
__global__ void __launch_bounds__(kSumCols * kSumWays)
rmsnorm_dweight_kernel(const float *part, int parts, int D, float *__restrict__ dweight) {
  __shared__ float red[kSumWays][kSumCols];
  stream_order();
  const int lane = threadIdx.x % kSumCols, way = threadIdx.x / kSumCols;
  const int c = blockIdx.x * kSumCols + lane;
  float s = 0.0f;
  if (c < D)
    for (int p = way; p < parts; p += kSumWays) s += load_global(part + (size_t)p * D + c);
  red[way][lane] = s;
  __syncthreads();
  if (way == 0 && c < D) {
#pragma unroll
    for (int i = 1; i < kSumWays; ++i) s += red[i][lane];
    dweight[c] = s;
  }
}

// How a row of `cols` columns is dealt out: chunks per thread, and the most threads that takes (which sets
// the registers each may have).
struct Deal {
  int per_thread, most, team;       // team: a power of two of whole warps
};
Deal deal(int cols) {
  const int chunks = (cols + 7) / 8;
  Deal d;
  d.per_thread = chunks <= 512 ? 1 : chunks <= 1024 ? 2 : 4;
  d.most = chunks <= 2048 ? 512 : 1024;
  d.team = 32;
  while (d.team * d.per_thread < chunks) d.team *= 2;
  return d;
}

template <class T, int kV, int kMost>
cudaError_t run(const NormArgs &a, const Deal &l, cudaStream_t st) {
  const int threads = std::max(l.team, 128), per_block = threads / l.team;
  const dim3 grid((unsigned)((a.d.rows + (long long)per_block - 1) / per_block));
  const int pieces = rows_in_pieces(a.x, a.d.x_stride, a.d.cols, sizeof(T)) &&
                     rows_in_pieces(a.residual, a.d.residual_stride, a.d.cols, sizeof(T)) &&
                     rows_in_pieces(a.sum, a.d.sum_stride, a.d.cols, sizeof(T)) &&
                     rows_in_pieces(a.y, a.d.y_stride, a.d.cols, sizeof(T));
  const int w = weight_kind<T>(a.weight, a.d);
  if (a.q) return launch_kernel(rmsnorm_kernel<T, kV, kMost, true>, grid, (unsigned)threads, 0, st, 1, a, l.team, w, pieces);
  return launch_kernel(rmsnorm_kernel<T, kV, kMost, false>, grid, (unsigned)threads, 0, st, 1, a, l.team, w, pieces);
}

template <class T, int kV, int kMost>
cudaError_t run(const NormBackwardArgs &a, const Deal &l, cudaStream_t st) {
  const int pieces = rows_in_pieces(a.h, a.d.x_stride, a.d.cols, sizeof(T)) &&
                     rows_in_pieces(a.dy, a.d.y_stride, a.d.cols, sizeof(T)) &&
                     rows_in_pieces(a.dsum, a.d.residual_stride, a.d.cols, sizeof(T)) &&
                     rows_in_pieces(a.dx, a.d.sum_stride, a.d.cols, sizeof(T));
  return launch_kernel(rmsnorm_backward_kernel<T, kV, kMost>, dim3((unsigned)rmsnorm_parts(a.d.rows, a.d.cols)), (unsigned)l.team, 0,
                       st, 1, a, weight_kind<T>(a.weight, a.d), pieces);
}

template <class T, class Args>
cudaError_t run_type(const Args &a, cudaStream_t st) {
  const Deal l = deal(a.d.cols);
  if (l.most > 512) return run<T, 4, 1024>(a, l, st);
  return l.per_thread == 1 ? run<T, 1, 512>(a, l, st) : l.per_thread == 2 ? run<T, 2, 512>(a, l, st) : run<T, 4, 512>(a, l, st);
}
template <class Args>
cudaError_t run_any(const Args &a, cudaStream_t st) {
  if (a.d.type == XNOR_F32) return run_type<float>(a, st);
  return a.d.type == XNOR_BF16 ? run_type<__nv_bfloat16>(a, st) : run_type<__half>(a, st);
}

}  // namespace

int rmsnorm_parts(int rows, int cols) {
  const int per_sm = std::max(1, std::min(8, 1024 / deal(cols).team));
  return std::min(rows, per_sm * (int)kSms);
}

cudaError_t launch_rmsnorm(const NormArgs &a, cudaStream_t st) { return a.d.rows == 0 ? cudaSuccess : run_any(a, st); }

cudaError_t launch_rmsnorm_backward(const NormBackwardArgs &args, cudaStream_t st) {
  NormBackwardArgs a = args;
  if (a.dweight == nullptr) a.work = nullptr;
  cudaError_t e = a.d.rows > 0 ? run_any(a, st) : cudaSuccess;
  if (e != cudaSuccess || a.dweight == nullptr) return e;
  return launch_kernel(rmsnorm_dweight_kernel, dim3((unsigned)((a.d.cols + kSumCols - 1) / kSumCols)), kSumCols * kSumWays, 0, st, 1,
                       (const float *)a.work, rmsnorm_parts(a.d.rows, a.d.cols), a.d.cols, a.dweight);
}

}  // namespace xnor
