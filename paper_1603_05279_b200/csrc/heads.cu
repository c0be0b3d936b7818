// Root-mean-square norm of the queries' and keys' heads with the rotation by position, and its backward pass.
//
// Every value is read once and written once, so HBM would bound them.  8192 tokens of 32 and 8 heads of 128 in bfloat16 take 40.8 us
// (172 MB, 0.65 of a copy's rate), the backward pass of 4096 37 (128 MB, 0.54): 220 instructions for 512 values of a warp, at 1.8 per
// clock with 22 % of the warps a SM can have.  Two blocks per SM, with registers for the values under way: three (80 registers)
// took 45.7, four 55.6; two, three or four units under way 41.1, 40.7 and 40.4.  Loads have no condition: under one they were waited for at once.
// Tokens cut into parts, for blocks that end together, took longer (two 45.9, seven 67.2): the start of a token, its place and
// angles one after the other, costs what a few heads do.
#include <algorithm>

#include "heads.cuh"

namespace xnor {

__device__ int g_status_heads = 0;

namespace {

constexpr int kWarps = 8;

// The position's row of the table, or null: outside it, which is recorded and the token left as it is.
__device__ __forceinline__ bool angles_of(const HeadsArgs &A, int t, const float *&row) {
  row = nullptr;
  if (A.d.rot == 0) return true;
  const int p = (int)load_global(reinterpret_cast<const uint32_t *>(A.pos) + t);
  if (p < 0 || p >= A.d.positions) {
    atomicMax(&g_status_heads, (int)XNOR_ERR_BOUNDS);
    return false;
  }
  row = A.table + (size_t)p * A.d.rot;
  return true;
}

// ---- whole chunks ------------------------------------------------------------------------------------------------
// A warp has a token's angles and goes through its heads, kHeads at a time (a unit: of queries or of keys), every
// parts-th unit, the next one's values under way.  Few tokens are shared by many warps.
template <class T, int kDim>
struct HeadUnits {
  int q_units, units;
  __device__ __forceinline__ explicit HeadUnits(const xnor_heads_desc &d)
      : q_units((d.q_heads + HeadLane<kDim>::kHeads - 1) / HeadLane<kDim>::kHeads), units(q_units + (d.k_heads + HeadLane<kDim>::kHeads - 1) / HeadLane<kDim>::kHeads) {}
};

template <class T, int kDim, bool kPairs>
__global__ void __launch_bounds__(32 * kWarps, 2)
heads_kernel(const HeadsArgs A, int parts) {
  using Lane = HeadLane<kDim>;
  const Lane lane(threadIdx.x & 31, A.d.rot, kPairs);
  const HeadUnits<T, kDim> U(A.d);
  const bool f32 = A.d.weight_type == XNOR_F32;
  const int items = A.d.rows * parts, step = parts * Lane::kHeads;
  stream_order();
  for (int item = (int)blockIdx.x * kWarps + (int)threadIdx.x / 32; item < items; item += (int)gridDim.x * kWarps) {
    const int t = item / parts, first = item - t * parts;
    const int first_k = first >= U.q_units ? first - U.q_units : (parts - (U.q_units - first) % parts) % parts;      // its first unit of keys
    const T *q = static_cast<const T *>(A.q) + t * A.d.q_stride, *k = static_cast<const T *>(A.k) + t * A.d.k_stride;
    if (A.d.q_heads == 0) q = k;                             // (read, but not used)
    if (A.d.k_heads == 0) k = q;
    auto fetch = [&](const T *from, int heads, int h, TwoChunks<T> &x) { x.load(from + (h < heads ? h : 0) * kDim, lane); };
    // the first units are under way while the token's angles are looked up
    TwoChunks<T> x_q, x_k;
    fetch(q, A.d.q_heads, first * Lane::kHeads + lane.sub, x_q);
    fetch(k, A.d.k_heads, first_k * Lane::kHeads + lane.sub, x_k);
    const float *row;
    if (!angles_of(A, t, row)) continue;
    Angles angles;
    if (lane.turns) angles.load(row, A.d.rot, lane.which);
    // units of one kind, `first`, first + parts, ..: their weights stay in registers, the next one's values are under way
    auto run = [&](int first, int units, int heads, const T *from, T *to, const void *weight, TwoChunks<T> &x) {
      if (first >= units) return;
      float w[16];
      if (A.d.norm) {
        load_head_weights<T>(weight, f32, lane.a, w);
        load_head_weights<T>(weight, f32, lane.b, w + 8);
      }
      auto finish = [&](int h, TwoChunks<T> &x) {
        float v[16];
        x.to_float(v);
        if (A.d.norm) {
          float s = 0.0f;
#pragma unroll
          for (int i = 0; i < 16; ++i) s = fmaf(v[i], v[i], s);
          const float r = __frsqrt_rn(lane.sum(s) * (1.0f / kDim) + A.d.eps);
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i] *= r * w[i];
        }
        if (lane.turns) turn<kPairs, 1>(v, angles);
        x.from_float(v);
        if (h < heads) x.store(to + h * kDim, lane);
      };
      TwoChunks<T> y;
      int h = first * Lane::kHeads + lane.sub;
#pragma unroll 1
      for (int u = first; u < units; u += 2 * parts, h += 2 * step) {
        fetch(from, heads, h + step, y);
        finish(h, x);
        if (u + parts >= units) break;
        fetch(from, heads, h + 2 * step, x);
        finish(h + step, y);
      }
    };
    run(first, U.q_units, A.d.q_heads, q, static_cast<T *>(A.q_out) + t * A.d.q_out_stride, A.q_weight, x_q);
    run(first_k, U.units - U.q_units, A.d.k_heads, k, static_cast<T *>(A.k_out) + t * A.d.k_out_stride, A.k_weight, x_k);
  }
}

// Blocks below q_blocks have queries, the others keys; a warp has every so-many-th item, of `each` units of a token.
struct BackwardItems {
  long long items;
  int heads, each, per_token;
  bool keys;
  int block, blocks;
  __device__ __forceinline__ BackwardItems(const HeadsArgs &A, int q_blocks, int at_once, int each_) : each(each_) {
    keys = (int)blockIdx.x >= q_blocks;
    block = keys ? (int)blockIdx.x - q_blocks : (int)blockIdx.x;
    blocks = keys ? (int)gridDim.x - q_blocks : q_blocks;
    heads = keys ? A.d.k_heads : A.d.q_heads;
    per_token = (heads + at_once * each - 1) / (at_once * each);
    items = (long long)A.d.rows * per_token;
  }
};
constexpr int kBackwardEach = 4;         // (8: 63.8 us against 41.1 for 4096 tokens, 32 and 8 heads of 128)

// g = the gradient turned back, u = weight g:  dx = rstd (u - x rstd^2 mean(u x)),  dweight += g x rstd.  A thread adds up its
// sixteen columns' dweight over all its heads, the block adds its threads' in a fixed order, and leaves a row of `work`.
template <class T, int kDim, bool kPairs>
__global__ void __launch_bounds__(32 * kWarps, 2)
heads_backward_kernel(const HeadsArgs A, int q_blocks) {
  using Lane = HeadLane<kDim>;
  __shared__ float sums[kWarps * Lane::kHeads][kDim + 4];
  const Lane lane(threadIdx.x & 31, A.d.rot, kPairs);
  const BackwardItems I(A, q_blocks, Lane::kHeads, kBackwardEach);
  const bool keys = I.keys;
  const T *x_all = static_cast<const T *>(keys ? A.k : A.q), *dy_all = static_cast<const T *>(keys ? A.dk_out : A.dq_out);
  T *dx_all = static_cast<T *>(keys ? A.k_out : A.q_out);
  const long long x_stride = keys ? A.d.k_stride : A.d.q_stride, dy_stride = keys ? A.d.dk_stride : A.d.dq_stride;
  const long long dx_stride = keys ? A.d.k_out_stride : A.d.q_out_stride;
  stream_order();
  float w[16], dw[16] = {};
  const void *weight = keys ? A.k_weight : A.q_weight;
  load_head_weights<T>(weight, A.d.weight_type == XNOR_F32, lane.a, w);
  load_head_weights<T>(weight, A.d.weight_type == XNOR_F32, lane.b, w + 8);
  for (long long item = (long long)I.block * kWarps + threadIdx.x / 32; item < I.items; item += (long long)I.blocks * kWarps) {
    const int t = (int)divide(item, I.per_token);
    const float *row;
    if (!angles_of(A, t, row)) continue;
    const T *x_row = x_all + t * x_stride, *dy_row = dy_all + t * dy_stride;
    T *dx_row = dx_all + t * dx_stride;
    const int h0 = (int)(item - (long long)t * I.per_token) * kBackwardEach * Lane::kHeads + lane.sub;
    auto fetch = [&](int i, TwoChunks<T> &x, TwoChunks<T> &dy) {
      const int h = h0 + i * Lane::kHeads;
      x.load(x_row + (h < I.heads ? h : 0) * kDim, lane);
      dy.load(dy_row + (h < I.heads ? h : 0) * kDim, lane);
    };
    Angles angles;
    auto finish = [&](int i, const TwoChunks<T> &xc, TwoChunks<T> &yc) {
      const int h = h0 + i * Lane::kHeads;
      float x[16], g[16];
      yc.to_float(g);
      if (lane.turns) turn<kPairs, -1>(g, angles);
      if (A.d.norm) {
        xc.to_float(x);
        float s = 0.0f, dot = 0.0f;
#pragma unroll
        for (int j = 0; j < 16; ++j) s = fmaf(x[j], x[j], s);
#pragma unroll
        for (int j = 0; j < 16; ++j) dot = fmaf(g[j] * w[j], x[j], dot);
        const float r = __frsqrt_rn(lane.sum(s) * (1.0f / kDim) + A.d.eps);
        const float k = lane.sum(dot) * (r * r * (1.0f / kDim));
        // (what a thread without a head has read is another's, and may be its gradient already, even infinite)
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          if (h < I.heads) dw[j] = fmaf(g[j] * r, x[j], dw[j]);
          g[j] = r * fmaf(-x[j], k, g[j] * w[j]);
        }
      }
      yc.from_float(g);
      if (h < I.heads) yc.store(dx_row + h * kDim, lane);
    };
    TwoChunks<T> x0, y0, x1, y1;
    fetch(0, x0, y0);
    if (lane.turns) angles.load(row, A.d.rot, lane.which);
#pragma unroll
    for (int i = 0; i < kBackwardEach; i += 2) {
      fetch(i + 1, x1, y1);
      finish(i, x0, y0);
      if (i + 2 < kBackwardEach) fetch(i + 2, x0, y0);
      if (h0 - lane.sub + (i + 1) * Lane::kHeads >= I.heads) break;
      finish(i + 1, x1, y1);
    }
  }
  if (A.work == nullptr) return;
  float *mine = sums[(threadIdx.x / 32) * Lane::kHeads + lane.sub];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    mine[lane.a + i] = dw[i];
    mine[lane.b + i] = dw[8 + i];
  }
  __syncthreads();
  for (int c = threadIdx.x; c < kDim; c += 32 * kWarps) {
    float s = 0.0f;
#pragma unroll 8
    for (int i = 0; i < kWarps * Lane::kHeads; ++i) s += sums[i][c];
    A.work[(size_t)blockIdx.x * kDim + c] = s;
  }
}

// ---- any head ----------------------------------------------------------------------------------------------------
// A warp has a head, a thread every 32nd of its pairs, value by value.  Pairs behind the rotated ones are of any two values.
constexpr int kMostPairs = kHeadsMaxDim / 64;
template <class T>
struct LoosePairs {
  __device__ __forceinline__ static void columns(const xnor_heads_desc &d, int p, int &a, int &b) {
    const int half = d.rot / 2;
    if (p >= half) { a = 2 * p; b = a + 1; }
    else if (d.pairs) { a = 2 * p; b = a + 1; }
    else { a = p; b = half + p; }
  }
  __device__ __forceinline__ static float read(const T *p) {
    if constexpr (sizeof(T) == 4) {
      return load_global(reinterpret_cast<const float *>(p));
    } else {
      return pair_to_float(load_global(reinterpret_cast<const uint16_t *>(p)), T()).x;
    }
  }
  __device__ __forceinline__ static void write(T *p, float v) {
    if constexpr (sizeof(T) == 4) *p = v;
    else *reinterpret_cast<uint16_t *>(p) = (uint16_t)float_to_pair(v, 0.0f, T());
  }
  __device__ __forceinline__ static float weight(const HeadsArgs &A, const void *w, int c) {
    if (w == nullptr) return 1.0f;
    return A.d.weight_type == XNOR_F32 ? load_global(static_cast<const float *>(w) + c) : read(static_cast<const T *>(w) + c);
  }
};
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

template <class T>
__global__ void __launch_bounds__(32 * kWarps)
heads_loose_kernel(const HeadsArgs A) {
  using P = LoosePairs<T>;
  const int lane = threadIdx.x & 31, heads = A.d.q_heads + A.d.k_heads, half = A.d.rot / 2, n = A.d.dim / 2;
  const long long items = (long long)A.d.rows * heads;
  stream_order();
  for (long long item = (long long)blockIdx.x * kWarps + threadIdx.x / 32; item < items; item += (long long)gridDim.x * kWarps) {
    const int t = (int)(item / heads), any = (int)(item % heads);
    const bool keys = any >= A.d.q_heads;
    const int h = keys ? any - A.d.q_heads : any;
    const float *row;
    if (!angles_of(A, t, row)) continue;
    const T *x = static_cast<const T *>(keys ? A.k : A.q) + t * (keys ? A.d.k_stride : A.d.q_stride) + h * A.d.dim;
    T *y = static_cast<T *>(keys ? A.k_out : A.q_out) + t * (keys ? A.d.k_out_stride : A.d.q_out_stride) + h * A.d.dim;
    float u[kMostPairs], v[kMostPairs], s = 0.0f;
#pragma unroll
    for (int i = 0; i < kMostPairs; ++i) {
      const int p = lane + 32 * i;
      u[i] = v[i] = 0.0f;
      if (p >= n) continue;
      int a, b;
      P::columns(A.d, p, a, b);
      u[i] = P::read(x + a);
      v[i] = P::read(x + b);
      s = fmaf(u[i], u[i], fmaf(v[i], v[i], s));
    }
    const float r = A.d.norm ? 1.0f / sqrtf(warp_sum(s) / (float)A.d.dim + A.d.eps) : 1.0f;
#pragma unroll
    for (int i = 0; i < kMostPairs; ++i) {
      const int p = lane + 32 * i;
      if (p >= n) continue;
      int a, b;
      P::columns(A.d, p, a, b);
      if (A.d.norm) {
        const void *w = keys ? A.k_weight : A.q_weight;
        u[i] *= r * P::weight(A, w, a);
        v[i] *= r * P::weight(A, w, b);
      }
      if (p < half) {
        const float c = load_global(row + p), sn = load_global(row + half + p), w = u[i] * c - v[i] * sn;
        v[i] = v[i] * c + u[i] * sn;
        u[i] = w;
      }
      P::write(y + a, u[i]);
      P::write(y + b, v[i]);
    }
  }
}

template <class T>
__global__ void __launch_bounds__(32 * kWarps)
heads_backward_loose_kernel(const HeadsArgs A, int q_blocks) {
  using P = LoosePairs<T>;
  __shared__ float sums[kWarps][kHeadsMaxDim];
  const BackwardItems I(A, q_blocks, 1, 1);
  const bool keys = I.keys;
  const int lane = threadIdx.x & 31, half = A.d.rot / 2, n = A.d.dim / 2;
  const void *weight = keys ? A.k_weight : A.q_weight;
  stream_order();
  float dwu[kMostPairs] = {}, dwv[kMostPairs] = {};
  for (long long item = (long long)I.block * kWarps + threadIdx.x / 32; item < I.items; item += (long long)I.blocks * kWarps) {
    const int t = (int)(item / I.heads), h = (int)(item % I.heads);
    const float *row;
    if (!angles_of(A, t, row)) continue;
    const T *x = static_cast<const T *>(keys ? A.k : A.q) + t * (keys ? A.d.k_stride : A.d.q_stride) + h * A.d.dim;
    const T *dy = static_cast<const T *>(keys ? A.dk_out : A.dq_out) + t * (keys ? A.d.dk_stride : A.d.dq_stride) + h * A.d.dim;
    T *dx = static_cast<T *>(keys ? A.k_out : A.q_out) + t * (keys ? A.d.k_out_stride : A.d.q_out_stride) + h * A.d.dim;
    float gu[kMostPairs], gv[kMostPairs], xu[kMostPairs], xv[kMostPairs], s = 0.0f, dot = 0.0f;
#pragma unroll
    for (int i = 0; i < kMostPairs; ++i) {
      const int p = lane + 32 * i;
      gu[i] = gv[i] = xu[i] = xv[i] = 0.0f;
      if (p >= n) continue;
      int a, b;
      P::columns(A.d, p, a, b);
      gu[i] = P::read(dy + a);
      gv[i] = P::read(dy + b);
      if (p < half) {
        const float c = load_global(row + p), sn = load_global(row + half + p), w = gu[i] * c + gv[i] * sn;
        gv[i] = gv[i] * c - gu[i] * sn;
        gu[i] = w;
      }
      if (!A.d.norm) continue;
      xu[i] = P::read(x + a);
      xv[i] = P::read(x + b);
      s = fmaf(xu[i], xu[i], fmaf(xv[i], xv[i], s));
      dot = fmaf(gu[i] * P::weight(A, weight, a), xu[i], fmaf(gv[i] * P::weight(A, weight, b), xv[i], dot));
    }
    const float mean = 1.0f / (float)A.d.dim;
    const float r = A.d.norm ? 1.0f / sqrtf(warp_sum(s) * mean + A.d.eps) : 1.0f, k = A.d.norm ? warp_sum(dot) * (r * r * mean) : 0.0f;
#pragma unroll
    for (int i = 0; i < kMostPairs; ++i) {
      const int p = lane + 32 * i;
      if (p >= n) continue;
      int a, b;
      P::columns(A.d, p, a, b);
      if (A.d.norm) {
        dwu[i] = fmaf(gu[i] * r, xu[i], dwu[i]);
        dwv[i] = fmaf(gv[i] * r, xv[i], dwv[i]);
        gu[i] = r * fmaf(-xu[i], k, gu[i] * P::weight(A, weight, a));
        gv[i] = r * fmaf(-xv[i], k, gv[i] * P::weight(A, weight, b));
      }
      P::write(dx + a, gu[i]);
      P::write(dx + b, gv[i]);
    }
  }
  if (A.work == nullptr) return;
#pragma unroll
  for (int i = 0; i < kMostPairs; ++i) {
    const int p = lane + 32 * i;
    if (p >= n) continue;
    int a, b;
    P::columns(A.d, p, a, b);
    sums[threadIdx.x / 32][a] = dwu[i];
    sums[threadIdx.x / 32][b] = dwv[i];
  }
  __syncthreads();
  for (int c = threadIdx.x; c < A.d.dim; c += 32 * kWarps) {
    float s = 0.0f;
    for (int i = 0; i < kWarps; ++i) s += sums[i][c];
    A.work[(size_t)blockIdx.x * A.d.dim + c] = s;
  }
}

// dweight[c] = sum over the blocks' rows, in a fixed order: a block has 32 columns of one weight, a warp every 32nd row.
__global__ void __launch_bounds__(1024)
heads_dweight_kernel(const float *work, int q_blocks, int blocks, int dim, float *dq_weight, float *dk_weight) {
  __shared__ float red[32][33];
  stream_order();
  const bool keys = blockIdx.y == 1;
  float *out = keys ? dk_weight : dq_weight;
  if (out == nullptr) return;
  const int lane = threadIdx.x & 31, way = threadIdx.x / 32, c = blockIdx.x * 32 + lane;
  const int first = keys ? q_blocks : 0, last = keys ? blocks : q_blocks;
  float s = 0.0f;
  for (int p = first + way; p < last; p += 8 * 32) {
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bool in = c < dim && p + 32 * i < last;
      v[i] = load_global_if(work + (in ? (size_t)(p + 32 * i) * dim + c : 0), in);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) s += v[i];
  }
  red[way][lane] = s;
  __syncthreads();
  s = warp_sum(red[lane][way]);
  const int col = blockIdx.x * 32 + way;
  if (lane == 0 && col < dim) out[col] = s;
}

bool strides_in_chunks(const HeadsArgs &a, size_t elem, bool backward) {
  const xnor_heads_desc &d = a.d;
  auto good = [&](const void *p, long long s) { return rows_in_pieces(p, s, d.dim, elem); };
  return heads_in_chunks(d) && good(a.q, d.q_stride) && good(a.q_out, d.q_out_stride) && good(a.k, d.k_stride) && good(a.k_out, d.k_out_stride) &&
         (!backward || (good(a.dq_out, d.dq_stride) && good(a.dk_out, d.dk_stride)));
}

unsigned blocks_for(long long items) { return (unsigned)std::min<long long>((items + kWarps - 1) / kWarps, 1 << 20); }

template <class T, int kDim>
cudaError_t run(const HeadsArgs &a, cudaStream_t st) {
  constexpr int kHeads = HeadLane<kDim>::kHeads;
  const int units = (a.d.q_heads + kHeads - 1) / kHeads + (a.d.k_heads + kHeads - 1) / kHeads;
  // as many warps as the GPU holds at once, then a warp has a token to itself
  const int parts = (int)std::min<long long>(units, std::max<long long>(1, 32ll * kSms / a.d.rows));
  const unsigned grid = blocks_for((long long)a.d.rows * parts);
  return a.d.pairs ? launch_kernel(heads_kernel<T, kDim, true>, dim3(grid), 32 * kWarps, 0, st, 1, a, parts)
                   : launch_kernel(heads_kernel<T, kDim, false>, dim3(grid), 32 * kWarps, 0, st, 1, a, parts);
}
template <class T>
cudaError_t run_type(const HeadsArgs &a, cudaStream_t st) {
  if (!strides_in_chunks(a, sizeof(T), false))
    return launch_kernel(heads_loose_kernel<T>, dim3(blocks_for((long long)a.d.rows * (a.d.q_heads + a.d.k_heads))), 32 * kWarps, 0, st, 1, a);
  return a.d.dim == 64 ? run<T, 64>(a, st) : a.d.dim == 128 ? run<T, 128>(a, st) : run<T, 256>(a, st);
}

// Blocks of the backward pass: two per SM at most, shared out by the heads.
struct BackwardBlocks { int q, k; };
BackwardBlocks backward_blocks(int rows, int q_heads, int k_heads) {
  const int most = 2 * (int)kSms;
  auto blocks = [&](int heads, int share) {
    if (heads == 0) return 0;
    return (int)std::min<long long>(std::max(1, share), ((long long)rows * heads + kWarps - 1) / kWarps);
  };
  const int k_share = k_heads == 0 ? 0 : q_heads == 0 ? most : (int)std::max(1ll, (long long)most * k_heads / (q_heads + k_heads));
  return {blocks(q_heads, std::max(1, most - k_share)), blocks(k_heads, k_share)};
}

template <class T, int kDim>
cudaError_t run_backward(const HeadsArgs &a, const BackwardBlocks &b, cudaStream_t st) {
  const dim3 grid((unsigned)(b.q + b.k));
  return a.d.pairs ? launch_kernel(heads_backward_kernel<T, kDim, true>, grid, 32 * kWarps, 0, st, 1, a, b.q)
                   : launch_kernel(heads_backward_kernel<T, kDim, false>, grid, 32 * kWarps, 0, st, 1, a, b.q);
}
template <class T>
cudaError_t run_backward_type(const HeadsArgs &a, const BackwardBlocks &b, cudaStream_t st) {
  if (!strides_in_chunks(a, sizeof(T), true))
    return launch_kernel(heads_backward_loose_kernel<T>, dim3((unsigned)(b.q + b.k)), 32 * kWarps, 0, st, 1, a, b.q);
  return a.d.dim == 64 ? run_backward<T, 64>(a, b, st) : a.d.dim == 128 ? run_backward<T, 128>(a, b, st) : run_backward<T, 256>(a, b, st);
}

}  // namespace

// (Does not depend on the device.)
int heads_parts(int rows, int q_heads, int k_heads) {
  const BackwardBlocks b = backward_blocks(rows, q_heads, k_heads);
  return b.q + b.k;
}

cudaError_t read_status_heads(int *status) {
  cudaError_t e = cudaMemcpyFromSymbol(status, g_status_heads, sizeof(int));
  if (e == cudaSuccess && *status != 0) {
    const int zero = 0;
    e = cudaMemcpyToSymbol(g_status_heads, &zero, sizeof(int));
  }
  return e;
}

cudaError_t launch_heads(const HeadsArgs &a, cudaStream_t st) {
  if (a.d.rows == 0) return cudaSuccess;
  if (a.d.type == XNOR_F32) return run_type<float>(a, st);
  return a.d.type == XNOR_BF16 ? run_type<__nv_bfloat16>(a, st) : run_type<__half>(a, st);
}

cudaError_t launch_heads_backward(const HeadsArgs &args, cudaStream_t st) {
  HeadsArgs a = args;
  if (!a.d.norm || (a.dq_weight == nullptr && a.dk_weight == nullptr)) a.work = nullptr;
  if (!a.d.norm) {
    // values and weights are not given then, and the kernel for whole chunks reads them all the same: the gradients stand in
    a.q = a.dq_out; a.d.q_stride = a.d.dq_stride;
    a.k = a.dk_out; a.d.k_stride = a.d.dk_stride;
    a.q_weight = a.k_weight = nullptr;
  }
  BackwardBlocks b = {0, 0};
  if (a.d.rows > 0) {
    b = backward_blocks(a.d.rows, a.d.q_heads, a.d.k_heads);
    const cudaError_t e = a.d.type == XNOR_F32 ? run_backward_type<float>(a, b, st)
                          : a.d.type == XNOR_BF16 ? run_backward_type<__nv_bfloat16>(a, b, st) : run_backward_type<__half>(a, b, st);
    if (e != cudaSuccess) return e;
  }
  if (a.dq_weight == nullptr && a.dk_weight == nullptr) return cudaSuccess;
  if (a.work == nullptr) b = {0, 0};           // no norm, no rows: zeros
  return launch_kernel(heads_dweight_kernel, dim3((unsigned)((a.d.dim + 31) / 32), 2), 1024, 0, st, 1, (const float *)a.work, b.q, b.q + b.k, a.d.dim,
                       a.dq_weight, a.dk_weight);
}

}  // namespace xnor
