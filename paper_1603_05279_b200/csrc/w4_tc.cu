// Many rows times 4-bit weights on the 5th-generation tensor cores.
//
// out[t][n] = x_scale[t] sum over groups g of scale[g][n] sum over k in g of (code - zero)[n][k] x[t][k].
// The contraction of one group runs on tcgen05.mma kind::f16 with exact 16-bit operands: the matrix operand is
// the 128 weight rows of a tile, expanded from 4 bits into tensor memory (code - zero, which is the same for a
// row's whole group), the other the rows of x in shared memory.  A group's sums leave tensor memory as they
// are finished, are multiplied with the group's scale and added up in fp32 registers, so that no weight is
// rounded: scaling the weights before the product would round each to the operands' 8 or 11 bits.
//
// A block (one per SM, persistent) computes 128 outputs x kRows rows.  A unit of work is one group and up to 128 rows:
// the accumulators are two buffers of tensor memory, so that the tensor core fills one while the other is drained;
// with 256 rows the buffers are the two halves of the rows, and an expanded group serves both.  (512 threads:)
//   promotion  8 warps (256 rows) or 4: a thread holds the sums of one output row, 128 rows of x at most
//   expansion  4 or 8 warps: a thread expands one weight row, 64 columns at a time, straight into tensor memory
//   one warp issues the products, three bring the rows of x into a ring of stages of 64 columns
// Where the tiles are too few for the GPU, the blocks of a cluster divide the columns, and add their sums through
// each other's shared memory in a fixed order.  Every wait is bounded; on expiry the block records
// XNOR_ERR_TIMEOUT, stops and frees its tensor memory.
#include <algorithm>

#include "umma_common.cuh"
#include "w4.cuh"

namespace xnor {

__device__ int g_status_w4 = 0;

namespace {

using namespace umma;

constexpr int kThreads = 512;
constexpr int kTileN = 128;                  // outputs (weight rows) of a tile: the lanes of tensor memory
constexpr int kChunk = 64;                   // columns of a stage
constexpr int kMmaWarp = 12, kLoadWarp = 13, kLoadWarps = 3;
constexpr int kABufs = 8, kACols = kChunk / 2;                 // expanded weights: 8 x 32 columns of tensor memory
constexpr int kDCols = 128, kATmem = 2 * kDCols;               // behind the two accumulators
constexpr int kMaxStages = 8;
constexpr uint32_t kCtrlBytes = 1024;
constexpr int kMaxSplitTc = 8;

template <int kRows>
struct Shape {
  static constexpr int kHalves = kRows > 128 ? 2 : 1;          // products of a unit: kUnit rows each
  static constexpr int kUnit = kRows / kHalves;
  static constexpr int kPromo = kHalves;                       // sets of four warps
  static constexpr int kExpand = 3 - kHalves;
  static constexpr uint32_t kPlane = kRows * 16 + 16;          // eight columns of all rows; 16 more keep the banks apart
  static constexpr uint32_t kStage = 8 * kPlane;
  static constexpr int kStages = kRows > 128 ? 6 : kMaxStages;
  static constexpr uint32_t kScaleBytes = kPromo * 4 * 512;    // a group's scales of x, per promotion warp
  static constexpr size_t kSmem = kCtrlBytes + kScaleBytes + (size_t)kStages * kStage;
  static_assert(kSmem <= 232448, "shared memory");
  static_assert(kHalves == 2 || (size_t)kStages * kStage >= (size_t)kRows * kTileN * 4, "room for the sums of a block");
};

struct TcParams {
  W4Args A;
  int col_tiles, row_tiles, token_tiles;    // chunks of columns; tiles of 128 outputs, of kRows rows
  int split, pieces;
  uint32_t idesc;
};

struct Smem {
  uint32_t afull, aempty, bfull, bempty, dfull, dempty, scales, ring;
  uint32_t *tmem_slot;
  volatile int *abort_flag;
};
__device__ __forceinline__ Smem carve(uint8_t *smem, uint32_t scale_bytes) {
  Smem s;
  s.afull = smem_u32(smem);
  s.aempty = s.afull + 8 * kABufs;
  s.bfull = s.aempty + 8 * kABufs;
  s.bempty = s.bfull + 8 * kMaxStages;
  s.dfull = s.bempty + 8 * kMaxStages;
  s.dempty = s.dfull + 16;
  s.tmem_slot = reinterpret_cast<uint32_t *>(smem + 16 * kABufs + 16 * kMaxStages + 32);
  s.abort_flag = reinterpret_cast<volatile int *>(s.tmem_slot + 1);
  s.scales = s.afull + kCtrlBytes;
  s.ring = s.scales + scale_bytes;
  return s;
}

__device__ __forceinline__ bool wait(const Smem &S, uint32_t bar, uint32_t parity) {
  return mbar_wait(bar, parity, S.abort_flag, &g_status_w4);
}
__device__ __forceinline__ bool wait_warp(const Smem &S, uint32_t bar, uint32_t parity) {
  return __all_sync(0xFFFFFFFFu, wait(S, bar, parity));
}

// A position in a ring of buffers and the parity of its uses.
struct Ring {
  uint32_t at = 0, parity = 0;
  __device__ __forceinline__ void step(uint32_t size) {
    if (++at == size) { at = 0; parity ^= 1u; }
  }
};

// The columns of a block, by its rank in the cluster: whole blocks of 128, so that no group is cut.
struct Span {
  int c0, c1, u0, u1;          // chunks and groups
  __device__ __forceinline__ Span(const TcParams &P, int rank) {
    const int blocks = (P.col_tiles + 1) / 2, group = P.A.d.group;
    const int b0 = (int)((long long)blocks * rank / P.split), b1 = (int)((long long)blocks * (rank + 1) / P.split);
    c0 = 2 * b0;
    c1 = min(2 * b1, P.col_tiles);
    u0 = b0 * (128 / group);
    u1 = min(b1 * (128 / group), (P.A.d.K + group - 1) / group);
  }
};

// D (+)= A (tensor memory, 128 x 16) B (shared memory, 16 x kUnit)
__device__ __forceinline__ void mma_tmem(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}

__device__ __forceinline__ uint32_t elect_one() {
  uint32_t pred = 0;
  asm volatile(
      "{\n\t.reg .b32 rx;\n\t.reg .pred px;\n\t"
      "elect.sync rx|px, %1;\n\t"
      "@px mov.s32 %0, 1;\n\t}"
      : "+r"(pred) : "r"(0xFFFFFFFFu));
  return pred;
}

// ------------------------------------------------------------------ the issuing thread
template <int kRows>
__device__ void mma_loop(const TcParams &P, const Smem &S, const Span &span, int tiles, uint32_t tmem) {
  using Sh = Shape<kRows>;
  const int group = P.A.d.group;
  Ring a, b, d;                                    // d: the accumulator (one half: both in turn)
  uint32_t dpar[2] = {1u, 1u};
  for (int tile = 0; tile < tiles; ++tile) {
    int acquired = span.c0;                        // chunks whose buffers are known to be full
    Ring aw = a, bw = b;
    for (int u = span.u0; u < span.u1; ++u) {
      const int k0 = u * group, steps = min(group, P.col_tiles * kChunk - k0) / 16;
      const bool ends = ((k0 + group) % kChunk) == 0 || u + 1 == span.u1;      // the unit's last chunk is done with
      const Ring a0 = a, b0 = b;
#pragma unroll 1
      for (int h = 0; h < Sh::kHalves; ++h) {
        const uint32_t buf = Sh::kHalves == 2 ? (uint32_t)h : d.at;
        if (!wait(S, S.dempty + 8u * buf, dpar[buf])) return;
        dpar[buf] ^= 1u;
        tc_fence_after();
        a = a0;
        b = b0;
        uint32_t accumulate = 0u;
#pragma unroll 1
        for (int s = 0; s < steps; s += 4 - (s + k0 / 16) % 4) {
          const int in_chunk = (k0 / 16 + s) % 4, c = (k0 + 16 * s) / kChunk;
          if (c >= acquired) {
            if (!wait(S, S.afull + 8u * aw.at, aw.parity) || !wait(S, S.bfull + 8u * bw.at, bw.parity)) return;
            tc_fence_after();
            aw.step(kABufs);
            bw.step(Sh::kStages);
            acquired = c + 1;
          }
          const uint32_t at = tmem + (uint32_t)(kATmem + (int)a.at * kACols + in_chunk * 8);
          const uint32_t bt = S.ring + b.at * Sh::kStage + (uint32_t)(2 * in_chunk) * Sh::kPlane + (uint32_t)(h * Sh::kUnit) * 16u;
          const int n = min(4 - in_chunk, steps - s);
#pragma unroll 1
          for (int i = 0; i < n; ++i) {
            mma_tmem(tmem + buf * kDCols, at + 8u * i, make_desc(bt + 2u * i * Sh::kPlane, Sh::kPlane, 128u), P.idesc, accumulate);
            accumulate = 1u;
          }
          const bool chunk_done = in_chunk + n == 4 || (ends && s + n == steps);
          if (chunk_done) {
            if (h == Sh::kHalves - 1) {
              umma_commit(S.aempty + 8u * a.at);
              umma_commit(S.bempty + 8u * b.at);
            }
            a.step(kABufs);
            b.step(Sh::kStages);
          }
        }
        umma_commit(S.dfull + 8u * buf);
      }
      if (Sh::kHalves == 1) d.at ^= 1u;
    }
  }
}

// ------------------------------------------------------------------ expansion of the weights
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t r[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}

// Set `which` of `sets` takes every sets-th chunk.  A thread expands one weight row: eight words of a chunk, which
// come in two chunks ahead.
template <class T, int kRows>
__device__ void expand_role(const TcParams &P, const Smem &S, const Span &span, int first, int step, int total, int which, int quarter,
                            int lane, uint32_t tmem) {
  constexpr int kSets = Shape<kRows>::kExpand;
  const int N = P.A.d.N, group = P.A.d.group, r = 32 * quarter + lane, per_tile = span.c1 - span.c0;
  const uint32_t t_lane = tmem + ((uint32_t)(32 * quarter) << 16) + kATmem;
  uint32_t seq = 0;                                 // chunks of all tiles in sequence: their buffers
  for (int tile = first; tile < total; tile += step, seq += (uint32_t)per_tile) {
    const int n = (tile % P.row_tiles) * kTileN + r, nc = min(n, N - 1);
    const uint2 *w = reinterpret_cast<const uint2 *>(P.A.w) +
                     ((size_t)(nc / kW4Rows) * P.col_tiles * 32 + 4 * (nc & 7)) * 2 + ((nc >> 3) & 1);
    struct Ahead { uint2 w[4]; uint32_t z[2]; };
    auto fetch = [&](int c, Ahead &f) {
      if (c >= span.c1) return;
#pragma unroll
      for (int t = 0; t < 4; ++t) f.w[t] = load_global(w + ((size_t)c * 32 + t) * 2);
      f.z[0] = f.z[1] = 8u;
      if (P.A.zeros) {
        const int last = (P.A.d.K - 1) / group;
        f.z[0] = load_global(P.A.zeros + (size_t)min(c * kChunk / group, last) * N + nc);
        f.z[1] = group == 32 ? load_global(P.A.zeros + (size_t)min(2 * c + 1, last) * N + nc) : f.z[0];
      }
    };
    const int skip = (int)((uint32_t)(which + kSets - (int)(seq % kSets)) % kSets);     // this set's first chunk of the tile
    Ahead f[2];
    fetch(span.c0 + skip, f[0]);
    fetch(span.c0 + skip + kSets, f[1]);
#pragma unroll 1
    for (int i = skip; i < per_tile; i += kSets) {
      const Ahead now = f[0];
      f[0] = f[1];
      fetch(span.c0 + i + 2 * kSets, f[1]);
      const uint32_t at = (seq + (uint32_t)i) % kABufs, use = (seq + (uint32_t)i) / kABufs;
      if (!wait_warp(S, S.aempty + 8u * at, (use & 1u) ^ 1u)) return;
      tc_fence_after();
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const uint32_t zero = w4_zero(now.z[half], T());
        uint32_t v[16];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int p = 0; p < 4; ++p) v[4 * t + p] = w4_pair(half == 0 ? now.w[t].x : now.w[t].y, p, T(), zero);
        __syncwarp();
        tmem_st16(t_lane + at * kACols + 16u * half, v);
      }
      asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(S.afull + 8u * at);
    }
  }
}

// ------------------------------------------------------------------ the rows of x
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, uint32_t bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(__cvta_generic_to_global(src)), "r"(bytes) : "memory");
}

// Three warps share every stage.  Rows whose addresses allow it come in by asynchronous 16-byte copies, two stages in
// flight; others, and 8-bit rows, which become 16-bit numbers, through registers.  Shared memory holds
// [columns / 8][row][16 bytes], the operand layout without swizzle; missing rows and columns are zeros.
template <int kType, int kRows>
__device__ void load_role(const TcParams &P, const Smem &S, const Span &span, int first, int step, int total, int w, int lane) {
  using Sh = Shape<kRows>;
  const int K = P.A.d.K, piece = lane & 7;
  const bool async = RowsOf<kType>::kBytes == 2 && P.pieces;
  constexpr int kDepth = 2;
  Ring fill, done;
  int pending = 0;
  auto finish = [&]() {                              // the oldest stage in flight is complete
    fence_proxy_async();
    __syncwarp();
    if (lane == 0) mbar_arrive(S.bfull + 8u * done.at);
    done.step(Sh::kStages);
    --pending;
  };
  for (int tile = first; tile < total; tile += step) {
    const long long tok0 = (long long)(tile / P.row_tiles) * kRows;
    const int rows = (int)min((long long)kRows, P.A.r.rows - tok0);
    const uint8_t *x = static_cast<const uint8_t *>(P.A.x) + tok0 * P.A.r.x_stride * RowsOf<kType>::kBytes;
    const long long row_bytes = P.A.r.x_stride * RowsOf<kType>::kBytes;
#pragma unroll 1
    for (int c = span.c0; c < span.c1; ++c) {
      if (!wait_warp(S, S.bempty + 8u * fill.at, fill.parity ^ 1u)) {
        asm volatile("cp.async.wait_all;" ::: "memory");
        return;
      }
      const int k = c * kChunk + 8 * piece;
      const uint32_t dst = S.ring + fill.at * Sh::kStage + (uint32_t)piece * Sh::kPlane;
      int row = 4 * w + (lane >> 3);
      if (async) {
        const uint32_t bytes = (uint32_t)max(0, min(16, 2 * (K - k)));
        const uint8_t *src = x + (long long)row * row_bytes + 2 * (bytes > 0 ? k : 0);
#pragma unroll 4
        for (; row < kRows; row += 4 * kLoadWarps, src += 4 * kLoadWarps * row_bytes)
          copy16(dst + (uint32_t)row * 16u, row < rows ? src : x, row < rows ? bytes : 0u);
        asm volatile("cp.async.commit_group;" ::: "memory");
        ++pending;
        if (pending > kDepth) {
          asm volatile("cp.async.wait_group %0;" ::"n"(kDepth) : "memory");
          finish();
        }
      } else {
#pragma unroll 1
        for (; row < kRows; row += 4 * kLoadWarps * 4) {
          uint32_t v[4][4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int rr = row + 4 * kLoadWarps * i;
            if (rr < rows) {
              load_x8<kType>(x + (long long)rr * row_bytes, k, K, P.pieces, v[i]);
            } else {
#pragma unroll
              for (int q = 0; q < 4; ++q) v[i][q] = 0u;
            }
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int rr = row + 4 * kLoadWarps * i;
            if (rr < kRows) sts128(dst + (uint32_t)rr * 16u, v[i][0], v[i][1], v[i][2], v[i][3]);
          }
        }
        ++pending;
        finish();
      }
      fill.step(Sh::kStages);
    }
  }
  if (async) {
    asm volatile("cp.async.wait_all;" ::: "memory");
    while (pending > 0) finish();
  }
}

// ------------------------------------------------------------------ promotion: sums of groups -> sums of a row
__device__ __forceinline__ void store_out(const W4Args &A, long long row, int n, float v) {
  const size_t at = (size_t)(row * A.r.out_stride) + n;
  if (A.r.out_type == XNOR_F32) static_cast<float *>(A.out)[at] = v;
  else if (A.r.out_type == XNOR_BF16) static_cast<__nv_bfloat16 *>(A.out)[at] = __float2bfloat16_rn(v);
  else static_cast<__half *>(A.out)[at] = __float2half_rn(v);
}

__device__ __forceinline__ float4 lds_f4(uint32_t addr) {
  uint32_t v[4];
  lds128(addr, v);
  return make_float4(__uint_as_float(v[0]), __uint_as_float(v[1]), __uint_as_float(v[2]), __uint_as_float(v[3]));
}

template <int kRows>
__device__ bool promote_role(const TcParams &P, const Smem &S, const Span &span, int first, int step, int total, int set, int quarter,
                             int lane, uint32_t tmem) {
  using Sh = Shape<kRows>;
  constexpr int kUnit = Sh::kUnit;
  const W4Args &A = P.A;
  const int N = A.d.N;
  const bool x_groups = A.x_scales != nullptr && A.r.x_group != 0;
  const int G = (A.d.K + A.d.group - 1) / A.d.group;
  const uint32_t t_lane = tmem + ((uint32_t)(32 * quarter) << 16);
  const uint32_t my_scales = S.scales + (uint32_t)(4 * set + quarter) * 512u;
  uint32_t parity[2] = {0u, 0u}, next = 0u;
  for (int tile = first; tile < total; tile += step) {
    const int n = (tile % P.row_tiles) * kTileN + 32 * quarter + lane, nc = min(n, N - 1);
    const long long tok0 = (long long)(tile / P.row_tiles) * kRows + set * kUnit;
    float acc[kUnit];
#pragma unroll
    for (int i = 0; i < kUnit; ++i) acc[i] = 0.0f;
    float scale = span.u0 < span.u1 ? load_global(A.scales + (size_t)span.u0 * N + nc) : 0.0f;
#pragma unroll 1
    for (int u = span.u0; u < span.u1; ++u) {
      const float s = scale;
      if (u + 1 < span.u1) scale = load_global(A.scales + (size_t)(u + 1) * N + nc);
      if (x_groups) {
        __syncwarp();
#pragma unroll
        for (int i = 0; i < (kUnit + 31) / 32; ++i) {
          const int col = lane + 32 * i;
          const float v = col < kUnit && tok0 + col < A.r.rows ? load_global(A.x_scales + (tok0 + col) * G + u) : 0.0f;
          if (col < kUnit) sts32(my_scales + 4u * col, __float_as_uint(v));
        }
        __syncwarp();
      }
      const uint32_t buf = Sh::kHalves == 2 ? (uint32_t)set : next;
      if (!wait_warp(S, S.dfull + 8u * buf, parity[buf])) return false;
      parity[buf] ^= 1u;
      next ^= 1u;
      tc_fence_after();
#pragma unroll
      for (int j = 0; j < kUnit / 16; ++j) {
        int32_t v[16];
        __syncwarp();
        tmem_ld16(t_lane + buf * kDCols + 16u * j, v);
        tmem_wait16(v);
        if (j + 1 == kUnit / 16) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(S.dempty + 8u * buf);
        }
        if (x_groups) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float4 f = lds_f4(my_scales + 64u * j + 16u * i);
            acc[16 * j + 4 * i] = fmaf(__int_as_float(v[4 * i]) * f.x, s, acc[16 * j + 4 * i]);
            acc[16 * j + 4 * i + 1] = fmaf(__int_as_float(v[4 * i + 1]) * f.y, s, acc[16 * j + 4 * i + 1]);
            acc[16 * j + 4 * i + 2] = fmaf(__int_as_float(v[4 * i + 2]) * f.z, s, acc[16 * j + 4 * i + 2]);
            acc[16 * j + 4 * i + 3] = fmaf(__int_as_float(v[4 * i + 3]) * f.w, s, acc[16 * j + 4 * i + 3]);
          }
        } else {
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[16 * j + i] = fmaf(__int_as_float(v[i]), s, acc[16 * j + i]);
        }
      }
    }
    if (P.split > 1) {                     // [row of x][output], for the cluster
#pragma unroll
      for (int i = 0; i < kUnit; ++i)
        sts32(S.ring + (uint32_t)(((set * kUnit + i) * kTileN + 32 * quarter + lane) * 4), __float_as_uint(acc[i]));
    } else if (n < N) {
      const float *xs = A.x_scales != nullptr && !x_groups ? A.x_scales : nullptr;
#pragma unroll
      for (int i = 0; i < kUnit; ++i)
        if (tok0 + i < A.r.rows) store_out(A, tok0 + i, n, xs ? acc[i] * load_global(xs + tok0 + i) : acc[i]);
    }
  }
  return true;
}

__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

template <int kType, int kRows>
__global__ void __launch_bounds__(kThreads, 1)
w4_tc_kernel(const __grid_constant__ TcParams P) {
  using Sh = Shape<kRows>;
  using T = typename RowsOf<kType>::T;
  extern __shared__ __align__(128) uint8_t smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const Smem S = carve(smem, Sh::kScaleBytes);
  if (threadIdx.x == 0) {
    for (int i = 0; i < kABufs; ++i) { mbar_init(S.afull + 8u * i, 4); mbar_init(S.aempty + 8u * i, 1); }
    for (int i = 0; i < kMaxStages; ++i) { mbar_init(S.bfull + 8u * i, kLoadWarps); mbar_init(S.bempty + 8u * i, 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(S.dfull + 8u * i, 1); mbar_init(S.dempty + 8u * i, 4); }
    *S.abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(S.tmem_slot)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  // the tensor memory is taken before any thread lets the next kernel start: a block of that kernel on this
  // SM could take it first, and then waits for this one
  __syncthreads();
  stream_order();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *S.tmem_slot;
  const int rank = (int)(blockIdx.x % (unsigned)P.split), first = (int)(blockIdx.x / (unsigned)P.split), step = (int)(gridDim.x / (unsigned)P.split);
  const int total = P.row_tiles * P.token_tiles, mine = first < total ? (total - first + step - 1) / step : 0;
  const Span span(P, rank);
  if (warp < 4 * Sh::kPromo) promote_role<kRows>(P, S, span, first, step, total, warp >> 2, warp & 3, lane, tmem);
  else if (warp < kMmaWarp) expand_role<T, kRows>(P, S, span, first, step, total, (warp >> 2) - Sh::kPromo, warp & 3, lane, tmem);
  else if (warp == kMmaWarp) {
    if (elect_one()) mma_loop<kRows>(P, S, span, mine, tmem);
    __syncwarp();
  } else load_role<kType, kRows>(P, S, span, first, step, total, warp - kLoadWarp, lane);
  tc_fence_before();
  __syncthreads();
  if (warp == kMmaWarp)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
  if (P.split == 1) return;
  // a cluster has one tile; its blocks write shares of the rows, each the sums of all in the same order
  cluster_barrier();
  const int n0 = (first % P.row_tiles) * kTileN;
  const long long tok0 = (long long)(first / P.row_tiles) * kRows;
  const bool row_scale = P.A.x_scales != nullptr && P.A.r.x_group == 0;
  const int r0 = kRows * rank / P.split, r1 = kRows * (rank + 1) / P.split;
  for (int e = r0 * kTileN + threadIdx.x; e < r1 * kTileN; e += kThreads) {
    const int n = e % kTileN;
    const long long row = tok0 + e / kTileN;
    if (row >= P.A.r.rows || n0 + n >= P.A.d.N) continue;
    float s = 0.0f;
    for (int i = 0; i < P.split; ++i) {
      uint32_t a;
      float v;
      asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(S.ring + 4u * (uint32_t)e), "r"(i));
      asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
      s += v;
    }
    if (row_scale) s *= load_global(P.A.x_scales + row);
    store_out(P.A, row, n0 + n, s);
  }
  cluster_barrier();
}

template <int kType, int kRows>
cudaError_t run(const W4Args &a, cudaStream_t st) {
  using Sh = Shape<kRows>;
  static bool attr_flags[64] = {};
  bool &attr_set = attr_done_for_current_device(attr_flags);
  if (!attr_set) {
    const cudaError_t e = cudaFuncSetAttribute(w4_tc_kernel<kType, kRows>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Sh::kSmem);
    if (e != cudaSuccess) { (void)cudaGetLastError(); return e; }
    attr_set = true;
  }
  TcParams P;
  P.A = a;
  P.col_tiles = w4_col_tiles(a.d);
  P.row_tiles = (a.d.N + kTileN - 1) / kTileN;
  P.token_tiles = (a.r.rows + kRows - 1) / kRows;
  P.pieces = rows_in_pieces(a.x, a.r.x_stride, 8, RowsOf<kType>::kBytes);
  const int total = P.row_tiles * P.token_tiles, sms = sm_count_of_current_device();
  // blocks divide the columns while that still adds SMs and each keeps four blocks of 128 columns
  P.split = 1;
  while (Sh::kHalves == 1 && P.split < kMaxSplitTc && 2 * P.split * total <= sms && P.col_tiles >= 16 * P.split) P.split *= 2;
  // instruction descriptor: D fp32, A and B bf16 or f16, both K-major, M = 128
  const uint32_t format = kType == XNOR_BF16 ? 1u : 0u;
  P.idesc = (1u << 4) | (format << 7) | (format << 10) | ((uint32_t)(Sh::kUnit >> 3) << 17) | ((uint32_t)(kTileN >> 4) << 24);
  const unsigned grid = P.split > 1 ? (unsigned)(total * P.split) : (unsigned)std::min(total, sms);
  return launch_kernel(w4_tc_kernel<kType, kRows>, dim3(grid), kThreads, Sh::kSmem, st, (unsigned)P.split, P);
}

// 256 rows of x per block halve the expansion per product; a block of them takes no share of a cluster (its two
// halves end one after the other), so they are for problems that fill the GPU.
template <int kType>
cudaError_t run_type(const W4Args &a, cudaStream_t st) {
  const long long tiles = (a.d.N + kTileN - 1) / kTileN * ((a.r.rows + 255ll) / 256);
  if (a.r.rows > 128 && 2 * tiles > sm_count_of_current_device()) return run<kType, 256>(a, st);
  if (a.r.rows <= 32) return run<kType, 32>(a, st);
  if (a.r.rows <= 64) return run<kType, 64>(a, st);
  return run<kType, 128>(a, st);
}

}  // namespace

cudaError_t launch_w4_many_rows(const W4Args &a, cudaStream_t st) {
  switch (a.r.x_type) {
    case XNOR_BF16: return run_type<XNOR_BF16>(a, st);
    case XNOR_F16: return run_type<XNOR_F16>(a, st);
    case XNOR_I8: return run_type<XNOR_I8>(a, st);
    default: return run_type<XNOR_E4M3>(a, st);
  }
}

cudaError_t read_status_w4(int *status) {
  cudaError_t e = cudaMemcpyFromSymbol(status, g_status_w4, sizeof(int));
  if (e == cudaSuccess && *status != 0) {
    const int zero = 0;
    e = cudaMemcpyToSymbol(g_status_w4, &zero, sizeof(int));
  }
  return e;
}

}  // namespace xnor
