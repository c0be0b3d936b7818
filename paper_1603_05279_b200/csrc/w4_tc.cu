// Many rows times 4-bit weights on the 5th-generation tensor cores.
//
// out[t][n] = x_scale[t] sum over groups g of scale[g][n] sum over k in g of (code - zero)[n][k] x[t][k].
// The contraction of one group runs on tcgen05.mma kind::f16 with exact 16-bit operands: the matrix operand is
// the 128 weight rows of a tile, expanded from 4 bits into tensor memory (code - zero, which is the same for a
// row's whole group), the other the rows of x in shared memory.  A group's sums leave tensor memory as they
// are finished, are multiplied with the group's scale and added up in fp32 registers, so that no weight is
// rounded: scaling the weights before the product would round each to the operands' 8 or 11 bits.
//
// A block (one per SM, persistent) computes 128 outputs x kRows rows of x.  A unit of work is one group: its sums
// have two buffers in tensor memory, so that the tensor core fills one while the other is drained.  20 warps (16):
//   promotion  8 warps (4 up to 64 rows): a thread holds the sums of one output and up to 96 rows of x
//   expansion  8 warps: a thread expands one weight row, 64 columns at a time, straight into tensor memory
//   one warp issues the products; one copies the rows of x, by tensor copies, into a ring of stages of 64 columns
//   (where they cannot be copied as they are, three warps bring them through registers)
// Where the tiles are too few for the GPU, the blocks of a cluster divide the columns, and add their sums through
// each other's shared memory in a fixed order.  Every wait is bounded; on expiry the block records
// XNOR_ERR_TIMEOUT, stops and frees its tensor memory.
#include <cuda.h>

#include <algorithm>
#include <atomic>

#include "umma_common.cuh"
#include "w4.cuh"

namespace xnor {

__device__ int g_status_w4 = 0;

namespace {

using namespace umma;

constexpr int kTileN = 128;                  // outputs (weight rows) of a tile: the lanes of tensor memory
constexpr int kChunk = 64;                   // columns of a stage
constexpr int kLoadWarps = 3;
constexpr int kACols = kChunk / 2;           // tensor-memory columns of a chunk of expanded weights
constexpr int kMaxStages = 8;
constexpr uint32_t kCtrlBytes = 1024;
constexpr int kMaxSplitTc = 8;

template <int kRows>
struct Shape {
  static constexpr int kPromo = kRows > 64 ? 2 : 1;            // sets of four warps
  static constexpr int kUnit = kRows / kPromo;                 // rows of x of a set
  static constexpr int kExpand = 2;
  static constexpr int kMmaWarp = 4 * (kPromo + kExpand), kLoadWarp = kMmaWarp + 1;
  static constexpr int kThreads = 32 * (kMmaWarp + 4);
  static constexpr int kATmem = kRows > 128 ? 2 * kRows : 256; // behind the two accumulators
  static constexpr int kStages = (512 - kATmem) / kACols;      // chunks: weights in tensor memory, rows of x in shared
  static constexpr uint32_t kStage = kRows * kChunk * 2;       // a row of x: 128 bytes, swizzled
  static constexpr uint32_t kScaleBytes = 8 * 512;             // a group's scales of x, per promotion warp
  static constexpr size_t kSmem = 1024 + kCtrlBytes + kScaleBytes + (size_t)kStages * kStage;   // (1024: to align the ring)
  // Registers per thread as launched, and after they are dealt out anew: the promotion's hold its sums.
  static constexpr int kRegs = kThreads == 512 ? 128 : 96;
  static constexpr int kPromoRegs = kRows > 128 ? 144 : kRows > 64 ? 128 : 128, kOtherRegs = kRows > 128 ? 64 : kRows > 64 ? 72 : 128;
  static_assert(kPromo * 128 * kPromoRegs + (kThreads - kPromo * 128) * kOtherRegs <= kThreads * kRegs, "registers");
  static_assert(kSmem <= 232448 && kStages <= kMaxStages, "shared and tensor memory");
  static_assert((size_t)kStages * kStage >= (size_t)kRows * kTileN * 4 || kRows > 128, "room for the sums of a block");
};

struct TcParams {
  CUtensorMap x_map;                        // the rows of x, 64 columns x kRows rows at a time
  W4Args A;
  int col_tiles, row_tiles, token_tiles;    // chunks of columns; tiles of 128 outputs, of kRows rows
  int split, pieces, copies;                // copies: x_map is there
  uint32_t idesc;
};

struct Smem {
  uint32_t full, empty, dfull, dempty, scales, ring;
  uint32_t *tmem_slot;
  volatile int *abort_flag;
};
__device__ __forceinline__ Smem carve(uint8_t *smem, uint32_t scale_bytes) {
  Smem s;
  s.full = smem_u32(smem);
  s.empty = s.full + 8 * kMaxStages;
  s.dfull = s.empty + 8 * kMaxStages;
  s.dempty = s.dfull + 16;
  s.tmem_slot = reinterpret_cast<uint32_t *>(smem + 16 * kMaxStages + 32);
  s.abort_flag = reinterpret_cast<volatile int *>(s.tmem_slot + 1);
  s.scales = s.full + kCtrlBytes;
  s.ring = (s.scales + scale_bytes + 1023u) & ~1023u;
  return s;
}

__device__ __forceinline__ bool wait(const Smem &S, uint32_t bar, uint32_t parity) {
  return mbar_wait(bar, parity, S.abort_flag, &g_status_w4);
}
__device__ __forceinline__ bool wait_warp(const Smem &S, uint32_t bar, uint32_t parity) {
  return __all_sync(0xFFFFFFFFu, wait(S, bar, parity));
}

// The same as straight code, for the warps whose registers hold sums: a call would have them move around it.
__device__ __forceinline__ bool wait_inline(const Smem &S, uint32_t bar, uint32_t parity) {
  if (mbar_try(bar, parity)) return true;
  const long long t0 = clock64();
  bool ok = false;
#pragma unroll 1
  while (!ok && *S.abort_flag == 0) {
    ok = mbar_try(bar, parity);
    if (!ok && clock64() - t0 > kWaitCycles) {
      *S.abort_flag = 1;
      atomicExch(&g_status_w4, (int)XNOR_ERR_TIMEOUT);
    }
  }
  return ok;
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
// Operand of the rows of x: 128-byte rows, swizzled in groups of eight (1024 bytes); 16 columns are 32 bytes on.
__device__ __forceinline__ uint64_t swizzled_desc(uint32_t addr) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | (1ull << 16) | ((uint64_t)(1024u >> 4) << 32) | (1ull << 46) | (2ull << 61);
}

template <int kRows>
__device__ void mma_loop(const TcParams &P, const Smem &S, const Span &span, int tiles, uint32_t tmem) {
  using Sh = Shape<kRows>;
  const int group = P.A.d.group;
  const uint32_t idesc = P.idesc;
  const uint64_t desc0 = swizzled_desc(S.ring);
  Ring r;
  bool ready = false;                              // the stage at hand was seen to be full
  uint32_t buf = 0u, dpar = 1u;                    // the accumulator and the parity of its being drained
  // n products of 16 columns from column 16 `from` of the chunk at hand
  auto products = [&](int from, int n, uint32_t accumulate) {
    const uint32_t d = tmem + buf * (uint32_t)kRows, at = tmem + (uint32_t)Sh::kATmem + r.at * kACols + 8u * (uint32_t)from;
    const uint64_t bt = desc0 + (uint64_t)(r.at * (Sh::kStage >> 4) + 2u * (uint32_t)from);
    mma_tmem(d, at, bt, idesc, accumulate);
    mma_tmem(d, at + 8u, bt + 2u, idesc, 1u);
    if (n > 2) {
      mma_tmem(d, at + 16u, bt + 4u, idesc, 1u);
      mma_tmem(d, at + 24u, bt + 6u, idesc, 1u);
    }
  };
  auto acquire = [&]() {
    if (!ready && !wait(S, S.full + 8u * r.at, r.parity)) return false;
    tc_fence_after();
    // (the next stage's barrier is looked at before this one's products are issued)
    Ring next = r;
    next.step(Sh::kStages);
    ready = mbar_try(S.full + 8u * next.at, next.parity);
    return true;
  };
  auto release = [&]() {
    umma_commit(S.empty + 8u * r.at);
    r.step(Sh::kStages);
  };
  for (int tile = 0; tile < tiles; ++tile) {
    int c = span.c0;
#pragma unroll 1
    for (int u = span.u0; u < span.u1; ++u) {
      if (!wait(S, S.dempty + 8u * buf, dpar)) return;
      tc_fence_after();
      if (group == 32) {                           // half a chunk
        const int half = u & 1;
        if (half == 0 && !acquire()) return;
        products(2 * half, 2, 0u);
        if (half == 1 || u + 1 == span.u1) release();
      } else {
        if (!acquire()) return;
        products(0, 4, 0u);
        release();
        ++c;
        if (group == 128 && c < span.c1) {
          if (!acquire()) return;
          products(0, 4, 1u);
          release();
          ++c;
        }
      }
      umma_commit(S.dfull + 8u * buf);
      buf ^= 1u;
      if (buf == 0u) dpar ^= 1u;
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

// Set `which` takes every kExpand-th chunk.  A thread expands one weight row: eight words of a chunk, which come
// in two chunks ahead.
struct Ahead {
  uint2 w[4];
  uint32_t z[2];
};

template <class T, int kRows>
__device__ void expand_role(const TcParams &P, const Smem &S, const Span &span, int first, int step, int total, int which, int quarter,
                            int lane, uint32_t tmem) {
  using Sh = Shape<kRows>;
  constexpr int kSets = Sh::kExpand;
  const int N = P.A.d.N, group = P.A.d.group, r = 32 * quarter + lane, per_tile = span.c1 - span.c0;
  const int last_group = (P.A.d.K - 1) / group;
  const uint32_t t_lane = tmem + ((uint32_t)(32 * quarter) << 16) + (uint32_t)Sh::kATmem;
  uint32_t seq = 0;                                 // chunks of all tiles in sequence: their buffers
  for (int tile = first; tile < total; tile += step, seq += (uint32_t)per_tile) {
    const int nc = min((tile % P.row_tiles) * kTileN + r, N - 1);
    const uint2 *w = reinterpret_cast<const uint2 *>(P.A.w) +
                     ((size_t)(nc / kW4Rows) * P.col_tiles * 32) * 2 + ((nc >> 3) & 1);
    auto fetch = [&](int i, Ahead &f) {
      if (i >= per_tile) return;
      const int c = span.c0 + i;
#pragma unroll
      for (int t = 0; t < 4; ++t) f.w[t] = load_global(w + ((size_t)c * 32 + w4_place(nc, 8 * t)) * 2);
      f.z[0] = f.z[1] = 8u;
      if (P.A.zeros) {
        f.z[0] = load_global(P.A.zeros + (size_t)min(c * kChunk / group, last_group) * N + nc);
        f.z[1] = group == 32 ? load_global(P.A.zeros + (size_t)min(2 * c + 1, last_group) * N + nc) : f.z[0];
      }
    };
    auto expand = [&](int i, const Ahead &f) {
      const uint32_t at = (seq + (uint32_t)i) % Sh::kStages, use = (seq + (uint32_t)i) / Sh::kStages;
      if (!wait_warp(S, S.empty + 8u * at, (use & 1u) ^ 1u)) return false;
      tc_fence_after();
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const uint32_t zero = w4_zero(f.z[half], T());
        uint32_t v[16];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int p = 0; p < 4; ++p) v[4 * t + p] = w4_pair(half == 0 ? f.w[t].x : f.w[t].y, p, T(), zero);
        tmem_st16(t_lane + at * kACols + 16u * half, v);
      }
      asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(S.full + 8u * at);
      return true;
    };
    const int skip = (int)(((uint32_t)(which + kSets) - seq % kSets) % kSets);     // this set's first chunk of the tile
    Ahead f0, f1;                                   // (two by name: moving one to the other would wait for its loads)
    fetch(skip, f0);
    fetch(skip + kSets, f1);
#pragma unroll 1
    for (int i = skip; i < per_tile; i += 2 * kSets) {
      if (!expand(i, f0)) return;
      fetch(i + 2 * kSets, f0);
      if (i + kSets >= per_tile) break;
      if (!expand(i + kSets, f1)) return;
      fetch(i + 3 * kSets, f1);
    }
  }
}

// ------------------------------------------------------------------ the rows of x
// One thread copies a stage with one tensor copy, which also fills what does not exist with zeros.
template <int kRows>
__device__ void copy_role(const TcParams &P, const Smem &S, const Span &span, int first, int step, int total) {
  constexpr uint32_t kStages = Shape<kRows>::kStages;
  Ring r;
  for (int tile = first; tile < total; tile += step) {
    const int tok0 = (tile / P.row_tiles) * kRows;
#pragma unroll 1
    for (int c = span.c0; c < span.c1; ++c) {
      if (!wait(S, S.empty + 8u * r.at, r.parity ^ 1u)) {
        // gave up: the copies in flight must land before the block's shared memory is released
        for (uint32_t s = 0; s < kStages; ++s)
          for (int i = 0; i < (1 << 12) && !mbar_try(S.full + 8u * s, s < r.at ? r.parity : r.parity ^ 1u); ++i) {}
        return;
      }
      const uint32_t bar = S.full + 8u * r.at;
      mbar_arrive_expect_tx(bar, Shape<kRows>::kStage);
      asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                   ::"r"(S.ring + r.at * Shape<kRows>::kStage), "l"(&P.x_map), "r"(c * kChunk), "r"(tok0), "r"(bar) : "memory");
      r.step(kStages);
    }
  }
}

// Three warps share every stage: rows in 8 bits become 16-bit numbers, others are at addresses that tensor copies
// do not take.
template <int kType, int kRows>
__device__ void load_role(const TcParams &P, const Smem &S, const Span &span, int first, int step, int total, int w, int lane) {
  using Sh = Shape<kRows>;
  const int K = P.A.d.K, piece = lane & 7;
  Ring fill;
  for (int tile = first; tile < total; tile += step) {
    const long long tok0 = (long long)(tile / P.row_tiles) * kRows;
    const int rows = (int)min((long long)kRows, P.A.r.rows - tok0);
    const long long row_bytes = P.A.r.x_stride * RowsOf<kType>::kBytes;
    const uint8_t *x = static_cast<const uint8_t *>(P.A.x) + tok0 * row_bytes;
#pragma unroll 1
    for (int c = span.c0; c < span.c1; ++c) {
      if (!wait_warp(S, S.empty + 8u * fill.at, fill.parity ^ 1u)) return;
      const int k = c * kChunk + 8 * piece;
      const uint32_t dst = S.ring + fill.at * Sh::kStage;
#pragma unroll 1
      for (int row = 4 * w + (lane >> 3); row < kRows; row += 4 * kLoadWarps * 4) {
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
          if (rr < kRows) sts128(dst + (uint32_t)rr * 128u + (uint32_t)((piece ^ (rr & 7)) * 16), v[i][0], v[i][1], v[i][2], v[i][3]);
        }
      }
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) mbar_arrive(S.full + 8u * fill.at);
      fill.step(Sh::kStages);
    }
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
__device__ void promote_role(const TcParams &P, const Smem &S, const Span &span, int first, int step, int total, int set, int quarter,
                             int lane, uint32_t tmem) {
  using Sh = Shape<kRows>;
  constexpr int kUnit = Sh::kUnit;
  const W4Args &A = P.A;
  const int N = A.d.N;
  const bool x_groups = A.x_scales != nullptr && A.r.x_group != 0;
  const int G = (A.d.K + A.d.group - 1) / A.d.group;
  const uint32_t t_lane = tmem + ((uint32_t)(32 * quarter) << 16);
  const uint32_t my_scales = S.scales + (uint32_t)(4 * set + quarter) * 512u;
  uint32_t buf = 0u, parity = 0u;
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
      if (!__all_sync(0xFFFFFFFFu, wait_inline(S, S.dfull + 8u * buf, parity))) return;
      tc_fence_after();
      // 32 values at a time: a load of tensor memory takes as long for 16
      constexpr int kLoad = kRows > 64 ? 16 : 32;
#pragma unroll
      for (int j = 0; j < kUnit / kLoad; ++j) {
        int32_t v[kLoad];
        const uint32_t from = t_lane + buf * (uint32_t)kRows + (uint32_t)(set * kUnit + kLoad * j);
        tmem_ld16(from, v);
        if constexpr (kLoad == 32) { tmem_ld16(from + 16u, v + 16); tmem_wait16(v + 16); }
        tmem_wait16(v);
        if (j + 1 == kUnit / kLoad) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(S.dempty + 8u * buf);
        }
        if (x_groups) {
#pragma unroll
          for (int i = 0; i < kLoad / 4; ++i) {
            const float4 f = lds_f4(my_scales + (uint32_t)(4 * kLoad * j + 16 * i));
            float *to = acc + kLoad * j + 4 * i;
            to[0] = fmaf(__int_as_float(v[4 * i]) * f.x, s, to[0]);
            to[1] = fmaf(__int_as_float(v[4 * i + 1]) * f.y, s, to[1]);
            to[2] = fmaf(__int_as_float(v[4 * i + 2]) * f.z, s, to[2]);
            to[3] = fmaf(__int_as_float(v[4 * i + 3]) * f.w, s, to[3]);
          }
        } else {
#pragma unroll
          for (int i = 0; i < kLoad; ++i) acc[kLoad * j + i] = fmaf(__int_as_float(v[i]), s, acc[kLoad * j + i]);
        }
      }
      buf ^= 1u;
      if (buf == 0u) parity ^= 1u;
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
}

__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

template <int kType, int kRows>
__global__ void __launch_bounds__(Shape<kRows>::kThreads, 1)
w4_tc_kernel(const __grid_constant__ TcParams P) {
  using Sh = Shape<kRows>;
  using T = typename RowsOf<kType>::T;
  extern __shared__ __align__(1024) uint8_t smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const Smem S = carve(smem, Sh::kScaleBytes);
  if (threadIdx.x == 0) {
    // a stage is full with four expanding warps' arrivals and those that bring the rows
    for (int i = 0; i < Sh::kStages; ++i) { mbar_init(S.full + 8u * i, 4 + (P.copies ? 1 : kLoadWarps)); mbar_init(S.empty + 8u * i, 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(S.dfull + 8u * i, 1); mbar_init(S.dempty + 8u * i, 4 * Sh::kPromo); }
    *S.abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == Sh::kMmaWarp) {
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
  if (warp < 4 * Sh::kPromo) {
    if constexpr (Sh::kPromoRegs != Sh::kRegs) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(Sh::kPromoRegs));
    promote_role<kRows>(P, S, span, first, step, total, warp >> 2, warp & 3, lane, tmem);
  } else {
    if constexpr (Sh::kOtherRegs != Sh::kRegs) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(Sh::kOtherRegs));
    if (warp < Sh::kMmaWarp) {
      expand_role<T, kRows>(P, S, span, first, step, total, (warp >> 2) - Sh::kPromo, warp & 3, lane, tmem);
    } else if (warp == Sh::kMmaWarp) {
      if (elect_one()) mma_loop<kRows>(P, S, span, mine, tmem);
    } else if (!P.copies) {
      load_role<kType, kRows>(P, S, span, first, step, total, warp - Sh::kLoadWarp, lane);
    } else if (warp == Sh::kLoadWarp) {
      if (elect_one()) copy_role<kRows>(P, S, span, first, step, total);
    }
    __syncwarp();
  }
  tc_fence_before();
  __syncthreads();
  if (warp == Sh::kMmaWarp)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
  if (P.split == 1) return;
  // a cluster has one tile; its blocks write shares of the rows, each the sums of all in the same order
  cluster_barrier();
  const int n0 = (first % P.row_tiles) * kTileN;
  const long long tok0 = (long long)(first / P.row_tiles) * kRows;
  const bool row_scale = P.A.x_scales != nullptr && P.A.r.x_group == 0;
  const int r0 = kRows * rank / P.split, r1 = kRows * (rank + 1) / P.split;
  for (int e = r0 * kTileN + threadIdx.x; e < r1 * kTileN; e += Sh::kThreads) {
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

// The driver's function that makes tensor maps, looked up once (no library is linked for it).
using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                 const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiled encode_tiled() {
  static std::atomic<EncodeTiled> known{nullptr};
  EncodeTiled f = known.load(std::memory_order_relaxed);
  if (f == nullptr) {
    void *p = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) == cudaSuccess &&
        found == cudaDriverEntryPointSuccess) {
      f = (EncodeTiled)p;
      known.store(f, std::memory_order_relaxed);
    } else {
      (void)cudaGetLastError();
    }
  }
  return f;
}

// Whether the rows can be copied as they are, and their map.
template <int kType>
bool map_rows(const W4Args &a, int rows, CUtensorMap *map) {
  if (RowsOf<kType>::kBytes != 2 || !rows_in_pieces(a.x, a.r.x_stride, 8, 2) || a.r.x_stride < a.d.K) return false;
  const EncodeTiled encode = encode_tiled();
  if (encode == nullptr) return false;
  const cuuint64_t size[2] = {(cuuint64_t)a.d.K, (cuuint64_t)a.r.rows}, stride[1] = {(cuuint64_t)a.r.x_stride * 2};
  const cuuint32_t box[2] = {kChunk, (cuuint32_t)rows}, each[2] = {1, 1};
  return encode(map, kType == XNOR_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2,
                const_cast<void *>(a.x), size, stride, box, each, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
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
  P.copies = map_rows<kType>(a, kRows, &P.x_map);
  P.A = a;
  P.col_tiles = w4_col_tiles(a.d);
  P.row_tiles = (a.d.N + kTileN - 1) / kTileN;
  P.token_tiles = (a.r.rows + kRows - 1) / kRows;
  P.pieces = rows_in_pieces(a.x, a.r.x_stride, 8, RowsOf<kType>::kBytes);
  const int total = P.row_tiles * P.token_tiles, sms = sm_count_of_current_device();
  // blocks divide the columns while that still adds SMs and each keeps four blocks of 128 columns
  P.split = 1;
  while (P.split < kMaxSplitTc && 2 * P.split * total <= sms && P.col_tiles >= 16 * P.split) P.split *= 2;
  // instruction descriptor: D fp32, A and B bf16 or f16, both K-major, M = 128
  const uint32_t format = kType == XNOR_BF16 ? 1u : 0u;
  P.idesc = (1u << 4) | (format << 7) | (format << 10) | ((uint32_t)(kRows >> 3) << 17) | ((uint32_t)(kTileN >> 4) << 24);
  const unsigned grid = P.split > 1 ? (unsigned)(total * P.split) : (unsigned)std::min(total, sms);
  return launch_kernel(w4_tc_kernel<kType, kRows>, dim3(grid), Sh::kThreads, Sh::kSmem, st, (unsigned)P.split, P);
}

template <int kType>
cudaError_t run_type(const W4Args &a, cudaStream_t st) {
  const long long tiles = (a.d.N + kTileN - 1) / kTileN * ((a.r.rows + 191ll) / 192);
  if (a.r.rows > 128 && 2 * tiles > sm_count_of_current_device()) return run<kType, 192>(a, st);
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
