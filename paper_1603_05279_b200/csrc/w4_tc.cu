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
// have two buffers in tensor memory (four up to 64 rows), so that the tensor core fills one while another is drained.  Warps:
//   promotion  8 (4 up to 64 rows): a thread holds the sums of one output and up to 96 rows of x
//   expansion  8: a thread expands one weight row, 64 columns at a time, from shared straight into tensor memory
//   one issues the products, one copies the packed weights into a deep ring in shared memory (bulk copies), one the
//   rows of x, by tensor copies, into the stages of 64 columns that the products read; rows that cannot be copied as
//   they are, in 8 bits above all, come through the registers of six warps instead
// Where the tiles are too few for the GPU, the blocks of a cluster divide the columns, and add their sums through
// each other's shared memory in a fixed order.  Every wait is bounded; on expiry the block records
// XNOR_ERR_TIMEOUT, stops and frees its tensor memory.
#include <cuda.h>

#include <algorithm>
#include <climits>
#include <atomic>

#include "umma_common.cuh"
#include "w4.cuh"

namespace xnor {

__device__ int g_status_w4 = 0;

namespace {

using namespace umma;

constexpr int kTileN = 128;                  // outputs (weight rows) of a tile: the lanes of tensor memory
constexpr int kChunk = 64;                   // columns of a stage
constexpr int kACols = kChunk / 2;           // tensor-memory columns of a chunk of expanded weights
constexpr int kMaxStages = 8, kWeightStages = 8, kMaxBufs = 4;
constexpr uint32_t kWeightChunk = 4096;      // a chunk of packed weights: 8 tiles of 16 x 64
constexpr uint32_t kWeightStage = 2 * kWeightChunk;            // chunks of two expanding sets
constexpr uint32_t kCtrlBytes = 1024;
constexpr int kMaxSplitTc = 8;
constexpr int kAhead = 8;                    // groups whose scales are under way

template <int kRows, bool kCopies>           // kCopies: the rows come by tensor copies
struct Shape {
  static constexpr int kPromo = kRows > 64 ? 2 : 1;            // sets of four warps
  static constexpr int kUnit = kRows / kPromo;                 // rows of x of a set
  static constexpr int kExpand = kRows > 64 ? 2 : 4;           // sets of four warps
  static constexpr int kOther = kCopies ? 4 : 8, kLoadWarps = kOther - 2;
  static constexpr int kMmaWarp = 4 * (kPromo + kExpand), kWeightWarp = kMmaWarp + 1, kLoadWarp = kMmaWarp + 2;
  static constexpr int kThreads = 32 * (kMmaWarp + kOther);
  static constexpr int kBufs = kRows > 64 ? 2 : 4;             // accumulators
  static constexpr int kATmem = kRows > 128 ? 2 * kRows : 256; // behind them
  static constexpr int kStages = (512 - kATmem) / kACols;      // chunks: weights in tensor memory, rows of x in shared
  static constexpr uint32_t kStage = kRows * kChunk * 2;       // a row of x: 128 bytes, swizzled
  static constexpr uint32_t kScaleBytes = 8 * (512 + kAhead * 128);          // per promotion warp: a group's scales of x, its outputs' of groups ahead
  static constexpr size_t kSmem = 1024 + kCtrlBytes + kScaleBytes + kWeightStages * kWeightStage + (size_t)kStages * kStage;   // (1024: to align the ring)
  // Registers per thread as launched, and after they are dealt out anew: the promotion's hold its sums.
  static constexpr int kRegs = kThreads == 640 ? 96 : kThreads == 768 ? 80 : 72;
  static constexpr int kPromoRegs = kRows > 128 ? 144 : kRows > 64 ? (kCopies ? 128 : 112) : kRows > 32 ? (kCopies ? 128 : 112) : 120;
  static constexpr int kOtherRegs = kRows > 128 ? 64 : kRows > 64 ? (kCopies ? 72 : 64) : kCopies ? (kRows > 32 ? 64 : 72) : 64;
  static_assert(kPromo * 128 * kPromoRegs + (kThreads - kPromo * 128) * kOtherRegs <= kThreads * kRegs, "registers");
  static_assert(kSmem <= 232448 && kStages <= kMaxStages && (kStages & (kStages - 1)) == 0, "shared and tensor memory");
  static_assert((size_t)kStages * kStage >= (size_t)kRows * kTileN * 4 || kRows > 128, "room for the sums of a block");
};

struct TcParams {
  CUtensorMap x_map;                        // the rows of x, 64 columns x kRows rows at a time
  W4Args A;
  int col_tiles, row_tiles, token_tiles;    // chunks of columns; tiles of 128 outputs, of kRows rows
  int split, pieces;                        // pieces: rows in 8 bits can be read in pieces of eight
  uint32_t idesc, magic;                    // magic: W4Type's
};

struct Smem {
  uint32_t full, empty, wfull, wempty, dfull, dempty, scales, weights, ring;
  uint32_t *tmem_slot;
  volatile int *abort_flag;
};
__device__ __forceinline__ Smem carve(uint8_t *smem, uint32_t scale_bytes) {
  Smem s;
  s.full = smem_u32(smem);
  s.empty = s.full + 8 * kMaxStages;
  s.wfull = s.empty + 8 * kMaxStages;
  s.wempty = s.wfull + 8 * kWeightStages;
  s.dfull = s.wempty + 8 * kWeightStages;
  s.dempty = s.dfull + 8 * kMaxBufs;
  s.tmem_slot = reinterpret_cast<uint32_t *>(smem + 16 * (kMaxStages + kWeightStages + kMaxBufs));
  s.abort_flag = reinterpret_cast<volatile int *>(s.tmem_slot + 1);
  s.scales = s.full + kCtrlBytes;
  s.weights = s.scales + scale_bytes;
  s.ring = (s.weights + kWeightStages * kWeightStage + 1023u) & ~1023u;
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

// Every tile starts with stage 0 and accumulator 0, so that the issuing thread's addresses are constants.  `base` has
// the parities of the stages' next uses, and changes from tile to tile with those that were used an odd number of times.
template <int kStages>
struct Parities {
  uint32_t base = 0u, flip = 0u;
  __device__ __forceinline__ explicit Parities(int chunks) {
#pragma unroll
    for (int s = 0; s < kStages; ++s) flip |= (uint32_t)(((chunks - s + kStages - 1) / kStages) & 1) << s;      // (chunks > 0)
  }
  __device__ __forceinline__ uint32_t of(int i) const { return ((base >> (i % kStages)) ^ (uint32_t)(i / kStages)) & 1u; }
  __device__ __forceinline__ void next_tile() { base ^= flip; }
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

// ------------------------------------------------------------------ the issuing thread
// Operand of the rows of x: 128-byte rows, swizzled in groups of eight (1024 bytes); 16 columns are 32 bytes on.
__device__ __forceinline__ uint64_t swizzled_desc(uint32_t addr) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | (1ull << 16) | ((uint64_t)(1024u >> 4) << 32) | (1ull << 46) | (2ull << 61);
}

// One lap over the stages is straight-line code.
template <class Sh, int kRows, int kGroup>
__device__ __forceinline__ void mma_loop(const TcParams &P, const Smem &S, const Span &span, int tiles, uint32_t tmem) {
  const uint32_t idesc = P.idesc;
  const uint64_t desc0 = swizzled_desc(S.ring);
  const int n = span.c1 - span.c0, units = span.u1 - span.u0;
  Parities<Sh::kStages> par(n);
  uint32_t dpar = (1u << Sh::kBufs) - 1u;          // the accumulators: drained at first
  auto drained = [&](int buf) {
    const bool ok = wait(S, S.dempty + 8u * buf, (dpar >> buf) & 1u);
    dpar ^= 1u << buf;
    tc_fence_after();
    return ok;
  };
  // `count` products of 16 columns from column 16 `from` of stage s
  auto products = [&](int s, int buf, int from, int count, uint32_t accumulate) {
#pragma unroll
    for (int i = 0; i < count; ++i)
      mma_tmem(tmem + (uint32_t)(buf * kRows), tmem + (uint32_t)(Sh::kATmem + s * kACols + 8 * (from + i)),
               desc0 + (uint64_t)((uint32_t)s * (Sh::kStage >> 4) + 2u * (uint32_t)(from + i)), idesc, i > 0 ? 1u : accumulate);
  };
  for (int tile = 0; tile < tiles; ++tile, par.next_tile()) {
#pragma unroll 1
    for (int c = 0; c < n; c += Sh::kStages) {
#pragma unroll
      for (int s = 0; s < Sh::kStages; ++s) {
        if (c + s < n) {
          const int buf = (kGroup == 128 ? s / 2 : kGroup == 64 ? s : 2 * s) % Sh::kBufs;
          if ((kGroup != 128 || s % 2 == 0) && !drained(buf)) return;
          if (!wait(S, S.full + 8u * s, par.of(c + s))) return;
          tc_fence_after();
          if constexpr (kGroup == 32) {
            products(s, buf, 0, 2, 0u);
            umma_commit(S.dfull + 8u * buf);
            if (2 * (c + s) + 1 < units) {
              if (!drained(buf + 1)) return;
              products(s, buf + 1, 2, 2, 0u);
              umma_commit(S.dfull + 8u * (buf + 1));
            }
          } else {
            products(s, buf, 0, 4, kGroup == 128 && s % 2 == 1 ? 1u : 0u);
            if (kGroup == 64 || s % 2 == 1 || c + s + 1 == n) umma_commit(S.dfull + 8u * buf);
          }
          umma_commit(S.empty + 8u * s);
        }
      }
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

// Set `which` takes every kExpand-th chunk of a tile.  A thread expands one weight row: the eight words of a chunk.
template <class Sh, class T>
__device__ __forceinline__ void expand_role(const TcParams &P, const Smem &S, const Span &span, int first, int step, int total, int which,
                                            int quarter, int lane, uint32_t tmem) {
  constexpr int kSets = Sh::kExpand;
  const int N = P.A.d.N, group = P.A.d.group, r = 32 * quarter + lane, n = span.c1 - span.c0;
  const int last_group = (P.A.d.K - 1) / group;
  const uint32_t t_lane = tmem + ((uint32_t)(32 * quarter) << 16) + (uint32_t)Sh::kATmem;
  uint32_t from[4];                                 // this row's words of columns 8 t .. and 32 + 8 t ..
#pragma unroll
  for (int t = 0; t < 4; ++t) from[t] = S.weights + (uint32_t)(which & 1) * kWeightChunk + (uint32_t)((r / kW4Rows) * 512 + w4_place(r, 8 * t) * 16 + 4 * w4_word(r, 0));
  Parities<Sh::kStages> par(n);
  uint32_t seq = 0;                                 // pairs of chunks of all tiles in sequence: their places in the ring of weights
  for (int tile = first; tile < total; tile += step, seq += (uint32_t)(n + 1) / 2u, par.next_tile()) {
    const int nc = min((tile % P.row_tiles) * kTileN + r, N - 1);
    struct Zeros { uint32_t z[2]; };
    auto fetch = [&](int i, Zeros &f) {
      f.z[0] = f.z[1] = 8u;
      if (P.A.zeros && i < n) {
        const int c = span.c0 + i;
        f.z[0] = load_global(P.A.zeros + (size_t)min(c * kChunk / group, last_group) * N + nc);
        f.z[1] = group == 32 ? load_global(P.A.zeros + (size_t)min(2 * c + 1, last_group) * N + nc) : f.z[0];
        // (these come from memory: fetched into the L2 well ahead)
        asm volatile("prefetch.global.L2 [%0];" ::"l"(__cvta_generic_to_global(P.A.zeros + (size_t)min((c + 16) * kChunk / group, last_group) * N + nc)));
      }
    };
    auto expand = [&](int i, const Zeros &f) {
      const uint32_t pair = seq + (uint32_t)i / 2u, slot = pair % kWeightStages, use = pair / kWeightStages, s = (uint32_t)i % Sh::kStages;
      if (!wait_warp(S, S.wfull + 8u * slot, use & 1u)) return false;
      uint32_t w[8];
#pragma unroll
      for (int t = 0; t < 4; ++t) lds64(from[t] + slot * kWeightStage, w[t], w[4 + t]);
      __syncwarp();
      if (lane == 0) mbar_arrive(S.wempty + 8u * slot);
      if (i >= n) return true;                      // the last pair lacks this set's chunk
      if (!wait_warp(S, S.empty + 8u * s, par.of(i) ^ 1u)) return false;
      tc_fence_after();
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const typename W4Type<T>::Zero zero = W4Type<T>::zero(f.z[half]);
        uint32_t v[16];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          uint32_t e[4];
          W4Type<T>::expand(w[4 * half + t], zero, P.magic, e);
#pragma unroll
          for (int p = 0; p < 4; ++p) v[4 * t + p] = e[p];
        }
        tmem_st16(t_lane + s * kACols + 16u * half, v);
      }
      asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(S.full + 8u * s);
      return true;
    };
    Zeros f0, f1;                                   // (two by name: moving one to the other would wait for its loads)
    fetch(which, f0);
    fetch(which + kSets, f1);
#pragma unroll 1
    for (int i = which; i < ((n + 1) & ~1); i += 2 * kSets) {
      if (!expand(i, f0)) return;
      fetch(i + 2 * kSets, f0);
      if (i + kSets >= ((n + 1) & ~1)) break;
      if (!expand(i + kSets, f1)) return;
      fetch(i + 3 * kSets, f1);
    }
  }
}

// One thread copies the packed weights, two chunks of 128 rows at a time (one at a time it took longer than the
// rest at few rows of x: 32 rows times 16384x16384 69.9 us).
__device__ __forceinline__ void weight_role(const TcParams &P, const Smem &S, const Span &span, int first, int step, int total) {
  uint32_t slot = 0u, parity = 1u, started = 0u;
  for (int tile = first; tile < total; tile += step) {
    const uint8_t *w = reinterpret_cast<const uint8_t *>(P.A.w) + ((size_t)(tile % P.row_tiles) * P.col_tiles + span.c0) * kWeightChunk;
    uint32_t left = (uint32_t)(span.c1 - span.c0) * kWeightChunk;
#pragma unroll 1
    for (; left > 0u; ++started) {
      const uint32_t bytes = min(left, kWeightStage), bar = S.wfull + 8u * slot;
      if (!wait(S, S.wempty + 8u * slot, parity)) {
        // gave up: the copies in flight must land before the block's shared memory is released
        for (uint32_t u = started > kWeightStages ? started - kWeightStages : 0u; u < started; ++u)
          for (int i = 0; i < (1 << 12) && !mbar_try(S.wfull + 8u * (u % kWeightStages), (u / kWeightStages) & 1u); ++i) {}
        return;
      }
      mbar_arrive_expect_tx(bar, bytes);
      bulk_copy_g2s(S.weights + slot * kWeightStage, w, bytes, bar);
      w += bytes;
      left -= bytes;
      if (++slot == kWeightStages) { slot = 0u; parity ^= 1u; }
    }
  }
}

// ------------------------------------------------------------------ the rows of x
// One thread copies a stage with one tensor copy, which also fills what does not exist with zeros.
template <class Sh, int kRows>
__device__ __forceinline__ void copy_role(const TcParams &P, const Smem &S, const Span &span, int first, int step, int total) {
  const int n = span.c1 - span.c0;
  Parities<Sh::kStages> par(n);
  for (int tile = first; tile < total; tile += step, par.next_tile()) {
    const int tok0 = (tile / P.row_tiles) * kRows;
#pragma unroll 1
    for (int i = 0; i < n; ++i) {
      const uint32_t s = (uint32_t)i % Sh::kStages;
      if (!wait(S, S.empty + 8u * s, par.of(i) ^ 1u)) {
        // gave up: what is in flight lands within microseconds; the block's shared memory is not released before
        const long long t0 = clock64();
        while (clock64() - t0 < (1 << 20)) {}
        return;
      }
      const uint32_t bar = S.full + 8u * s;
      mbar_arrive_expect_tx(bar, Sh::kStage);
      asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                   ::"r"(S.ring + s * Sh::kStage), "l"(&P.x_map), "r"((span.c0 + i) * kChunk), "r"(tok0), "r"(bar) : "memory");
    }
  }
}

// A stage that is filled through registers: free, and filled by this warp.
template <class Sh>
__device__ __forceinline__ bool start_rows(const Smem &S, const Parities<Sh::kStages> &par, int i) {
  return wait_warp(S, S.empty + 8u * (i % Sh::kStages), par.of(i) ^ 1u);
}
template <class Sh>
__device__ __forceinline__ void finish_rows(const Smem &S, int i, int lane) {
  fence_proxy_async();
  __syncwarp();
  if (lane == 0) mbar_arrive(S.full + 8u * (i % Sh::kStages));
}

// Through registers: rows in 8 bits become 16-bit numbers.  The warps share every stage; a thread has eight columns of
// every (4 kLoadWarps)-th row, and where it can it loads them a chunk ahead.
template <class Sh, int kType, int kRows>
__device__ __forceinline__ void load_role(const TcParams &P, const Smem &S, const Span &span, int first, int step, int total, int w, int lane) {
  constexpr int kStep = 4 * Sh::kLoadWarps, kPass = (kRows + kStep - 1) / kStep;
  static_assert(RowsOf<kType>::kBytes == 1 && kPass <= 6, "a batch is a stage");
  const int K = P.A.d.K, n = span.c1 - span.c0, piece = lane & 7, row0 = 4 * w + (lane >> 3);
  const long long row_bytes = P.A.r.x_stride;
  Parities<Sh::kStages> par(n);
  for (int tile = first; tile < total; tile += step, par.next_tile()) {
    const long long tok0 = (long long)(tile / P.row_tiles) * kRows;
    const int rows = (int)min((long long)kRows, P.A.r.rows - tok0);
    const uint8_t *x = static_cast<const uint8_t *>(P.A.x) + tok0 * row_bytes;
    // (a row that does not exist is its last one's: no output reads it)
    struct Batch { uint32_t v[kPass][2]; };
    auto whole = [&](int i) { return (span.c0 + i + 1) * kChunk <= K; };
    auto load = [&](int i, Batch &b) {               // of a whole chunk: nothing but loads
      if (i >= n || !whole(i)) return;
      const uint8_t *from = x + ((span.c0 + i) * kChunk + 8 * piece);
#pragma unroll
      for (int p = 0; p < kPass; ++p)
        load_x8_raw<kType>(from + (long long)min(row0 + kStep * p, rows - 1) * row_bytes, 0, INT_MAX, true, b.v[p]);
    };
    auto put = [&](int i, int row, const uint32_t (&raw)[2]) {
      uint32_t v[4];
      x8_pairs<kType>(raw, v);
      if (row < kRows)
        sts128(S.ring + ((uint32_t)i % Sh::kStages) * Sh::kStage + (uint32_t)row * 128u + (uint32_t)((piece ^ (row & 7)) * 16), v[0], v[1], v[2], v[3]);
    };
    auto store = [&](int i, const Batch &b) {
      if (whole(i)) {
#pragma unroll
        for (int p = 0; p < kPass; ++p) put(i, row0 + kStep * p, b.v[p]);
      } else {
#pragma unroll 1
        for (int p = 0; p < kPass; ++p) {
          uint32_t raw[2];
          const int row = row0 + kStep * p;
          load_x8_raw<kType>(x + (long long)min(row, rows - 1) * row_bytes, (span.c0 + i) * kChunk + 8 * piece, K, true, raw);
          put(i, row, raw);
        }
      }
    };
    Batch b0, b1;
    load(0, b0);
    load(1, b1);
#pragma unroll 1
    for (int i = 0; i < n; i += 2) {
      if (!start_rows<Sh>(S, par, i)) return;
      store(i, b0);
      finish_rows<Sh>(S, i, lane);
      load(i + 2, b0);
      if (i + 1 >= n) break;
      if (!start_rows<Sh>(S, par, i + 1)) return;
      store(i + 1, b1);
      finish_rows<Sh>(S, i + 1, lane);
      load(i + 3, b1);
    }
  }
}

// Through registers from any address, as rows of an odd number of columns have them: a thread loads one aligned word of
// four bytes per row, so that a warp reads a chunk of one row (two in 8 bits) at once, and takes the bytes that belong to
// its neighbour's word from there; what lies behind the warp's words, a thread per row loads.  2048 bf16
// rows times 4096x4095: 537 us, 2035 value by value; tensor copies take 73 for 4096x4096.  Bound by the loads' latency:
// more than twelve rows of a warp under way at once do not fit the registers and spill (593 us).
template <class Sh, int kType, int kRows>
__device__ __forceinline__ void word_role(const TcParams &P, const Smem &S, const Span &span, int first, int step, int total, int w, int lane) {
  constexpr int kB = RowsOf<kType>::kBytes, kWords = kChunk * kB / 4, kAtOnce = 32 / kWords, kStep = kAtOnce * Sh::kLoadWarps;
  constexpr int kPass = (kRows + kStep - 1) / kStep, kParts = kPass > 6 ? 2 * ((kPass + 11) / 12) : 1, kBatch = (kPass + kParts - 1) / kParts;
  static_assert(kBatch * kAtOnce <= 32, "a thread for what lies behind each row");
  const int K = P.A.d.K, n = span.c1 - span.c0, word = lane % kWords, row0 = kAtOnce * w + lane / kWords;
  const int behind = kAtOnce * w + lane % kAtOnce + kStep * (lane / kAtOnce);       // the row whose next word this thread loads
  const long long row_bytes = P.A.r.x_stride * kB;
  const uint8_t *end = static_cast<const uint8_t *>(P.A.x) + (P.A.r.rows - 1) * row_bytes + (size_t)K * kB;
  uint32_t tail = 0u;                                // what exists of the word in which the rows end
  for (int i = 0; i < (int)((uintptr_t)end & 3u); ++i)
    tail |= (uint32_t)load_global(reinterpret_cast<const uint8_t *>((uintptr_t)end & ~(uintptr_t)3) + i) << (8 * i);
  Parities<Sh::kStages> par(n);
  for (int tile = first; tile < total; tile += step, par.next_tile()) {
    const long long tok0 = (long long)(tile / P.row_tiles) * kRows;
    const int rows = (int)min((long long)kRows, P.A.r.rows - tok0);
    const uint8_t *x = static_cast<const uint8_t *>(P.A.x) + tok0 * row_bytes;
    struct Batch { uint32_t v[kBatch], next; };
    // Chunks that end a word and more before a row's last byte: no word can lie behind the rows.
    auto inner = [&](int i) { return (span.c0 + i + 1) * kChunk * kB + 8 <= K * kB; };
    // (a row that does not exist is its last one's: no output reads it)
    auto place = [&](int i, int row, int at) {
      return (uintptr_t)(x + (size_t)(span.c0 + i) * (kChunk * kB) + 4 * at + (long long)min(row, rows - 1) * row_bytes) & ~(uintptr_t)3;
    };
    auto load = [&](int i, int part, Batch &b) {     // of an inner chunk: nothing but loads
      if (i >= n || !inner(i)) return;
      int r0 = row0 + kStep * kBatch * part;
      asm volatile("" : "+r"(r0));                   // (the addresses of all rows at once do not fit the registers)
#pragma unroll
      for (int p = 0; p < kBatch; ++p) b.v[p] = load_global(reinterpret_cast<const uint32_t *>(place(i, r0 + kStep * p, word)));
      b.next = load_global(reinterpret_cast<const uint32_t *>(place(i, behind + kStep * kBatch * part, kWords)));
    };
    const uint32_t low = 8u * (uint32_t)(uintptr_t)x, step8 = 8u * (uint32_t)row_bytes;
    auto put = [&](int i, int row, uint32_t mine, uint32_t other, uint32_t mask) {
      const uint32_t v = __funnelshift_r(mine, other, low + (uint32_t)row * step8) & mask;      // (by the address's bits modulo 32)
      const uint32_t to = S.ring + ((uint32_t)i % Sh::kStages) * Sh::kStage + (uint32_t)row * 128u;
      // (predicates, not branches: the shuffles of the next row would wait for the warp to join)
      if constexpr (kB == 2)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.lt.s32 p, %0, %1;\n\t@p st.shared.b32 [%2], %3;\n\t}"
                     ::"r"(row), "n"(kRows), "r"(to + (uint32_t)(((word >> 2) ^ (row & 7)) * 16 + (word & 3) * 4)), "r"(v) : "memory");
      else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.lt.s32 p, %0, %1;\n\t@p st.shared.v2.b32 [%2], {%3, %4};\n\t}"
                     ::"r"(row), "n"(kRows), "r"(to + (uint32_t)(((word >> 1) ^ (row & 7)) * 16 + (word & 1) * 8)),
                     "r"(x_pair<kType>(v, 0)), "r"(x_pair<kType>(v, 1)) : "memory");
    };
    auto store = [&](int i, int part, const Batch &b) {
      int r0 = row0 + kStep * kBatch * part;
      asm volatile("" : "+r"(r0));
      if (inner(i)) {
#pragma unroll
        for (int p = 0; p < kBatch; ++p) {
          const uint32_t other = __shfl_down_sync(0xFFFFFFFFu, b.v[p], 1), last = __shfl_sync(0xFFFFFFFFu, b.next, kAtOnce * p + lane / kWords);
          put(i, r0 + kStep * p, b.v[p], word == kWords - 1 ? last : other, 0xFFFFFFFFu);
        }
        return;
      }
      const int left = (K - (span.c0 + i) * kChunk) * kB - 4 * word;                 // bytes of this word that exist
      const uint32_t mask = left >= 4 ? 0xFFFFFFFFu : left <= 0 ? 0u : (1u << (8 * left)) - 1u;
      auto read = [&](uintptr_t p) {
        return p + 4u <= (uintptr_t)end ? load_global(reinterpret_cast<const uint32_t *>(p)) : p < (uintptr_t)end ? tail : 0u;
      };
#pragma unroll 1
      for (int p0 = 0; p0 < kBatch; p0 += 2, r0 += 2 * kStep) {
        uint32_t mine[2], other[2];
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          mine[p] = read(place(i, r0 + kStep * p, word));
          other[p] = read(place(i, r0 + kStep * p, word + 1));
        }
#pragma unroll
        for (int p = 0; p < 2; ++p)
          if (p0 + p < kBatch) put(i, r0 + kStep * p, mine[p], other[p], mask);
      }
    };
    Batch b0, b1;
    load(0, 0, b0);
    load(kParts == 1 ? 1 : 0, kParts == 1 ? 0 : 1, b1);
#pragma unroll 1
    for (int i = 0; i < n; i += kParts == 1 ? 2 : 1) {
      if (!start_rows<Sh>(S, par, i)) return;
      if constexpr (kParts == 1) {
        store(i, 0, b0);
        finish_rows<Sh>(S, i, lane);
        load(i + 2, 0, b0);
        if (i + 1 >= n) break;
        if (!start_rows<Sh>(S, par, i + 1)) return;
        store(i + 1, 0, b1);
        finish_rows<Sh>(S, i + 1, lane);
        load(i + 3, 0, b1);
      } else {
#pragma unroll
        for (int q = 0; q < kParts; q += 2) {
          const bool last = q + 2 == kParts;
          store(i, q, b0);
          load(last ? i + 1 : i, last ? 0 : q + 2, b0);
          store(i, q + 1, b1);
          if (last) finish_rows<Sh>(S, i, lane);
          load(last ? i + 1 : i, last ? 1 : q + 3, b1);
        }
      }
    }
  }
}

// ------------------------------------------------------------------ promotion: sums of groups -> sums of a row
__device__ __forceinline__ void convert(float v, float *p) { *p = v; }
__device__ __forceinline__ void convert(float v, __nv_bfloat16 *p) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ void convert(float v, __half *p) { *p = __float2half_rn(v); }

// The sums of one output and kUnit rows of x, `left` of which exist: a warp stores 32 neighbouring outputs of a row.
template <int kUnit, class Out>
__device__ __forceinline__ void store_column(const float (&acc)[kUnit], Out *p, long long stride, int left) {
  if (left >= kUnit) {
#pragma unroll
    for (int i = 0; i < kUnit; ++i, p += stride) convert(acc[i], p);
  } else {
#pragma unroll
    for (int i = 0; i < kUnit; ++i, p += stride)
      if (i < left) convert(acc[i], p);
  }
}

// Four neighbouring outputs, `left` of which exist.
template <class Out>
__device__ __forceinline__ void store_four(const float4 &v, Out *p, int left) {
  convert(v.x, p);
  if (left > 1) convert(v.y, p + 1);
  if (left > 2) convert(v.z, p + 2);
  if (left > 3) convert(v.w, p + 3);
}

__device__ __forceinline__ float4 lds_f4(uint32_t addr) {
  uint32_t v[4];
  lds128(addr, v);
  return make_float4(__uint_as_float(v[0]), __uint_as_float(v[1]), __uint_as_float(v[2]), __uint_as_float(v[3]));
}

template <class Sh, int kRows>
__device__ __forceinline__ void promote_role(const TcParams &P, const Smem &S, const Span &span, int first, int step, int total, int set, int quarter,
                             int lane, uint32_t tmem) {
  constexpr int kUnit = Sh::kUnit;
  const W4Args &A = P.A;
  const int N = A.d.N;
  const bool x_groups = A.x_scales != nullptr && A.r.x_group != 0;
  const int G = (A.d.K + A.d.group - 1) / A.d.group;
  const uint32_t t_lane = tmem + ((uint32_t)(32 * quarter) << 16);
  const uint32_t my_scales = S.scales + (uint32_t)(4 * set + quarter) * (512u + kAhead * 128u), my_ring = my_scales + 512u + 4u * lane;
  // Few rows of x take few instructions per group, and its scales come from memory: eight groups are under way then
  // (32 rows times 16384x16384 69.9 -> 56.2 us, with four expanding sets).  Many rows have the time of one group's
  // products for a load from the L2, and no slots to spare (2048 rows times 8192x8192 234 us, 240 with the ring).
  constexpr bool kRing = kRows <= 64;
  // Two groups at a time where their sums fit the registers: a group's waits and loads follow each other.
  constexpr int kPair = kRows <= 32 ? 2 : 1;
  // A group's scale of this output, into its place of the ring; a copy or none, so that the copies count the groups
  auto ahead = [&](int u, int nc) {
    if (u < span.u1)
      asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(my_ring + 128u * ((uint32_t)u % kAhead)),
                   "l"(__cvta_generic_to_global(A.scales + (size_t)u * N + nc)) : "memory");
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  uint32_t dpar = 0u;                               // the accumulators' parities
  for (int tile = first; tile < total; tile += step) {
    const int n = (tile % P.row_tiles) * kTileN + 32 * quarter + lane, nc = min(n, N - 1);
    const long long tok0 = (long long)(tile / P.row_tiles) * kRows + set * kUnit;
    float acc[kUnit];
#pragma unroll
    for (int i = 0; i < kUnit; ++i) acc[i] = 0.0f;
    float next = 0.0f;
    if constexpr (kRing) {
#pragma unroll
      for (int i = 0; i < kAhead - kPair; ++i) ahead(span.u0 + i, nc);
    } else {
      if (span.u0 < span.u1) next = load_global(A.scales + (size_t)span.u0 * N + nc);
    }
#pragma unroll 1
    for (int u = span.u0; u < span.u1; u += kPair) {
      float s[kPair];
      s[0] = next;
      if constexpr (kRing) {
#pragma unroll
        for (int h = 0; h < kPair; ++h) ahead(u + kAhead - kPair + h, nc);
        asm volatile("cp.async.wait_group %0;" ::"n"(kAhead - kPair) : "memory");
#pragma unroll
        for (int h = 0; h < kPair; ++h) s[h] = __uint_as_float(lds32(my_ring + 128u * ((uint32_t)(u + h) % kAhead)));  // (each lane reads what it copied)
      } else {
        if (u + 1 < span.u1) next = load_global(A.scales + (size_t)(u + 1) * N + nc);
      }
      const int count = kPair == 1 ? 1 : min(kPair, span.u1 - u);
      if (x_groups) {
        __syncwarp();
#pragma unroll
        for (int i = 0; i < (kPair * kUnit + 31) / 32; ++i) {
          const int at = lane + 32 * i, col = at % kUnit, h = at / kUnit;
          const float v = h < count && tok0 + col < A.r.rows ? load_global(A.x_scales + (tok0 + col) * G + u + h) : 0.0f;
          if (h < kPair) sts32(my_scales + 4u * at, __float_as_uint(v));
        }
        __syncwarp();
      }
      const uint32_t buf = (uint32_t)(u - span.u0) % Sh::kBufs;
      bool ok = true;
#pragma unroll
      for (int h = 0; h < kPair; ++h)
        if (h < count) {
          ok = ok && wait_inline(S, S.dfull + 8u * (buf + h), (dpar >> (buf + h)) & 1u);
          dpar ^= 1u << (buf + h);
        }
      if (!__all_sync(0xFFFFFFFFu, ok)) {
        asm volatile("cp.async.wait_all;" ::: "memory");
        return;
      }
      tc_fence_after();
      constexpr int kLoad = 16, kLoads = kUnit / kLoad;
      const uint32_t from = t_lane + buf * (uint32_t)kRows + (uint32_t)(set * kUnit);
      auto release = [&](int h) {
        if (lane == 0) mbar_arrive(S.dempty + 8u * (buf + h));
      };
      auto add = [&](int j, int h, const int32_t (&v)[kLoad]) {
        if (x_groups) {
#pragma unroll
          for (int i = 0; i < kLoad / 4; ++i) {
            const float4 f = lds_f4(my_scales + (uint32_t)(4 * kUnit * h + 4 * kLoad * j + 16 * i));
            float *to = acc + kLoad * j + 4 * i;
            to[0] = fmaf(__int_as_float(v[4 * i]) * f.x, s[h], to[0]);
            to[1] = fmaf(__int_as_float(v[4 * i + 1]) * f.y, s[h], to[1]);
            to[2] = fmaf(__int_as_float(v[4 * i + 2]) * f.z, s[h], to[2]);
            to[3] = fmaf(__int_as_float(v[4 * i + 3]) * f.w, s[h], to[3]);
          }
        } else {
#pragma unroll
          for (int i = 0; i < kLoad; ++i) acc[kLoad * j + i] = fmaf(__int_as_float(v[i]), s[h], acc[kLoad * j + i]);
        }
      };
      if constexpr (kPair == 2) {
        int32_t vs[2][kLoads][kLoad];
#pragma unroll
        for (int j = 0; j < 2 * kLoads; ++j)       // (a group that does not exist: the first again, not added)
          tmem_ld16(from + (uint32_t)((j / kLoads < count ? j / kLoads : 0) * kRows + kLoad * (j % kLoads)), vs[j / kLoads][j % kLoads]);
#pragma unroll
        for (int j = 0; j < 2 * kLoads; ++j) tmem_wait16(vs[j / kLoads][j % kLoads]);
        tc_fence_before();
        __syncwarp();
        release(0);
        if (count == 2) release(1);
#pragma unroll
        for (int j = 0; j < kLoads; ++j) add(j, 0, vs[0][j]);
        if (count == 2) {
#pragma unroll
          for (int j = 0; j < kLoads; ++j) add(j, 1, vs[1][j]);
        }
      } else {
        // 16 values at a time; the next load is under way while these are added
        int32_t vs[2][kLoad];
        tmem_ld16(from, vs[0]);
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
          tmem_wait16(vs[j & 1]);
          if (j + 1 < kLoads) {
            tmem_ld16(from + (uint32_t)(kLoad * (j + 1)), vs[(j + 1) & 1]);
          } else {
            tc_fence_before();
            __syncwarp();
            release(0);
          }
          add(j, 0, vs[j & 1]);
        }
      }
    }
    if (P.split > 1) {                     // [row of x][output], for the cluster
#pragma unroll
      for (int i = 0; i < kUnit; ++i)
        sts32(S.ring + (uint32_t)(((set * kUnit + i) * kTileN + 32 * quarter + lane) * 4), __float_as_uint(acc[i]));
    } else {
      if (A.x_scales != nullptr && !x_groups) {                   // a scale for each row
        __syncwarp();
#pragma unroll
        for (int i = 0; i < (kUnit + 31) / 32; ++i) {
          const int col = lane + 32 * i;
          const float v = col < kUnit && tok0 + col < A.r.rows ? load_global(A.x_scales + tok0 + col) : 0.0f;
          if (col < kUnit) sts32(my_scales + 4u * col, __float_as_uint(v));
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < kUnit / 4; ++i) {
          const float4 f = lds_f4(my_scales + 16u * i);
          acc[4 * i] *= f.x; acc[4 * i + 1] *= f.y; acc[4 * i + 2] *= f.z; acc[4 * i + 3] *= f.w;
        }
      }
      if (n < N) {
        const long long at = tok0 * A.r.out_stride + n;
        const int left = (int)min((long long)kUnit, A.r.rows - tok0);
        if (A.r.out_type == XNOR_F32) store_column(acc, static_cast<float *>(A.out) + at, A.r.out_stride, left);
        else if (A.r.out_type == XNOR_BF16) store_column(acc, static_cast<__nv_bfloat16 *>(A.out) + at, A.r.out_stride, left);
        else store_column(acc, static_cast<__half *>(A.out) + at, A.r.out_stride, left);
      }
    }
  }
}

template <int kType, int kRows, bool kCopies>
__global__ void __launch_bounds__(Shape<kRows, kCopies>::kThreads, 1)
w4_tc_kernel(const __grid_constant__ TcParams P) {
  using Sh = Shape<kRows, kCopies>;
  using T = typename RowsOf<kType>::T;
  extern __shared__ __align__(1024) uint8_t smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const Smem S = carve(smem, Sh::kScaleBytes);
  if (threadIdx.x == 0) {
    // a stage is full with four expanding warps' arrivals and those that bring the rows
    for (int i = 0; i < Sh::kStages; ++i) { mbar_init(S.full + 8u * i, 4 + (kCopies ? 1 : Sh::kLoadWarps)); mbar_init(S.empty + 8u * i, 1); }
    for (int i = 0; i < kWeightStages; ++i) { mbar_init(S.wfull + 8u * i, 1); mbar_init(S.wempty + 8u * i, 8); }
    for (int i = 0; i < Sh::kBufs; ++i) { mbar_init(S.dfull + 8u * i, 1); mbar_init(S.dempty + 8u * i, 4 * Sh::kPromo); }
    *S.abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (kCopies && warp == Sh::kLoadWarp && lane == 0)
    asm volatile("prefetch.tensormap [%0];" ::"l"(&P.x_map) : "memory");
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
    promote_role<Sh, kRows>(P, S, span, first, step, total, warp >> 2, warp & 3, lane, tmem);
  } else {
    if constexpr (Sh::kOtherRegs != Sh::kRegs) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(Sh::kOtherRegs));
    if (warp < Sh::kMmaWarp) {
      expand_role<Sh, T>(P, S, span, first, step, total, (warp >> 2) - Sh::kPromo, warp & 3, lane, tmem);
    } else if (warp == Sh::kMmaWarp) {
      if (elect_one()) {
        if (P.A.d.group == 128) mma_loop<Sh, kRows, 128>(P, S, span, mine, tmem);
        else if (P.A.d.group == 64) mma_loop<Sh, kRows, 64>(P, S, span, mine, tmem);
        else mma_loop<Sh, kRows, 32>(P, S, span, mine, tmem);
      }
    } else if (warp == Sh::kWeightWarp) {
      if (elect_one()) weight_role(P, S, span, first, step, total);
    } else if constexpr (kCopies) {
      if (warp == Sh::kLoadWarp && elect_one()) copy_role<Sh, kRows>(P, S, span, first, step, total);
    } else {
      bool done = false;
      if constexpr (RowsOf<kType>::kBytes == 1) {
        if (P.pieces) { load_role<Sh, kType, kRows>(P, S, span, first, step, total, warp - Sh::kLoadWarp, lane); done = true; }
      }
      if (!done) word_role<Sh, kType, kRows>(P, S, span, first, step, total, warp - Sh::kLoadWarp, lane);
    }
    __syncwarp();
  }
  tc_fence_before();
  __syncthreads();
  if (warp == Sh::kMmaWarp)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
  if (P.split == 1) return;
  // a cluster has one tile; its blocks write shares of the rows, each the sums of all in the same order
  cluster_sync();
  const int n0 = (first % P.row_tiles) * kTileN;
  const long long tok0 = (long long)(first / P.row_tiles) * kRows;
  const bool row_scale = P.A.x_scales != nullptr && P.A.r.x_group == 0;
  const int r0 = kRows * rank / P.split, r1 = kRows * (rank + 1) / P.split;
  for (int e = r0 * (kTileN / 4) + threadIdx.x; e < r1 * (kTileN / 4); e += Sh::kThreads) {       // four outputs each
    const int n = n0 + 4 * (e % (kTileN / 4));
    const long long row = tok0 + e / (kTileN / 4);
    if (row >= P.A.r.rows || n >= P.A.d.N) continue;
    float4 v[kMaxSplitTc];
#pragma unroll
    for (int i = 0; i < kMaxSplitTc; ++i) {
      if (i >= P.split) continue;
      uint32_t a;
      asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(S.ring + 16u * (uint32_t)e), "r"(i));
      asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[i].x), "=f"(v[i].y), "=f"(v[i].z), "=f"(v[i].w) : "r"(a) : "memory");
    }
    float4 s = v[0];
#pragma unroll
    for (int i = 1; i < kMaxSplitTc; ++i)
      if (i < P.split) { s.x += v[i].x; s.y += v[i].y; s.z += v[i].z; s.w += v[i].w; }
    if (row_scale) {
      const float f = load_global(P.A.x_scales + row);
      s.x *= f; s.y *= f; s.z *= f; s.w *= f;
    }
    const long long at = row * P.A.r.out_stride + n;
    const int left = P.A.d.N - n;
    if (P.A.r.out_type == XNOR_F32) store_four(s, static_cast<float *>(P.A.out) + at, left);
    else if (P.A.r.out_type == XNOR_BF16) store_four(s, static_cast<__nv_bfloat16 *>(P.A.out) + at, left);
    else store_four(s, static_cast<__half *>(P.A.out) + at, left);
  }
  cluster_sync();
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
bool copied(const W4Args &a) {
  return RowsOf<kType>::kBytes == 2 && rows_in_pieces(a.x, a.r.x_stride, 8, 2) && a.r.x_stride >= a.d.K && encode_tiled() != nullptr;
}
template <int kType>
bool map_rows(const W4Args &a, int rows, CUtensorMap *map) {
  const cuuint64_t size[2] = {(cuuint64_t)a.d.K, (cuuint64_t)a.r.rows}, stride[1] = {(cuuint64_t)a.r.x_stride * 2};
  const cuuint32_t box[2] = {kChunk, (cuuint32_t)rows}, each[2] = {1, 1};
  return encode_tiled()(map, kType == XNOR_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2,
                        const_cast<void *>(a.x), size, stride, box, each, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                        CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int kType, int kRows, bool kCopies>
cudaError_t run(const W4Args &a, cudaStream_t st) {
  using Sh = Shape<kRows, kCopies>;
  static bool attr_flags[64] = {};
  bool &attr_set = attr_done_for_current_device(attr_flags);
  if (!attr_set) {
    const cudaError_t e = cudaFuncSetAttribute(w4_tc_kernel<kType, kRows, kCopies>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Sh::kSmem);
    if (e != cudaSuccess) { (void)cudaGetLastError(); return e; }
    attr_set = true;
  }
  TcParams P;
  if constexpr (kCopies) {
    if (!map_rows<kType>(a, kRows, &P.x_map)) return cudaErrorInvalidValue;
  }
  P.A = a;
  P.magic = W4Type<typename RowsOf<kType>::T>::kMagic;
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
  return launch_kernel(w4_tc_kernel<kType, kRows, kCopies>, dim3(grid), Sh::kThreads, Sh::kSmem, st, (unsigned)P.split, P);
}

template <int kType, bool kCopies>
cudaError_t run_rows(const W4Args &a, cudaStream_t st) {
  if (a.r.rows <= 16) return run<kType, 16, kCopies>(a, st);
  if (a.r.rows <= 32) return run<kType, 32, kCopies>(a, st);
  if (a.r.rows <= 64) return run<kType, 64, kCopies>(a, st);
  return run<kType, 128, kCopies>(a, st);
}
template <int kType>
cudaError_t run_type(const W4Args &a, cudaStream_t st) {
  if constexpr (RowsOf<kType>::kBytes == 2) {
    if (copied<kType>(a)) {
      const long long tiles = (a.d.N + kTileN - 1) / kTileN * ((a.r.rows + 191ll) / 192);
      if (a.r.rows > 128 && 2 * tiles > sm_count_of_current_device()) return run<kType, 192, true>(a, st);
      return run_rows<kType, true>(a, st);
    }
  }
  return run_rows<kType, false>(a, st);
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
