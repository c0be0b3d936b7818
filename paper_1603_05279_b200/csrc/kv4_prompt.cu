// Attention over the cache in 4 bits for many new tokens of a sequence, on the 5th-generation tensor cores.
//
// A block computes one item: up to 256 rows (queries of a head's group, token by token) in two halves of 128, over their
// context in tiles of 128 tokens.  S = Q K^T (128 x 128) and O += P V run on tcgen05.mma kind::f16 with fp32 sums in tensor memory:
// S and O of both halves fill it, and P, in F16, lies where S lay.  Keys and values become code - zero, exactly, in shared
// memory; a key's scale multiplies its column of S, a value's its column of P (rounded to F16 as in the kernel for few
// rows).  The softmax is one pass with a running maximum that may be left behind by 2^3, so that O is rescaled rarely.
//
// Warps: 0 - 7  softmax: a thread has a row of its half; it also brings the row's query and takes its output away
//        8 - 11 expansion: 4-bit records into operands of 128 tokens (three stages), and the columns' scales
//        12     issues the products: while one half's softmax runs, the other half's P V and the next Q K^T
//        13     copies records into a ring in shared memory, a thread a record
// Where there are too few items for the GPU, the blocks of an item divide its context, and a second kernel joins
// their sums.  Every wait is bounded; on expiry the block records XNOR_ERR_TIMEOUT, stops and frees its tensor memory.
#include <algorithm>
#include <climits>

#include "kv4_attention.cuh"

namespace xnor {

__device__ int g_status_kv4_prompt = 0;

namespace {

using namespace umma;

constexpr int kHalf = 128, kItemRows = 2 * kHalf;
constexpr int kTokens = 128, kRecords = kTokens / kKvTokens;     // of a tile
constexpr int kOperands = 3, kRawStages = 2, kScaleBufs = 4;
constexpr int kExpandWarp = 8, kMmaWarp = 12, kCopyWarp = 13, kThreads = 16 * 32;
constexpr int kSoftmaxRegs = 184, kOtherRegs = 72, kLaunchRegs = 128;
static_assert(8 * 32 * (kSoftmaxRegs + kOtherRegs) <= kThreads * kLaunchRegs, "registers");
constexpr int kMaxSplits = 8;

template <int kDim>
struct Layout {
  static constexpr uint32_t kOperand = kTokens * kDim * 2;       // also of 128 queries
  static constexpr uint32_t kRaw = kRecords * kv4_record(kDim);
  static constexpr uint32_t kRawFull = 0, kRawEmpty = kRawFull + 8 * kRawStages, kFull = kRawEmpty + 8 * kRawStages, kEmpty = kFull + 8 * kOperands;
  static constexpr uint32_t kSFull = kEmpty + 8 * kOperands, kPFull = kSFull + 16, kQFull = kPFull + 16;
  static constexpr uint32_t kScaled = kQFull + 16, kTmem = kScaled + 8 * kScaleBufs, kAbort = kTmem + 4, kItem = kAbort + 4, kMask = kItem + 32, kExponent = kMask + 4 * kRawStages;
  static constexpr uint32_t kThere = kExponent + 4 * kScaleBufs;
  static constexpr uint32_t kScales = 512, kRing = kScales + kScaleBufs * 2 * kTokens * 4;
  static constexpr uint32_t kQ = kRing + kRawStages * kRaw;      // (rounded up to 1024 in memory)
  static constexpr uint32_t kBytes = kQ + 1024 + 2 * kOperand + kOperands * kOperand;
  static_assert(kThere + 4 * kScaleBufs <= kScales && kBytes <= 232448, "shared memory");
  static constexpr uint32_t kO = 256;                            // tensor memory: S of both halves, then O
};

struct Params {
  Kv4Args A;
  Tiling T;
  long long blocks;
  int splits, q_pieces, out_pieces;
  uint32_t magic, magic16;     // W4Type's of the queries' type and of F16
};

// One of the call's items, or none: rank in the row of items of a head (sequences, in them the longest context first).
struct Item {
  int b, tile, rank;
  bool there;
};
__device__ __forceinline__ Item item_of(const Params &P, int rank, int lane) {
  const Kv4Where &W = P.A.w;
  const int per = (W.d.seqs + 31) / 32;
  long long mine = 0;
#pragma unroll 4
  for (int i = 0; i < per; ++i) {
    const int b = lane * per + i;
    if (b >= W.d.seqs) break;
    Sequence s;
    s.load(W, P.T, b);
    mine += s.tiles;
  }
  long long before = mine;
#pragma unroll
  for (int o = 1; o < 32; o *= 2) {
    const long long v = __shfl_up_sync(0xffffffffu, before, o);
    if (lane >= o) before += v;
  }
  before -= mine;
  Item r = {0, 0, rank, rank >= before && rank < before + mine};
  if (r.there)
    for (int i = lane * per;; ++i) {
      Sequence s;
      s.load(W, P.T, i);
      if (rank < before + s.tiles) { r.b = i; r.tile = s.tiles - 1 - (int)(rank - before); break; }
      before += s.tiles;
    }
  const uint32_t who = __ballot_sync(0xffffffffu, r.there);
  r.there = who != 0;
  if (!r.there) return r;
  r.b = __shfl_sync(0xffffffffu, r.b, __ffs((int)who) - 1);
  r.tile = __shfl_sync(0xffffffffu, r.tile, __ffs((int)who) - 1);
  return r;
}
// The rank of an item of sequence b's tile; the same for all threads.
__device__ __forceinline__ int rank_of(const Params &P, int b, int tile, int lane) {
  int mine = 0;
#pragma unroll 4
  for (int i = lane; i < b; i += 32) {
    Sequence s;
    s.load(P.A.w, P.T, i);
    mine += s.tiles;
  }
  Sequence s;
  s.load(P.A.w, P.T, b);
  return __reduce_add_sync(0xffffffffu, mine) + s.tiles - 1 - tile;
}

// An item's tiles of context, and the share of them that one of its blocks has.
struct Span {
  int tiles, splits, first, last;
  __device__ __forceinline__ Span(const Params &P, const Sequence &s, int tile, int split) {
    const long long end_row = min((long long)s.n * P.T.group, (long long)(tile + 1) * kItemRows);
    const int last_token = (int)((end_row - 1) / P.T.group);
    const int seen = min(s.len, max(0, s.lead + s.start + last_token + 1));            // tokens that any of its rows sees
    tiles = (seen + kTokens - 1) / kTokens;
    splits = min(P.splits, max(1, tiles / 4));
    first = (int)((long long)tiles * split / splits);
    last = (int)((long long)tiles * (split + 1) / splits);
  }
};

__device__ __forceinline__ size_t partial_floats(int dim) { return (size_t)kItemRows * (dim + 2); }

struct Block {                // what all roles know
  const Params &P;
  Sequence s;
  int b, head, tile, first, last;
  bool two, direct;           // both halves have rows; the block has the whole context
  uint32_t smem, q, operands, tmem;
  uint8_t *ptr;
  volatile int *abort_flag;
  float *partial;
};

__device__ __forceinline__ bool wait(const Block &B, uint32_t bar, uint32_t parity) { return mbar_wait(bar, parity, B.abort_flag, &g_status_kv4_prompt); }
__device__ __forceinline__ bool wait_warp(const Block &B, uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, wait(B, bar, parity)); }

// The same as straight code, for the warps whose registers are full: a call has registers of its own.
__device__ __forceinline__ bool wait_inline(const Block &B, uint32_t bar, uint32_t parity) {
  bool ok = mbar_try(bar, parity);
  if (!ok) {
    const long long t0 = clock64();
#pragma unroll 1
    while (!ok && *B.abort_flag == 0) {
      ok = mbar_try(bar, parity);
      if (!ok && clock64() - t0 > kWaitCycles) {
        *B.abort_flag = 1;
        atomicExch(&g_status_kv4_prompt, (int)XNOR_ERR_TIMEOUT);
      }
    }
  }
  return __all_sync(0xffffffffu, ok);
}

// ---- copies --------------------------------------------------------------------------------------------------------
template <int kDim>
__device__ __forceinline__ void copy_role(const Block &B, int lane) {
  using L = Layout<kDim>;
  const Params &P = B.P;
  auto find = [&](int tile) {
    const int rec = tile * kRecords + lane;
    return tile < B.last && lane < kRecords && rec * kKvTokens < B.s.len ? kv4_find(P.A.w, B.b, rec, B.head) : -2ll;
  };
  long long next = find(B.first);
  for (int t = B.first; t < B.last; ++t) {
    const int i = t - B.first;
    const uint32_t slot = (uint32_t)i % kRawStages, parity = (uint32_t)(i / kRawStages) & 1u, full = B.smem + L::kRawFull + 8u * slot;
    const long long now = next;
    next = find(t + 1);
    if (!wait_warp(B, B.smem + L::kRawEmpty + 8u * slot, parity ^ 1u)) {
      // gave up: copies in flight must land before the block's shared memory is released
      const long long t0 = clock64();
      while (clock64() - t0 < (1 << 20)) {}
      return;
    }
    const uint32_t there = __ballot_sync(0xffffffffu, now >= 0);
    if (now == -1) atomicMax(&g_status_kv4_prompt, (int)XNOR_ERR_BOUNDS);
    if (lane == 0) {
      sts32(B.smem + L::kMask + 4u * slot, there);
      mbar_arrive_expect_tx(full, (uint32_t)__popc(there) * kv4_record(kDim));
    }
    __syncwarp();
    if (now >= 0)
      bulk_copy_g2s(B.smem + L::kRing + slot * L::kRaw + (uint32_t)lane * kv4_record(kDim), P.A.cache + (size_t)now * kv4_record(kDim), kv4_record(kDim), full);
  }
}

// ---- expansion -------------------------------------------------------------------------------------------------------
// Operands: rows of 64 values (128 bytes), swizzled in groups of eight; blocks of 64 columns one after the other.  Keys: a row is a
// token.  Values: a row is a column of O, its values tokens; so eight tokens' codes are transposed on the way, by
// choosing bytes of two tokens at a time.
template <class T, int kDim>
__device__ __forceinline__ void expand_role(const Block &B, int id) {
  using L = Layout<kDim>;
  using V = W4Type<__half>;
  constexpr uint32_t kRecord = kv4_record(kDim);
  constexpr int kQuads = kDim / 32;                        // of words in a token's codes
  const int lane = id & 31;
  const float scale2 = B.P.A.r.scale * kLog2e;
  float *scales = reinterpret_cast<float *>(B.ptr + L::kScales);
  int e = kLeastScale;
  uint32_t op = 0u;                                        // operands so far
  for (int t = B.first; t < B.last; ++t) {
    const int i = t - B.first;
    const uint32_t slot = (uint32_t)i % kRawStages, raw = B.smem + L::kRing + slot * L::kRaw, buf = (uint32_t)i % kScaleBufs;
    if (!wait_warp(B, B.smem + L::kRawFull + 8u * slot, (uint32_t)(i / kRawStages) & 1u)) return;
    const uint32_t there = lds32(B.smem + L::kMask + 4u * slot);
    uint32_t stage = op % kOperands;
    if (!wait_warp(B, B.smem + L::kEmpty + 8u * stage, ((op / kOperands) & 1u) ^ 1u)) return;
    {
      // the columns' scales; all warps find the largest value's
      int above = e;
#pragma unroll
      for (int k = 0; k < kTokens / 32; ++k) {
        const int tok = lane + 32 * k;
        const bool in = (there >> (tok / kKvTokens) & 1u) && t * kTokens + tok < B.s.len;
        if (in) above = max(above, scale_above(kv4_scale(lds32(raw + (uint32_t)(tok / kKvTokens) * kRecord + kv4_words(kDim, true) + 4u * (tok % kKvTokens)))));
      }
      e = __reduce_max_sync(0xffffffffu, above);
      const bool in = (there >> (id / kKvTokens) & 1u) && t * kTokens + id < B.s.len;
      const uint32_t words = raw + (uint32_t)(id / kKvTokens) * kRecord + 4u * (id % kKvTokens);
      scales[(2 * buf) * kTokens + id] = in ? kv4_scale(lds32(words + kv4_words(kDim, false))) * scale2 : 0.0f;
      scales[(2 * buf + 1) * kTokens + id] = in ? kv4_scale(lds32(words + kv4_words(kDim, true))) * power_of_two(12 - e) : 0.0f;
      if (id == 0) {
        sts32(B.smem + L::kExponent + 4u * buf, (uint32_t)e);
        sts32(B.smem + L::kThere + 4u * buf, there);
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(B.smem + L::kScaled + 8u * buf);
    }
    {
      const uint32_t to = B.operands + stage * L::kOperand;
#pragma unroll
      for (int k = 0; k < kQuads; ++k) {
        // neighbours in a quarter of a warp: four tokens, two quads; neither loads nor stores meet in a bank more than twice
        const int j = id + 128 * k;
        const int quad = (j & 1) + 2 * (j / 256), tok = ((j >> 1) & 3) + 4 * ((j >> 3) & 31);
        const uint32_t from = raw + (uint32_t)(tok / kKvTokens) * kRecord, slot_of = (uint32_t)(tok % kKvTokens);
        uint32_t c[4];
        lds128(from + slot_of * (kDim / 2) + 16u * quad, c);
        const typename W4Type<T>::Zero z = W4Type<T>::zero(lds32(from + kv4_words(kDim, false) + 4u * slot_of) & 15u);
        const uint32_t row = to + (uint32_t)(quad / 2) * (kTokens * 128) + (uint32_t)tok * 128u;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          uint32_t v[4];
          W4Type<T>::expand(c[w], z, B.P.magic, v);
          sts128(row + (uint32_t)((((quad & 1) * 4 + w) ^ (tok & 7)) * 16), v[0], v[1], v[2], v[3]);
        }
      }
    }
    fence_proxy_async();
    __syncwarp();
    if (lane == 0) mbar_arrive(B.smem + L::kFull + 8u * stage);
    ++op;
    stage = op % kOperands;
    if (!wait_warp(B, B.smem + L::kEmpty + 8u * stage, ((op / kOperands) & 1u) ^ 1u)) return;
    {
      const uint32_t to = B.operands + stage * L::kOperand;
      // a thread: eight tokens of one word (eight columns).  Neighbours: eight octets of tokens, whose words are taken from
      // other quads and in the other order of two tokens, so that they lie in other banks.
      const int octet = (id & 7) + 8 * ((id >> 5) & 1), odd = octet & 1;
      const uint32_t from = raw + (uint32_t)(octet / 2) * kRecord + kv4_codes(kDim, true) + (uint32_t)(8 * odd) * (kDim / 2);
      uint32_t za[4], zb[4];
      {
        const uint32_t words = raw + (uint32_t)(octet / 2) * kRecord + kv4_words(kDim, true) + 32u * odd;
        uint32_t w[8];
        lds128(words, *reinterpret_cast<uint32_t (*)[4]>(w));
        lds128(words + 16u, *reinterpret_cast<uint32_t (*)[4]>(w + 4));
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t z = (w[2 * j] & 15u) | (w[2 * j + 1] & 15u) << 16;
          za[j] = 0x64006400u | z;
          zb[j] = 0xD400D400u | z << 4;
        }
      }
      const uint32_t low = odd ? 0x1054u : 0x5410u, high = odd ? 0x3276u : 0x7632u;
#pragma unroll 1
      for (int k = 0; k < kDim / 64; ++k) {                // 8 lanes x 4 words x 2 halves of the warps
        const int quad = ((octet >> 1) + 2 * k + (id >> 6)) & (kQuads - 1), word = 4 * quad + ((id >> 3) & 3);
        uint32_t c[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) c[j] = lds32(from + (uint32_t)(j ^ odd) * (kDim / 2) + 4u * word);
        const uint32_t block = to + (uint32_t)(octet / 8) * (kDim * 128), slot_of = (uint32_t)(octet & 7);
#pragma unroll
        for (int h = 0; h < 2; ++h) {                      // even, odd columns
          uint32_t v[4][4];
#pragma unroll
          for (int j = 0; j < 4; ++j) V::expand(__byte_perm(c[2 * j], c[2 * j + 1], h == 0 ? low : high), {za[j], zb[j]}, B.P.magic16, v[j]);
#pragma unroll
          for (int p = 0; p < 4; ++p) {
            const uint32_t column = (uint32_t)(2 * p + h);
            sts128(block + ((uint32_t)(8 * word) + column) * 128u + ((slot_of ^ column) * 16u), v[0][p], v[1][p], v[2][p], v[3][p]);
          }
        }
      }
    }
    fence_proxy_async();
    __syncwarp();
    if (lane == 0) {
      mbar_arrive(B.smem + L::kFull + 8u * stage);
      mbar_arrive(B.smem + L::kRawEmpty + 8u * slot);
    }
    ++op;
  }
}

// ---- products ------------------------------------------------------------------------------------------------------
__device__ __forceinline__ uint64_t swizzled_desc(uint32_t addr) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | (1ull << 16) | ((uint64_t)(1024u >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ void mma_shared(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void mma_tmem(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// D fp32, A and B of one 16-bit type, both K-major, M = 128.
__host__ __device__ constexpr uint32_t instruction(bool bf16, int n) {
  return (1u << 4) | ((bf16 ? 1u : 0u) << 7) | ((bf16 ? 1u : 0u) << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(kHalf >> 4) << 24);
}

template <class T, int kDim>
__device__ __forceinline__ void mma_role(const Block &B) {
  using L = Layout<kDim>;
  constexpr uint32_t kSDesc = instruction(std::is_same<T, __nv_bfloat16>::value, kTokens), kODesc = instruction(false, kDim);
  const int n = B.last - B.first, halves = B.two ? 2 : 1;
  const uint64_t q0 = swizzled_desc(B.q), op0 = swizzled_desc(B.operands);
  auto qk = [&](int half, uint32_t stage) {
#pragma unroll
    for (int k = 0; k < kDim / 16; ++k) {
      const uint64_t step = (uint64_t)((uint32_t)(k / 4) * (kTokens * 128 / 16) + 2u * (uint32_t)(k % 4));
      mma_shared(B.tmem + (uint32_t)(half * kTokens), q0 + (uint64_t)((uint32_t)half * (L::kOperand / 16)) + step, op0 + (uint64_t)(stage * (L::kOperand / 16)) + step, kSDesc,
                 k > 0 ? 1u : 0u);
    }
    umma_commit(B.smem + L::kSFull + 8u * half);
  };
  auto pv = [&](int half, uint32_t stage, bool first) {
#pragma unroll
    for (int k = 0; k < kTokens / 16; ++k) {
      const uint64_t step = (uint64_t)((uint32_t)(k / 4) * (kDim * 128 / 16) + 2u * (uint32_t)(k % 4));
      mma_tmem(B.tmem + L::kO + (uint32_t)(half * kDim), B.tmem + (uint32_t)(half * kTokens + 8 * k), op0 + (uint64_t)(stage * (L::kOperand / 16)) + step, kODesc,
               first && k == 0 ? 0u : 1u);
    }
  };
  auto full = [&](uint32_t op) { return wait(B, B.smem + L::kFull + 8u * (op % kOperands), (op / kOperands) & 1u); };
  for (int h = 0; h < halves; ++h)
    if (!wait(B, B.smem + L::kQFull + 8u * h, 0u)) return;
  if (!full(0u)) return;
  tc_fence_after();
  for (int h = 0; h < halves; ++h) qk(h, 0u);
  umma_commit(B.smem + L::kEmpty);
#pragma unroll 1
  for (int i = 0; i < n; ++i) {
    const uint32_t values = 2u * (uint32_t)i + 1u, keys = values + 1u;
    if (!full(values)) return;
    for (int h = 0; h < halves; ++h) {
      if (!wait(B, B.smem + L::kPFull + 8u * h, (uint32_t)i & 1u)) return;
      tc_fence_after();
      pv(h, values % kOperands, i == 0);
      if (h + 1 == halves) umma_commit(B.smem + L::kEmpty + 8u * (values % kOperands));
      if (i + 1 < n) {
        if (h == 0 && !full(keys)) return;
        tc_fence_after();
        qk(h, keys % kOperands);                           // (behind P V, whose P it overwrites)
        if (h + 1 == halves) umma_commit(B.smem + L::kEmpty + 8u * (keys % kOperands));
      } else {
        umma_commit(B.smem + L::kSFull + 8u * h);          // O is done
      }
    }
  }
}

// ---- softmax -------------------------------------------------------------------------------------------------------
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
        "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr) : "memory");
}
// Every tcgen05.ld of this thread has returned; the registers are operands so that nothing uses them before.
__device__ __forceinline__ void tmem_wait32(uint32_t (&r)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]),
                 "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]),
                 "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
               :: "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ float4 lds_float4(uint32_t addr) {
  uint32_t v[4];
  lds128(addr, v);
  return make_float4(__uint_as_float(v[0]), __uint_as_float(v[1]), __uint_as_float(v[2]), __uint_as_float(v[3]));
}

// Two fp32 operations at once.
__device__ __forceinline__ uint64_t pack2(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 unpack2(uint64_t v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(pack2(a.x, a.y)), "l"(pack2(b.x, b.y)));
  return unpack2(r);
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(pack2(a.x, a.y)), "l"(pack2(b.x, b.y)));
  return unpack2(r);
}

template <class T, int kDim>
__device__ __forceinline__ void softmax_role(const Block &B, int half, int quarter, int lane) {
  using L = Layout<kDim>;
  const Params &P = B.P;
  const int in_tile = 32 * quarter + lane;
  const long long r = (long long)B.tile * kItemRows + half * kHalf + in_tile;
  const int token = (int)(r / P.T.group), head = B.head * P.T.group + (int)(r - (long long)token * P.T.group);
  const bool in = token < B.s.n;
  const long long row = B.s.start + token;
  const int limit = in ? min(B.s.lead + B.s.start + token, B.s.len - 1) : INT_MAX;        // the last token that it sees
  if (half == 1 && !B.two) return;
  // the query, 64 columns a block
  {
    const T *q = static_cast<const T *>(P.A.q) + (in ? row * P.A.r.q_stride + (long long)head * kDim : 0);
    const uint32_t to = B.q + (uint32_t)half * L::kOperand + (uint32_t)in_tile * 128u;
#pragma unroll
    for (int c = 0; c < kDim / 8; ++c) {
      Chunk<T> v;
      v.load(q + 8 * c, P.q_pieces, in ? 8 : 0);
      sts128(to + (uint32_t)(c / 8) * (kTokens * 128) + (uint32_t)(((c & 7) ^ (in_tile & 7)) * 16), v.w[0], v.w[1], v.w[2], v.w[3]);
    }
    fence_proxy_async();
    __syncwarp();
    if (lane == 0) mbar_arrive(B.smem + L::kQFull + 8u * half);
  }
  const uint32_t lanes = B.tmem + ((uint32_t)(32 * quarter) << 16), S = lanes + (uint32_t)(half * kTokens), O = lanes + L::kO + (uint32_t)(half * kDim);
  const int n = B.last - B.first, least = __reduce_min_sync(0xffffffffu, limit);
  float m = -INFINITY, l = 0.0f;
  int e = kLeastScale;
#pragma unroll 1
  for (int i = 0; i < n; ++i) {
    const uint32_t buf = (uint32_t)i % kScaleBufs;
    if (!wait_inline(B, B.smem + L::kSFull + 8u * half, (uint32_t)i & 1u) ||
        !wait_inline(B, B.smem + L::kScaled + 8u * buf, (uint32_t)(i / kScaleBufs) & 1u))
      return;
    tc_fence_after();
    const uint32_t ks = B.smem + L::kScales + 2u * buf * kTokens * 4u, vs = ks + kTokens * 4u;
    const int e_now = (int)lds32(B.smem + L::kExponent + 4u * buf);
    const uint32_t there = lds32(B.smem + L::kThere + 4u * buf);
    const int t0 = (B.first + i) * kTokens;
    float2 x[kTokens / 2];
    float top = -INFINITY;
    const bool whole = there == (1u << kRecords) - 1u && t0 + kTokens - 1 <= least;
    {
      uint32_t a[32], b[32];
      auto scaled = [&](int c, const uint32_t (&raw)[32]) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float4 f = lds_float4(ks + 16u * (uint32_t)(8 * c + j));
          x[16 * c + 2 * j] = mul2(make_float2(__uint_as_float(raw[4 * j]), __uint_as_float(raw[4 * j + 1])), make_float2(f.x, f.y));
          x[16 * c + 2 * j + 1] = mul2(make_float2(__uint_as_float(raw[4 * j + 2]), __uint_as_float(raw[4 * j + 3])), make_float2(f.z, f.w));
        }
      };
      tmem_ld32(S, a);
      tmem_wait32(a);
      tmem_ld32(S + 32u, b);
      scaled(0, a);
      tmem_wait32(b);
      tmem_ld32(S + 64u, a);
      scaled(1, b);
      tmem_wait32(a);
      tmem_ld32(S + 96u, b);
      scaled(2, a);
      tmem_wait32(b);
      scaled(3, b);
    }
    if (!whole) {
#pragma unroll
      for (int j = 0; j < kTokens / 2; ++j) {
        const bool here = there >> (2 * j / kKvTokens) & 1u;
        if (!here || t0 + 2 * j > limit) x[j].x = -INFINITY;
        if (!here || t0 + 2 * j + 1 > limit) x[j].y = -INFINITY;
      }
    }
    float top1 = -INFINITY;
#pragma unroll
    for (int j = 0; j < kTokens / 2; j += 2) {
      top = fmaxf(top, fmaxf(x[j].x, x[j].y));
      top1 = fmaxf(top1, fmaxf(x[j + 1].x, x[j + 1].y));
    }
    top = fmaxf(top, top1);
    // (m = -infinity: any number exceeds it)
    if (__any_sync(0xffffffffu, top > m + kRaise || e_now > e)) {
      const float above = top > m + kRaise ? top : m;
      const float f = above == -INFINITY ? 1.0f : exp2_fast(m - above), down = f * power_of_two(e - e_now);
      m = above;
      e = e_now;
      l *= f;
      if (i > 0) {                                         // (S of this tile came behind P V of the last one: O is there)
#pragma unroll
        for (int c = 0; c < kDim / 16; ++c) {
          int32_t o[16];
          uint32_t scaled[16];
          tmem_ld16(O + 16u * c, o);
          tmem_wait16(o);
#pragma unroll
          for (int j = 0; j < 16; ++j) scaled[j] = __float_as_uint(__int_as_float(o[j]) * down);
          tmem_st16(O + 16u * c, scaled);
        }
      }
    }
    const float base = m == -INFINITY ? 0.0f : -m;
    const float2 base2 = make_float2(base, base);
    float2 sum = make_float2(0.0f, 0.0f), sum1 = sum;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      uint32_t p[16];
#pragma unroll
      for (int j = 0; j < 16; j += 2) {
        const float4 f = lds_float4(vs + 16u * (uint32_t)(8 * c + j / 2));
        float2 u = add2(x[16 * c + j], base2), v = add2(x[16 * c + j + 1], base2);
        u = make_float2(exp2_fast(u.x), exp2_fast(u.y));
        v = make_float2(exp2_fast(v.x), exp2_fast(v.y));
        sum = add2(sum, u);
        sum1 = add2(sum1, v);
        u = mul2(u, make_float2(f.x, f.y));
        v = mul2(v, make_float2(f.z, f.w));
        if (!whole) {                                      // (a token that is not seen may stand for anything)
          if (x[16 * c + j].x == -INFINITY) u.x = 0.0f;
          if (x[16 * c + j].y == -INFINITY) u.y = 0.0f;
          if (x[16 * c + j + 1].x == -INFINITY) v.x = 0.0f;
          if (x[16 * c + j + 1].y == -INFINITY) v.y = 0.0f;
        }
        p[j] = float_to_pair(u.x, u.y, __half());
        p[j + 1] = float_to_pair(v.x, v.y, __half());
      }
      tmem_st16(S + 16u * c, p);
    }
    l += (sum.x + sum.y) + (sum1.x + sum1.y);
    tmem_wait_st();
    tc_fence_before();
    __syncwarp();
    if (lane == 0) mbar_arrive(B.smem + L::kPFull + 8u * half);
  }
  // ---- the row's output, or its sums for the kernel that joins them
  if (n > 0) {
    if (!wait_inline(B, B.smem + L::kSFull + 8u * half, (uint32_t)n & 1u)) return;
    tc_fence_after();
  }
  const bool blind = limit < 0 || n == 0;
  const float back = power_of_two(e - 12), inv = B.direct ? back / l : back;
  T *out = static_cast<T *>(P.A.out) + row * P.A.r.out_stride + (long long)head * kDim;
  float *partial = B.partial + (size_t)(half * kHalf + in_tile) * kDim, *stats = B.partial + (size_t)kItemRows * kDim + 2 * (half * kHalf + in_tile);
#pragma unroll
  for (int c = 0; c < kDim / 32; ++c) {
    uint32_t o[32];
    if (n > 0) {
      tmem_ld32(O + 32u * c, o);
      tmem_wait32(o);
    }
    if (!in) continue;
#pragma unroll
    for (int j = 0; j < 32; ++j) o[j] = n > 0 && !(B.direct && blind) ? __float_as_uint(__uint_as_float(o[j]) * inv) : 0u;
    if (B.direct) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        Chunk<T> v;
        v.from_float(*reinterpret_cast<const float (*)[8]>(o + 8 * j));
        v.store(out + 32 * c + 8 * j, P.out_pieces, 8);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        reinterpret_cast<uint4 *>(partial + 32 * c)[j] = make_uint4(o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]);
    }
  }
  if (!in) return;
  if (B.direct) {
    if (P.A.lse) P.A.lse[row * P.A.r.q_heads + head] = blind ? -INFINITY : (m + log2f(l)) * kLn2;
  } else {
    stats[0] = m;
    stats[1] = l;
  }
}

template <class T, int kDim>
__global__ void __launch_bounds__(kThreads, 1)
kv4_prompt_kernel(const __grid_constant__ Params P) {
  using L = Layout<kDim>;
  extern __shared__ __align__(1024) uint8_t smem_ptr[];
  const uint32_t smem = smem_u32(smem_ptr);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(smem_ptr + L::kTmem);
  int *found = reinterpret_cast<int *>(smem_ptr + L::kItem);
  volatile int *abort_flag = reinterpret_cast<volatile int *>(smem_ptr + L::kAbort);
  if (threadIdx.x == 0) {
    for (int i = 0; i < kRawStages; ++i) { mbar_init(smem + L::kRawFull + 8u * i, 1); mbar_init(smem + L::kRawEmpty + 8u * i, 4); }
    for (int i = 0; i < kOperands; ++i) { mbar_init(smem + L::kFull + 8u * i, 4); mbar_init(smem + L::kEmpty + 8u * i, 1); }
    for (int i = 0; i < kScaleBufs; ++i) mbar_init(smem + L::kScaled + 8u * i, 4);
    for (int i = 0; i < 2; ++i) { mbar_init(smem + L::kSFull + 8u * i, 1); mbar_init(smem + L::kPFull + 8u * i, 4); mbar_init(smem + L::kQFull + 8u * i, 4); }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  // (the tensor memory is taken before any thread lets the next kernel start)
  __syncthreads();
  stream_order();
  const int split = (int)(blockIdx.x % (unsigned)P.splits), at = (int)(blockIdx.x / (unsigned)P.splits);
  if (warp == kCopyWarp) {
    const Item item = item_of(P, at / P.A.w.d.kv_heads, lane);
    if (lane == 0) { found[0] = item.b; found[1] = item.tile; found[2] = item.there; }
  } else if (warp == kMmaWarp) {
    P.T.check_lengths(P.A.w, lane, &g_status_kv4_prompt);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  Block B = {P, {}, found[0], at % P.A.w.d.kv_heads, found[1], 0, 0, false, false, smem, 0u, 0u, *tmem_slot, smem_ptr, abort_flag, nullptr};
  bool work = found[2] != 0;
  if (work) {
    B.s.load(P.A.w, P.T, B.b);
    const Span span(P, B.s, B.tile, split);
    work = split < span.splits;
    B.first = span.first;
    B.last = span.last;
    B.two = (long long)B.s.n * P.T.group - (long long)B.tile * kItemRows > kHalf;
    B.direct = span.splits == 1;
    B.q = (smem + L::kQ + 1023u) & ~1023u;
    B.operands = B.q + 2u * L::kOperand;
    B.partial = static_cast<float *>(P.A.work) + (size_t)blockIdx.x * partial_floats(kDim);
  }
  if (work) {
    if (warp < kExpandWarp) {
      asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
      softmax_role<T, kDim>(B, warp >> 2, warp & 3, lane);
    } else {
      asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
      if (B.first < B.last) {
        if (warp < kMmaWarp) {
          expand_role<T, kDim>(B, (int)threadIdx.x - 32 * kExpandWarp);
        } else if (warp == kMmaWarp) {
          if (elect_one()) mma_role<T, kDim>(B);
        } else if (warp == kCopyWarp) {
          copy_role<kDim>(B, lane);
        }
      }
      __syncwarp();
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kMmaWarp)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(B.tmem), "r"(512u) : "memory");
}

// Joins the sums of an item's blocks: a warp has a row (token and head).
constexpr int kJoinWarps = 4;
template <class T, int kDim>
__global__ void __launch_bounds__(32 * kJoinWarps)
kv4_prompt_join_kernel(const Params P) {
  const int lane = threadIdx.x & 31;
  const long long item = (long long)blockIdx.x * kJoinWarps + threadIdx.x / 32;
  stream_order();
  const int token = (int)(item / P.A.r.q_heads), head = (int)(item % P.A.r.q_heads), kv_head = head / P.T.group;
  if (token >= P.A.r.rows) return;
  int b, place;
  if (!find_sequence(P.A.w, token, lane, b, place)) return;
  Sequence s;
  s.load(P.A.w, P.T, b);
  if (s.n == 0) return;
  const long long r = (long long)(token - s.start) * P.T.group + head % P.T.group;
  const int tile = (int)(r / kItemRows), in_tile = (int)(r - (long long)tile * kItemRows);
  const Span span(P, s, tile, 0);
  if (span.splits == 1) return;
  const long long block = ((long long)rank_of(P, b, tile, lane) * P.A.w.d.kv_heads + kv_head) * P.splits;
  if (block + span.splits > P.blocks) return;              // (starts that do not rise)
  const float *work = static_cast<const float *>(P.A.work);
  auto part = [&](int i) { return work + (size_t)(block + i) * partial_floats(kDim); };
  float top = -INFINITY;
  for (int i = 0; i < span.splits; ++i) top = fmaxf(top, load_global(part(i) + (size_t)kItemRows * kDim + 2 * in_tile));
  float total = 0.0f, acc[kDim / 32] = {};
  for (int i = 0; i < span.splits; ++i) {
    const float *stats = part(i) + (size_t)kItemRows * kDim + 2 * in_tile;
    const float f = top == -INFINITY ? 0.0f : exp2_fast(load_global(stats) - top);
    total = fmaf(f, load_global(stats + 1), total);
#pragma unroll
    for (int c = 0; c < kDim / 32; ++c) acc[c] = fmaf(f, load_global(part(i) + (size_t)in_tile * kDim + lane + 32 * c), acc[c]);
  }
  const bool blind = place < 0;
  const float inv = 1.0f / total;
  T *out = static_cast<T *>(P.A.out) + token * P.A.r.out_stride + (long long)head * kDim;
#pragma unroll
  for (int c = 0; c < kDim / 32; ++c) {
    const uint32_t v = float_to_pair(blind ? 0.0f : acc[c] * inv, 0.0f, T());
    reinterpret_cast<uint16_t *>(out)[lane + 32 * c] = (uint16_t)v;
  }
  if (lane == 0 && P.A.lse) P.A.lse[(long long)token * P.A.r.q_heads + head] = blind ? -INFINITY : (top + log2f(total)) * kLn2;
}

// Items of a head, at most, and the blocks that share one: as many as fill the GPU.
struct Plan { long long items; int splits; };
Plan plan(const xnor_kv4_desc &d, const xnor_kv4_rows &r) {
  const int group = r.q_heads / d.kv_heads;
  const long long items = ((long long)r.rows * group) / kItemRows + std::min<long long>(d.seqs, r.rows);
  return {items, (int)std::min<long long>(kMaxSplits, std::max<long long>(1, (long long)kSms / (items * d.kv_heads)))};
}

template <class T, int kDim>
cudaError_t run(const Kv4Args &a, int least_rows, cudaStream_t st) {
  using L = Layout<kDim>;
  static bool flags[64] = {};
  cudaError_t e = allow_shared(kv4_prompt_kernel<T, kDim>, L::kBytes, flags);
  if (e != cudaSuccess) return e;
  const Plan p = plan(a.w.d, a.r);
  const long long blocks = p.items * a.w.d.kv_heads * p.splits;
  if (blocks > INT_MAX) return cudaErrorInvalidConfiguration;
  const Params P = {a, {a.r.q_heads / a.w.d.kv_heads, kItemRows, kTokens, a.r.rows, least_rows, INT_MAX}, blocks, p.splits,
                    rows_in_pieces(a.q, a.r.q_stride, kDim, 2), rows_in_pieces(a.out, a.r.out_stride, kDim, 2), W4Type<T>::kMagic, W4Type<__half>::kMagic};
  e = launch_kernel(kv4_prompt_kernel<T, kDim>, dim3((unsigned)blocks), kThreads, L::kBytes, st, 1, P);
  if (e != cudaSuccess || p.splits == 1) return e;
  const long long rows = (long long)a.r.rows * a.r.q_heads;
  return launch_kernel(kv4_prompt_join_kernel<T, kDim>, dim3((unsigned)((rows + kJoinWarps - 1) / kJoinWarps)), 32 * kJoinWarps, 0, st, 1, P);
}
template <class T>
cudaError_t run_type(const Kv4Args &a, int least_rows, cudaStream_t st) { return a.w.d.dim == 64 ? run<T, 64>(a, least_rows, st) : run<T, 128>(a, least_rows, st); }

// From how many rows of a sequence on the tensor cores take it.
constexpr int kFewRows = 64;

}  // namespace

size_t kv4_prompt_work_bytes(const xnor_kv4_desc &d, const xnor_kv4_rows &r) {
  const Plan p = plan(d, r);
  return p.splits == 1 ? 0 : (size_t)(p.items * d.kv_heads * p.splits) * kItemRows * (d.dim + 2) * sizeof(float);
}

cudaError_t launch_kv4_prompt(const Kv4Args &a, int least_rows, cudaStream_t st) {
  return a.r.type == XNOR_BF16 ? run_type<__nv_bfloat16>(a, least_rows, st) : run_type<__half>(a, least_rows, st);
}

cudaError_t read_status_kv4_prompt(int *status) {
  cudaError_t e = cudaMemcpyFromSymbol(status, g_status_kv4_prompt, sizeof(int));
  if (e == cudaSuccess && *status != 0) {
    const int zero = 0;
    e = cudaMemcpyToSymbol(g_status_kv4_prompt, &zero, sizeof(int));
  }
  return e;
}

// Sequences of few rows go to one kernel, those of many to the other; which there are, only the device knows, but no
// sequence has more than `most`, and one alone may have any number.
size_t kv4_work_bytes(const xnor_kv4_desc &d, const xnor_kv4_rows &r) {
  return std::max(kv4_few_work_bytes(d, r), kv4_most_rows(d, r) > kFewRows ? kv4_prompt_work_bytes(d, r) : 0);
}

cudaError_t launch_kv4_attention(const Kv4Args &a, cudaStream_t st) {
  if (a.r.rows == 0) return cudaSuccess;
  if (kv4_most_rows(a.w.d, a.r) <= kFewRows) return launch_kv4_few(a, INT_MAX, st);
  if (a.w.d.seqs == 1) return launch_kv4_prompt(a, 0, st);
  const cudaError_t e = launch_kv4_few(a, kFewRows, st);
  return e == cudaSuccess ? launch_kv4_prompt(a, kFewRows, st) : e;
}

}  // namespace xnor
