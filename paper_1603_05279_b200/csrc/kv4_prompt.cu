// Attention over the cache in 4 bits for many new tokens of a sequence, on the 5th-generation tensor cores.
//
// A block computes one item: up to 256 rows (queries of a head's group, token by token) in two halves of 128, over their
// context in tiles of 128 tokens, 64 at a step.  S = Q K^T (128 x 64) and O += P V run on tcgen05.mma kind::f16 with fp32 sums in tensor
// memory: two S and an O of both halves fill it, and P, in F16 (in one part or two), lies where S lay.  Two S, so that the products of a step run while the
// softmax is busy with another (one S of 128 tokens left the tensor cores idle while both halves weighed: 545 us for two
// prompts of 4096 tokens).  Keys and values become code - zero, exactly, in shared
// memory; a key's scale multiplies its column of S, a value's its column of P (rounded to F16 as in the kernel for few
// rows).  The softmax is one pass with a running maximum that may be left behind by 2^8, so that O is rescaled rarely.
//
// Warps: 0 - 7  softmax of 32 rows each, whose queries they bring and whose output they take away
//        8 - 11 keys from 4-bit records into operands of 128 tokens (three stages); 12 - 15 values
//        16     issues the products
//        17     copies records into a ring in shared memory, a thread a record
//        18     the columns' scales, and what the values' are rounded by (done by the warps of keys, which others wait for: 437 us for 394)
// Steps that all of an item's rows see whole, and those with masked tokens, are two loops: in the latter each row has a power of two of its
// own that P is rounded by, for it must not go by tokens that the row does not see (as one loop, whose registers did not do: 419 us for 408
// for two prompts of 4000 tokens and 30 single ones; one prompt of 128 tokens, which has no other steps, takes 1 us more than when
// rows shared it).
// Two prompts of 4096 tokens, 32 heads of 128 on 8: 393 us with the other kernel's launches, 684 TFLOP/s of what is not masked, 0.40 of a matrix product's rate; the tensor
// pipe is busy 33 % of the time.  When it took 427 an item of two halves took 2800 clocks for 128 tokens, of which the products alone would take
// 1600, and 27,000 before its first and after its last (its place, its queries, the first records, its output).  Tried: turns of the
// halves by barriers 583 us against 470 at the time, one block that goes on from item to item 582 (it spills), two chains of products no change.
// Where there are too few items for the GPU, the blocks of an item divide its context, and a second kernel joins
// their sums.  Every wait is bounded; on expiry the block records XNOR_ERR_TIMEOUT, stops and frees its tensor memory.
#include <algorithm>
#include <climits>
#include <type_traits>

#include "kv4_attention.cuh"

namespace xnor {

__device__ int g_status_kv4_prompt = 0;

namespace {

using namespace umma;

constexpr int kHalf = 128, kItemRows = 2 * kHalf;
constexpr int kTokens = 128, kRecords = kTokens / kKvTokens;     // of a tile
constexpr int kStep = 64, kStepRecords = kStep / kKvTokens;
constexpr int kOperands = 3, kRawStages = 2, kScaleBufs = 4;
constexpr int kKeyWarp = 8, kValueWarp = 12, kMmaWarp = 16, kCopyWarp = 17, kScaleWarp = 18, kThreads = 20 * 32;
constexpr int kSoftmaxRegs = 144, kOtherRegs = 64, kLaunchRegs = 96;
static_assert(kKeyWarp * 32 * kSoftmaxRegs + (kThreads - kKeyWarp * 32) * kOtherRegs <= kThreads * kLaunchRegs, "registers");
constexpr int kMaxSplits = 8;

template <int kDim>
struct Layout {
  static constexpr uint32_t kOperand = kTokens * kDim * 2;       // also of 128 queries
  static constexpr uint32_t kRaw = kRecords * kv4_record(kDim);
  static constexpr uint32_t kRawFull = 0, kRawEmpty = kRawFull + 8 * kRawStages, kFull = kRawEmpty + 8 * kRawStages, kEmpty = kFull + 8 * kOperands;
  static constexpr uint32_t kSFull = kEmpty + 8 * kOperands, kPFull = kSFull + 32, kODone = kPFull + 32, kLast = kODone + 16, kQFull = kLast + 16;      // [half][S]
  static constexpr uint32_t kScaled = kQFull + 16, kTmem = kScaled + 8 * kScaleBufs, kAbort = kTmem + 4, kItem = kAbort + 4, kMask = kItem + 48, kExponent = kMask + 4 * kRawStages;
  static constexpr uint32_t kThere = kExponent + 8 * kScaleBufs;
  static constexpr uint32_t kScales = 512, kUpTo = kScales + kScaleBufs * 2 * kTokens * 4, kRing = kUpTo + kScaleBufs * kTokens * 4;
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
  int tiles, splits, first, last, steps;
  Span() = default;
  __device__ __forceinline__ Span(const Params &P, const Sequence &s, int tile, int split) {
    const int last_token = (min(s.n * P.T.group, (tile + 1) * kItemRows) - 1) / P.T.group;
    const int seen = min(s.len, max(0, s.lead + s.start + last_token + 1));            // tokens that any of its rows sees
    tiles = (seen + kTokens - 1) / kTokens;
    splits = min(P.splits, max(1, tiles / 4));
    first = tiles / splits * split + min(split, tiles % splits);
    last = first + tiles / splits + (split < tiles % splits ? 1 : 0);
    steps = (min(last * kTokens, seen) - first * kTokens + kStep - 1) / kStep;
  }
};

__device__ __forceinline__ size_t partial_floats(int dim) { return (size_t)kItemRows * (dim + 2); }

struct Block {                // what all roles know
  const Params &P;
  Sequence s;
  int b, head, tile, first, last, steps;
  int whole;                  // steps, from the first on, whose tokens all of the item's rows see
  bool two, direct;           // both halves have rows; the block has the whole context
  uint32_t smem, q, operands;
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
    if (!wait_warp(B, B.smem + L::kRawEmpty + 8u * slot, parity ^ 1u)) return;
    const uint32_t there = __ballot_sync(0xffffffffu, now >= 0);
    if (now == -1) record_bounds(&g_status_kv4_prompt);
    if (lane == 0) {
      sts32(B.smem + L::kMask + 4u * slot, there);
      mbar_arrive_expect_tx(full, (uint32_t)__popc(there) * kv4_record(kDim));
    }
    __syncwarp();
    if (now >= 0)
      bulk_copy_g2s(B.smem + L::kRing + slot * L::kRaw + (uint32_t)lane * kv4_record(kDim), P.A.cache + (size_t)now * kv4_record(kDim), kv4_record(kDim), full);
  }
}

// Exponents of powers of two above values' scales, of a thread's four rows: a signed byte each.
__device__ __forceinline__ constexpr uint32_t four_times(int e) { return ((uint32_t)e & 255u) * 0x01010101u; }
__device__ __forceinline__ int exponent(uint32_t e, int row) { return (int)(int8_t)(e >> (8 * row)); }

// ---- scales --------------------------------------------------------------------------------------------------------
// The columns' scales, four tokens a thread.  The values' are given relative to a power of two 2^e above the largest so far, in a step that
// all rows see whole; of others they are as they are in the cache, with the exponent up to each token beside them, and a row takes
// that of the last token that it sees.  (Buffers are free: a tile's records come after the values of the tile four before it were used.)
template <int kDim>
__device__ __forceinline__ void scale_role(const Block &B, int lane) {
  using L = Layout<kDim>;
  const float scale2 = B.P.A.r.scale * kLog2e;
  int e = kLeastScale;
#pragma unroll 1
  for (int t = B.first; t < B.last; ++t) {
    const int i = t - B.first;
    const uint32_t slot = (uint32_t)i % kRawStages, buf = (uint32_t)i % kScaleBufs;
    if (!wait_warp(B, B.smem + L::kRawFull + 8u * slot, (uint32_t)(i / kRawStages) & 1u)) return;
    const uint32_t there = lds32(B.smem + L::kMask + 4u * slot);
    const uint32_t words = B.smem + L::kRing + slot * L::kRaw + (uint32_t)(lane / 4) * kv4_record(kDim) + 16u * (lane % 4);
    uint32_t k[4], v[4], upto[4];
    lds128(words + kv4_words(kDim, false), k);
    lds128(words + kv4_words(kDim, true), v);
    int above = kLeastScale;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool in = (there >> (lane / 4) & 1u) && t * kTokens + 4 * lane + j < B.s.len;
      k[j] = in ? __float_as_uint(kv4_scale(k[j]) * scale2) : 0u;
      v[j] = in ? __float_as_uint(kv4_scale(v[j])) : 0u;
      above = max(above, scale_above(__uint_as_float(v[j])));
      upto[j] = (uint32_t)above;
    }
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
      const int x = __shfl_up_sync(0xffffffffu, above, o);
      if (lane >= o) above = max(above, x);
    }
    const int x = __shfl_up_sync(0xffffffffu, above, 1), before = lane > 0 ? max(e, x) : e;
#pragma unroll
    for (int j = 0; j < 4; ++j) upto[j] = (uint32_t)max((int)upto[j], before);
    const int half = max(e, __shfl_sync(0xffffffffu, above, 15));
    e = max(e, __shfl_sync(0xffffffffu, above, 31));
    const bool first = 2 * i < B.whole, second = 2 * i + 1 < B.whole;
    const int e0 = second ? e : half;
    const float lift = lane < 16 ? (first ? power_of_two(kLift - e0) : 1.0f) : second ? power_of_two(kLift - e) : 1.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = __float_as_uint(__uint_as_float(v[j]) * lift);
    const uint32_t to = B.smem + L::kScales + 4u * (2u * buf * kTokens + 4u * lane);
    sts128(to, k[0], k[1], k[2], k[3]);
    sts128(to + 4u * kTokens, v[0], v[1], v[2], v[3]);
    sts128(B.smem + L::kUpTo + 4u * (buf * kTokens + 4u * lane), upto[0], upto[1], upto[2], upto[3]);
    if (lane == 0) {
      sts32(B.smem + L::kExponent + 8u * buf, (uint32_t)e0);
      sts32(B.smem + L::kExponent + 8u * buf + 4u, (uint32_t)e);
      sts32(B.smem + L::kThere + 4u * buf, there);
    }
    __syncwarp();
    if (lane == 0) {
      mbar_arrive(B.smem + L::kScaled + 8u * buf);
      mbar_arrive(B.smem + L::kRawEmpty + 8u * slot);
    }
  }
}

// ---- expansion -------------------------------------------------------------------------------------------------------
// Operands: rows of 64 values (128 bytes), swizzled in groups of eight; blocks of 64 columns one after the other.  Keys: a row is a
// token.  Values: a row is a column of O, its values tokens; so eight tokens' codes are transposed on the way, by
// choosing bytes of two tokens at a time.
template <class T, int kDim>
__device__ __forceinline__ void key_role(const Block &B, int id) {
  using L = Layout<kDim>;
  constexpr uint32_t kRecord = kv4_record(kDim);
  constexpr int kQuads = kDim / 32;                        // of words in a token's codes
  const int lane = id & 31;
#pragma unroll 1
  for (int t = B.first; t < B.last; ++t) {
    const int i = t - B.first;
    const uint32_t op = 2u * (uint32_t)i, stage = op % kOperands;
    const uint32_t slot = (uint32_t)i % kRawStages, raw = B.smem + L::kRing + slot * L::kRaw;
    if (!wait_warp(B, B.smem + L::kRawFull + 8u * slot, (uint32_t)(i / kRawStages) & 1u)) return;
    if (!wait_warp(B, B.smem + L::kEmpty + 8u * stage, ((op / kOperands) & 1u) ^ 1u)) return;
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
    if (lane == 0) {
      mbar_arrive(B.smem + L::kFull + 8u * stage);
      mbar_arrive(B.smem + L::kRawEmpty + 8u * slot);
    }
  }
}

template <int kDim>
__device__ __forceinline__ void value_role(const Block &B, int id) {
  using L = Layout<kDim>;
  using V = W4Type<__half>;
  constexpr uint32_t kRecord = kv4_record(kDim);
  constexpr int kQuads = kDim / 32;
#pragma unroll 1
  for (int t = B.first; t < B.last; ++t) {
    const int i = t - B.first;
    const uint32_t op = 2u * (uint32_t)i + 1u, stage = op % kOperands;
    const uint32_t slot = (uint32_t)i % kRawStages, raw = B.smem + L::kRing + slot * L::kRaw;
    if (!wait_warp(B, B.smem + L::kRawFull + 8u * slot, (uint32_t)(i / kRawStages) & 1u)) return;
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
    if ((id & 31) == 0) {
      mbar_arrive(B.smem + L::kFull + 8u * stage);
      mbar_arrive(B.smem + L::kRawEmpty + 8u * slot);
    }
  }
}

// ---- products ------------------------------------------------------------------------------------------------------
__device__ __forceinline__ uint64_t swizzled_desc(uint32_t addr) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | (1ull << 16) | ((uint64_t)(1024u >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
// The whole warp runs the loop, and one thread issues: so the warp's waits and fences need no second meeting.
__device__ __forceinline__ void mma_shared(uint32_t leader, uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(leader) : "memory");
}
__device__ __forceinline__ void mma_tmem(uint32_t leader, uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(leader) : "memory");
}
__device__ __forceinline__ void commit(uint32_t leader, uint32_t bar) {
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
      "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}"
      ::"r"(bar), "r"(leader) : "memory");
}
// D fp32, A and B of one 16-bit type, both K-major, M = 128.
__host__ __device__ constexpr uint32_t instruction(bool bf16, int n) {
  return (1u << 4) | ((bf16 ? 1u : 0u) << 7) | ((bf16 ? 1u : 0u) << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(kHalf >> 4) << 24);
}

template <class T, int kDim>
__device__ __forceinline__ void mma_role(const Block &B) {
  using L = Layout<kDim>;
  constexpr uint32_t kSDesc = instruction(std::is_same<T, __nv_bfloat16>::value, kStep), kODesc = instruction(false, kDim);
  const int n = B.steps, halves = B.two ? 2 : 1;
  const uint32_t leader = elect_one();
  const uint64_t q0 = swizzled_desc(B.q), op0 = swizzled_desc(B.operands);
  auto full = [&](uint32_t op) {
    const bool ok = wait_warp(B, B.smem + L::kFull + 8u * (op % kOperands), (op / kOperands) & 1u);
    tc_fence_after();
    return ok;
  };
  auto free_operand = [&](uint32_t op) { commit(leader, B.smem + L::kEmpty + 8u * (op % kOperands)); };
  // S of step j, of half h
  auto qk = [&](int h, int j) {
    const uint32_t op = (uint32_t)j & ~1u, sub = (uint32_t)j & 1u;
    if (sub == 0u && h == 0 && !full(op)) return false;
    const uint64_t queries = q0 + (uint64_t)((uint32_t)h * (L::kOperand / 16)), keys = op0 + (uint64_t)((op % kOperands) * (L::kOperand / 16) + sub * (kStep * 128 / 16));
    const uint32_t to = (uint32_t)h * kTokens + sub * kStep;
#pragma unroll
    for (int k = 0; k < kDim / 16; ++k) {
      const uint64_t step = (uint64_t)((uint32_t)(k / 4) * (kTokens * 128 / 16) + 2u * (uint32_t)(k % 4));
      mma_shared(leader, to, queries + step, keys + step, kSDesc, k > 0 ? 1u : 0u);
    }
    commit(leader, B.smem + L::kSFull + 16u * h + 8u * sub);
    if (h + 1 == halves && (sub == 1u || j + 1 == n)) free_operand(op);
    return true;
  };
  for (int h = 0; h < halves; ++h)
    if (!wait_warp(B, B.smem + L::kQFull + 8u * h, 0u)) return;
  for (int j = 0; j < min(n, 2); ++j)
    for (int h = 0; h < halves; ++h)
      if (!qk(h, j)) return;
#pragma unroll 1
  for (int j = 0; j < n; ++j) {
    const uint32_t op = (uint32_t)j | 1u, sub = (uint32_t)j & 1u;
    if (sub == 0u && !full(op)) return;
    const uint64_t values = op0 + (uint64_t)((op % kOperands) * (L::kOperand / 16) + sub * (kDim * 128 / 16));
#pragma unroll 1
    for (int h = 0; h < halves; ++h) {
      if (!wait_warp(B, B.smem + L::kPFull + 16u * h + 8u * sub, (uint32_t)(j >> 1) & 1u)) return;
      tc_fence_after();
      const uint32_t to = L::kO + (uint32_t)h * kDim, weights = (uint32_t)h * kTokens + sub * kStep;
#pragma unroll
      for (int k = 0; k < kStep / 16; ++k) mma_tmem(leader, to, weights + 8u * k, values + (uint64_t)(2 * k), kODesc, j == 0 && k == 0 ? 0u : 1u);
      if constexpr (kTwoParts<T>) {
#pragma unroll
        for (int k = 0; k < kStep / 16; ++k) mma_tmem(leader, to, weights + kStep / 2 + 8u * k, values + (uint64_t)(2 * k), kODesc, 1u);
      }
      if (j + 2 >= n) commit(leader, B.smem + (j + 1 < n ? L::kODone : L::kLast) + 8u * h);
      if (h + 1 == halves && (sub == 1u || j + 1 == n)) free_operand(op);
      if (j + 2 < n && !qk(h, j + 2)) return;              // (behind P V, whose P it overwrites)
    }
  }
}

// ---- softmax -------------------------------------------------------------------------------------------------------
// S and O leave tensor memory with two neighbouring columns of a row in a thread (rows g and g + 8 of 16, columns 2 t and
// 2 t + 1 of eight, for lane 4 g + t), and P goes back likewise: so a thread has four rows, which share the scales that it reads.
// (A row a thread took as many bytes of scales from shared memory as there are values of S, in competition with the products.)
__device__ __forceinline__ void tmem_ld_rows(uint32_t taddr, uint32_t (&r)[16]) {      // 16 rows x 32 columns
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x4.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st_rows(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.16x256b.x4.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
__device__ __forceinline__ void tmem_wait_rows(uint32_t (&r)[16]) { tmem_wait16(*reinterpret_cast<int32_t (*)[16]>(&r)); }
// P of 16 rows x 64 columns, in 32 columns of tensor memory.
__device__ __forceinline__ void tmem_st_weights(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.16x128b.x8.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

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
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(pack2(a.x, a.y)), "l"(pack2(b.x, b.y)), "l"(pack2(c.x, c.y)));
  return unpack2(r);
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(pack2(a.x, a.y)), "l"(pack2(b.x, b.y)));
  return unpack2(r);
}
__device__ __forceinline__ float2 lds_float2(uint32_t addr) {
  uint32_t a, b;
  lds64(addr, a, b);
  return make_float2(__uint_as_float(a), __uint_as_float(b));
}

// The weights of a step, against the rows' maxima m: p = exp2(s ks - m) times the values' scales, as pairs of F16; their sums before
// that; and the largest s ks - m, each of this thread's columns (2 t and 2 t + 1 of eight, of rows g, g + 8, g + 16 and g + 24 of 32;
// scales: theirs).  kCareful: records may be missing; and s ks is rounded before m is taken from it, and the largest s ks itself is
// given, so that as the maximum it gives a weight of 1 whatever its size.  kOwn: besides, columns from `seen` on (counted from 2 t)
// are not seen, and the values' scales are those of the cache, which each row takes times a power of two of its own (lifts: the exponents).
struct Scales { float2 k[kStep / 8], v[kStep / 8]; };
enum Care { kPlain, kCareful, kOwn };
// Two parts: p has what the rounding left behind the rounded weights.
template <Care kCare, int kParts>
__device__ __forceinline__ void weigh(uint32_t S, const Scales &scales, const float (&m)[4], const int (&seen)[4], uint32_t lifts, uint32_t there,
                                      uint32_t (&p)[kParts][2][16], float (&sum)[4], float (&top)[4]) {
  float2 sums[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    sums[r] = make_float2(0.0f, 0.0f);
    top[r] = -INFINITY;
  }
  uint32_t raw[2][2][16];
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    tmem_ld_rows(S + 32u * c, raw[c][0]);
    tmem_ld_rows(S + (16u << 16) + 32u * c, raw[c][1]);
  }
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    tmem_wait_rows(raw[c][0]);
    tmem_wait_rows(raw[c][1]);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int column = 32 * c + 8 * k;
      const float2 f = scales.k[4 * c + k], g = scales.v[4 * c + k];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const uint32_t *x = raw[c][r >> 1] + 4 * k + 2 * (r & 1);
        float2 u = make_float2(__uint_as_float(x[0]), __uint_as_float(x[1]));
        const int end = (there >> (column / kKvTokens) & 1u) ? (kCare == kOwn ? seen[r] : INT_MAX) : INT_MIN;
        if (kCare != kPlain) {
          u = mul2(u, f);
          if (column >= end) u.x = -INFINITY;
          if (column + 1 >= end) u.y = -INFINITY;
          top[r] = fmaxf(fmaxf(u.x, u.y), top[r]);
          u = add2(u, make_float2(-m[r], -m[r]));
        } else {
          u = fma2(u, f, make_float2(-m[r], -m[r]));
          top[r] = fmaxf(fmaxf(u.x, u.y), top[r]);
        }
        u = make_float2(exp2_fast(u.x), exp2_fast(u.y));
        sums[r] = add2(sums[r], u);
        if (kCare == kOwn) {
          const float lift = __uint_as_float((uint32_t)(exponent(lifts, r) + 127) << 23);
          u = mul2(u, make_float2(g.x * lift, g.y * lift));
        } else {
          u = mul2(u, g);
        }
        if (kCare != kPlain) {                             // (a token that is not seen may stand for anything)
          if (column >= end) u.x = 0.0f;
          if (column + 1 >= end) u.y = 0.0f;
        }
        uint32_t &w = p[0][r >> 1][2 * (4 * c + k) + (r & 1)];
        w = float_to_pair(u.x, u.y, __half());
        if constexpr (kParts == 2) {
          const float2 f = pair_to_float(w, __half());
          p[1][r >> 1][2 * (4 * c + k) + (r & 1)] = float_to_pair(u.x - f.x, u.y - f.y, __half());
        }
      }
    }
  }
#pragma unroll
  for (int r = 0; r < 4; ++r) sum[r] = sums[r].x + sums[r].y;
}

// Of four values for rows g, g + 8, .. that a thread has, the one for row `lane`.
__device__ __forceinline__ float of_row(const float (&v)[4], int lane) {
  float got = 0.0f;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const float x = __shfl_sync(0xffffffffu, v[r], 4 * (lane & 7));
    got = lane >> 3 == r ? x : got;
  }
  return got;
}

template <class T, int kDim>
__device__ __forceinline__ void softmax_role(const Block &B, int half, int quarter, int lane) {
  using L = Layout<kDim>;
  const Params &P = B.P;
  const int in_tile = 32 * quarter + lane, g = lane >> 2, t = lane & 3;
  if (half == 1 && !B.two) return;
  const int r = B.tile * kItemRows + half * kHalf + in_tile, token = r / P.T.group, head = B.head * P.T.group + r % P.T.group;
  const bool in = token < B.s.n;
  const long long row = B.s.start + token;
  const int limit = in ? min(B.s.lead + B.s.start + token, B.s.len - 1) : INT_MAX;        // the last token that the row of this lane sees
  // the queries, 64 columns a block: kDim / 8 lanes a row
  {
    constexpr int kLanes = kDim / 8, kRows = 32 / kLanes;
    const long long from = in ? row * P.A.r.q_stride + (long long)head * kDim : -1;
    const uint32_t to = B.q + (uint32_t)half * L::kOperand;
    const int c = lane % kLanes;
#pragma unroll
    for (int j = 0; j < 32 / kRows; j += 16 / (128 / kDim)) {
      constexpr int kAtOnce = 16 / (128 / kDim);
      Chunk<T> v[kAtOnce];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const long long at = __shfl_sync(0xffffffffu, from, (j + i) * kRows + lane / kLanes);
        v[i].load(static_cast<const T *>(P.A.q) + max(at, 0ll) + 8 * c, P.q_pieces, at >= 0 ? 8 : 0);
      }
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const int r = 32 * quarter + (j + i) * kRows + lane / kLanes;
        sts128(to + (uint32_t)(c / 8) * (kTokens * 128) + (uint32_t)(r * 128 + ((c & 7) ^ (r & 7)) * 16), v[i].w[0], v[i].w[1], v[i].w[2], v[i].w[3]);
      }
    }
    fence_proxy_async();
    __syncwarp();
    if (lane == 0) mbar_arrive(B.smem + L::kQFull + 8u * half);
  }
  const uint32_t lanes = (uint32_t)(32 * quarter) << 16, S = lanes + (uint32_t)(half * kTokens), O = lanes + L::kO + (uint32_t)(half * kDim);
  const int n = B.steps;
  // a row's maximum so far, 0 where it has seen nothing (`unset`: a bit for each), and the sum of its weights
  float m[4], l[4];
  int unset = 15;
  int e = kLeastScale;         // the values' scales so far are below 2^e: those of the steps that all rows see,
  uint32_t own = 0u;           // and from then on those that each row sees
#pragma unroll
  for (int j = 0; j < 4; ++j) m[j] = l[j] = 0.0f;
  bool calm = false;           // all of the warp's rows have a maximum, below 2^20 (from there on what rounding leaves of s ks - m would count)
  // Step i; false: gave up.
  auto step = [&](auto kOwnTag, int i) {
    constexpr bool kRowsOwn = decltype(kOwnTag)::value;
    const uint32_t tile = (uint32_t)(i >> 1), sub = (uint32_t)i & 1u, buf = tile % kScaleBufs;
    if (sub == 0u && !wait_inline(B, B.smem + L::kScaled + 8u * buf, (tile / kScaleBufs) & 1u)) return false;
    Scales scales;
    const uint32_t ks = B.smem + L::kScales + 4u * (2u * buf * kTokens + sub * kStep) + 8u * t;
#pragma unroll
    for (int k = 0; k < kStep / 8; ++k) {
      scales.k[k] = lds_float2(ks + 32u * k);
      scales.v[k] = lds_float2(ks + 4u * kTokens + 32u * k);
    }
    const int e_now = (int)lds32(B.smem + L::kExponent + 8u * buf + 4u * sub);
    const uint32_t there = lds32(B.smem + L::kThere + 4u * buf) >> (kStepRecords * sub) & ((1u << kStepRecords) - 1u);
    if (!wait_inline(B, B.smem + L::kSFull + 16u * half + 8u * sub, tile & 1u)) return false;
    tc_fence_after();
    const uint32_t here = S + sub * kStep;
    int seen[4] = {};
    uint32_t lifts = 0u, p[kTwoParts<T> ? 2 : 1][2][16], own_now = 0u;
    float sum[4], top[4];
    bool good = false;
    if (!kRowsOwn && calm && there == (1u << kStepRecords) - 1u && e_now == e) {
      weigh<kPlain>(here, scales, m, seen, 0u, 0u, p, sum, top);
      good = !__any_sync(0xffffffffu, fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) > kRaise);
    }
    if (!good) {
      // Where a maximum is left too far behind: that is raised, and the step weighed once more.  And steps with tokens that are missing or
      // masked: of the latter each row's powers of two are those up to its last token.
      bool moved;
      if constexpr (kRowsOwn) {
        const int t0 = B.first * kTokens + i * kStep;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int last = __shfl_sync(0xffffffffu, limit, g + 8 * j) - t0;      // in the step; below 0: none of it
          seen[j] = (last < 0 ? 0 : min(last, kStep) + 1) - 2 * t;
          const int in_tile = min(last + (int)sub * kStep, kTokens - 1);           // (the tile's, so that both of its steps have the same)
          const int v = in_tile < 0 ? exponent(own, j) : (int)lds32(B.smem + L::kUpTo + 4u * (buf * kTokens + (uint32_t)in_tile));
          own_now |= ((uint32_t)v & 255u) << (8 * j);
        }
        lifts = __vsub4(four_times(kLift), own_now);
        moved = __any_sync(0xffffffffu, own_now != own);
      } else {
        moved = e_now != e;
      }
#pragma unroll 1
      for (int attempt = 0;; ++attempt) {
        asm volatile("" : "+r"(lifts));                    // (else products with it are worked out before the loop, and spilled)
        weigh<kRowsOwn ? kOwn : kCareful>(here, scales, m, seen, lifts, there, p, sum, top);
        int up = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
#pragma unroll
          for (int x = 1; x < 4; x *= 2) top[j] = fmaxf(top[j], __shfl_xor_sync(0xffffffffu, top[j], x));
          if (top[j] > (unset >> j & 1 ? -INFINITY : m[j] + kRaise)) up |= 1 << j;
        }
        const bool again = attempt == 0 && __any_sync(0xffffffffu, up != 0);
        if (!again && !moved) break;
        float f[4];
        calm = true;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          f[j] = 1.0f;
          if (again && (up >> j & 1)) {
            f[j] = unset >> j & 1 ? 0.0f : exp2_fast(m[j] - top[j]);
            m[j] = top[j];
          }
          l[j] *= f[j];
          if (moved) f[j] *= kRowsOwn ? power_of_two(exponent(own, j) - exponent(own_now, j)) : power_of_two(e - e_now);
          calm = calm && fabsf(m[j]) < 1048576.0f;
        }
        if (again) unset &= ~up;
        calm = __all_sync(0xffffffffu, calm && unset == 0);
        if (kRowsOwn) own = own_now;
        else e = e_now;
        moved = false;
        if (i > 0) {
          // P V of the last step has to be done: the next step's S comes behind it
          if (!(i + 1 < n ? wait_inline(B, B.smem + L::kSFull + 16u * half + 8u * (sub ^ 1u), (uint32_t)((i + 1) >> 1) & 1u) : wait_inline(B, B.smem + L::kODone + 8u * half, 0u))) return false;
          tc_fence_after();
#pragma unroll 1
          for (int c = 0; c < kDim / 16; ++c) {
            const uint32_t at = O + (uint32_t)(c & 1) * (16u << 16) + 32u * (c / 2);
            const float f0 = c & 1 ? f[2] : f[0], f1 = c & 1 ? f[3] : f[1];
            uint32_t o[16];
            tmem_ld_rows(at, o);
            tmem_wait_rows(o);
#pragma unroll
            for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * (j & 2 ? f1 : f0));
            tmem_st_rows(at, o);
          }
        }
        if (!again) break;
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) l[j] += sum[j];
    tmem_st_weights(here, p[0][0]);
    tmem_st_weights(here + (16u << 16), p[0][1]);
    if constexpr (kTwoParts<T>) {
      tmem_st_weights(here + kStep / 2, p[1][0]);
      tmem_st_weights(here + kStep / 2 + (16u << 16), p[1][1]);
    }
    tmem_wait_st();
    tc_fence_before();
    __syncwarp();
    if (lane == 0) mbar_arrive(B.smem + L::kPFull + 16u * half + 8u * sub);
    return true;
  };
#pragma unroll 1
  for (int i = 0; i < B.whole; ++i)
    if (!step(std::false_type(), i)) return;
  own = four_times(e);
#pragma unroll 1
  for (int i = B.whole; i < n; ++i)
    if (!step(std::true_type(), i)) return;
  // ---- a row a thread: its output, or its sums for the kernel that joins them
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int x = 1; x < 4; x *= 2) l[j] += __shfl_xor_sync(0xffffffffu, l[j], x);
#pragma unroll
  for (int j = 0; j < 4; ++j) m[j] = unset >> j & 1 ? -INFINITY : m[j];
  float lifted[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) lifted[j] = power_of_two(exponent(own, j) - kLift);
  const float m_row = of_row(m, lane), l_row = of_row(l, lane), back = of_row(lifted, lane);
  if (n > 0) {
    if (!wait_inline(B, B.smem + L::kLast + 8u * half, 0u)) return;
    tc_fence_after();
  }
  const bool blind = l_row == 0.0f;                        // no token before it, or all of them outside the cache
  const float inv = B.direct ? back / l_row : back;
  float *partial = B.partial + (size_t)(half * kHalf + in_tile) * kDim, *stats = B.partial + (size_t)kItemRows * kDim + 2 * (half * kHalf + in_tile);
  int32_t o[kDim / 16][16];
  if (n > 0) {
#pragma unroll
    for (int c = 0; c < kDim / 16; ++c) tmem_ld16(O + 16u * c, o[c]);
#pragma unroll
    for (int c = 0; c < kDim / 16; ++c) tmem_wait16(o[c]);
  }
  const bool zero = n == 0 || (B.direct && blind);
  if (B.direct) {
    // by way of where the queries were (all products are done), so that lanes write neighbouring pieces of a row
    const uint32_t at = B.q + (uint32_t)half * L::kOperand;
#pragma unroll
    for (int c = 0; c < kDim / 8; ++c) {
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = zero ? 0.0f : __int_as_float(o[c / 2][8 * (c & 1) + j]) * inv;
      Chunk<T> w;
      w.from_float(v);
      sts128(at + (uint32_t)(c / 8) * (kTokens * 128) + (uint32_t)(in_tile * 128 + ((c & 7) ^ (in_tile & 7)) * 16), w.w[0], w.w[1], w.w[2], w.w[3]);
    }
    __syncwarp();
    constexpr int kLanes = kDim / 8, kRows = 32 / kLanes;
    const long long to = in ? row * P.A.r.out_stride + (long long)head * kDim : -1;
    const int c = lane % kLanes;
#pragma unroll
    for (int j = 0; j < 32 / kRows; ++j) {
      const int r = j * kRows + lane / kLanes;
      const long long place = __shfl_sync(0xffffffffu, to, r);
      Chunk<T> w;
      lds128(at + (uint32_t)(c / 8) * (kTokens * 128) + (uint32_t)((32 * quarter + r) * 128 + ((c & 7) ^ (r & 7)) * 16), w.w);
      if (place >= 0) w.store(static_cast<T *>(P.A.out) + place + 8 * c, P.out_pieces, 8);
    }
  } else if (in) {
#pragma unroll
    for (int c = 0; c < kDim / 4; ++c) {
      float4 v;
      v.x = zero ? 0.0f : __int_as_float(o[c / 4][4 * (c & 3)]) * inv;
      v.y = zero ? 0.0f : __int_as_float(o[c / 4][4 * (c & 3) + 1]) * inv;
      v.z = zero ? 0.0f : __int_as_float(o[c / 4][4 * (c & 3) + 2]) * inv;
      v.w = zero ? 0.0f : __int_as_float(o[c / 4][4 * (c & 3) + 3]) * inv;
      reinterpret_cast<float4 *>(partial)[c] = v;
    }
  }
  if (!in) return;
  if (B.direct) {
    if (P.A.lse) P.A.lse[row * P.A.r.q_heads + head] = blind ? -INFINITY : (m_row + log2f(l_row)) * kLn2;
  } else {
    stats[0] = m_row;
    stats[1] = l_row;
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
    for (int i = 0; i < kRawStages; ++i) { mbar_init(smem + L::kRawFull + 8u * i, 1); mbar_init(smem + L::kRawEmpty + 8u * i, 9); }
    for (int i = 0; i < kOperands; ++i) { mbar_init(smem + L::kFull + 8u * i, 4); mbar_init(smem + L::kEmpty + 8u * i, 1); }
    for (int i = 0; i < kScaleBufs; ++i) mbar_init(smem + L::kScaled + 8u * i, 1);
    for (int i = 0; i < 4; ++i) { mbar_init(smem + L::kSFull + 8u * i, 1); mbar_init(smem + L::kPFull + 8u * i, 4); }
    for (int i = 0; i < 2; ++i) { mbar_init(smem + L::kODone + 8u * i, 1); mbar_init(smem + L::kLast + 8u * i, 1); mbar_init(smem + L::kQFull + 8u * i, 4); }
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
    if (lane == 0) {
      Sequence s = {};
      Span span = {};
      if (item.there) {
        s.load(P.A.w, P.T, item.b);
        span = Span(P, s, item.tile, split);
      }
      found[0] = item.b; found[1] = item.tile; found[2] = item.there && split < span.splits && *tmem_slot == 0u;      // (all of it was taken: its addresses begin at 0)
      found[3] = s.start; found[4] = s.n; found[5] = s.len; found[6] = s.lead;
      found[7] = span.first; found[8] = span.last; found[9] = span.steps;
      found[10] = s.n * P.T.group - item.tile * kItemRows > kHalf;
      found[11] = span.splits == 1;
    }
  } else if (warp == kMmaWarp) {
    P.T.check_lengths(P.A.w, lane, &g_status_kv4_prompt);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  Block B = {P, {}, found[0], at % P.A.w.d.kv_heads, found[1], 0, 0, 0, 0, false, false, smem, 0u, 0u, smem_ptr, abort_flag, nullptr};
  const bool work = found[2] != 0;
  B.s.start = found[3]; B.s.n = found[4]; B.s.len = found[5]; B.s.lead = found[6];
  B.first = found[7]; B.last = found[8]; B.steps = found[9];
  B.whole = min(B.steps, max(0, min(B.s.lead + B.s.start + B.tile * kItemRows / P.T.group, B.s.len - 1) + 1 - B.first * kTokens) / kStep);
  B.two = found[10] != 0;
  B.direct = found[11] != 0;
  B.q = (smem + L::kQ + 1023u) & ~1023u;
  B.operands = B.q + 2u * L::kOperand;
  B.partial = static_cast<float *>(P.A.work) + (size_t)blockIdx.x * partial_floats(kDim);
  if (work) {
    if (warp < kKeyWarp) {
      asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
      softmax_role<T, kDim>(B, warp >> 2, warp & 3, lane);
    } else {
      asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
      if (B.first < B.last) {
        if (warp < kValueWarp) {
          key_role<T, kDim>(B, (int)threadIdx.x - 32 * kKeyWarp);
        } else if (warp < kMmaWarp) {
          value_role<kDim>(B, (int)threadIdx.x - 32 * kValueWarp);
        } else if (warp == kMmaWarp) {
          mma_role<T, kDim>(B);
        } else if (warp == kCopyWarp) {
          copy_role<kDim>(B, lane);
        } else if (warp == kScaleWarp) {
          scale_role<kDim>(B, lane);
        }
      }
      __syncwarp();
    }
  }
  tc_fence_before();
  __syncthreads();
  if (*abort_flag != 0) {
    // gave up: copies and products in flight must land before the block's memory is released
    const long long t0 = clock64();
    while (clock64() - t0 < (1 << 20)) {}
    __syncthreads();
  }
  if (warp == kMmaWarp)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(*tmem_slot), "r"(512u) : "memory");
}

// Joins the sums of an item's blocks: a warp has a row (token and head).
constexpr int kJoinWarps = 4;
template <class T, int kDim>
__global__ void __launch_bounds__(32 * kJoinWarps)
kv4_prompt_join_kernel(const Params P) {
  const int lane = threadIdx.x & 31;
  const uint32_t item = blockIdx.x * kJoinWarps + threadIdx.x / 32;        // (up to 2^30)
  stream_order();
  const int token = (int)(item / (uint32_t)P.A.r.q_heads), head = (int)(item % (uint32_t)P.A.r.q_heads), kv_head = head / P.T.group;
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
  const bool blind = total == 0.0f;                        // no token before it, or all of them outside the cache
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

// Up to how many rows of a sequence (new tokens x queries of a head) the kernel for few takes it: that one reads the context once
// for every 16 rows, this one once for 256.  us for 16, 32, 64, 96, 128 rows of every head, few against this:
//                                          dim 128, bfloat16                             dim 64
//   64 sequences of 4000 tokens, 8 heads   137 255 496 736 977   319 319 322 323 324     111 203 386 569 753   287 287 287 288 288
//   16 of 2000, 8 heads                     28  46  78 111 144    52  53  51  51  51      23  36  61  85 109    46  46  44  45  45
//   3 of 8000, 8 heads                      22  32  51  70  90    45  46  46  56  57      19  27  42  57  73    41  41  42  50  51   (blocks share an item)
//   1 of 4000, 8 heads                      16  17  19  23  26    21  21  22  23  24      13  14  17  19  21    19  19  19  20  20
//   4 of 1000, 4 heads                      15  15  17  20  22    25  26  28  29  29      13  13  15  16  19    23  24  26  27  26
// F16 moves both: 64 sequences 137 259 503 747 991, 364 366 368 370 372.
int few_rows(const xnor_kv4_desc &d) { return (long long)d.seqs * d.kv_heads > 16 ? 32 : 96; }

}  // namespace

size_t kv4_prompt_work_bytes(const xnor_kv4_desc &d, const xnor_kv4_rows &r) {
  // (enough for any call of fewer rows too: where blocks share items, they are no more than there are SMs)
  const long long blocks = std::min<long long>(kSms, plan(d, r).items * d.kv_heads * kMaxSplits);
  return (size_t)blocks * kItemRows * (d.dim + 2) * sizeof(float);
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
  return std::max(kv4_few_work_bytes(d, r), kv4_most_rows(d, r) > few_rows(d) ? kv4_prompt_work_bytes(d, r) : 0);
}

cudaError_t launch_kv4_attention(const Kv4Args &a, cudaStream_t st) {
  if (a.r.rows == 0) return cudaSuccess;
  const int few = few_rows(a.w.d);
  if (kv4_most_rows(a.w.d, a.r) <= few) return launch_kv4_few(a, INT_MAX, st);
  if (a.w.d.seqs == 1) return launch_kv4_prompt(a, 0, st);
  const cudaError_t e = launch_kv4_few(a, few, st);
  return e == cudaSuccess ? launch_kv4_prompt(a, few, st) : e;
}

}  // namespace xnor
