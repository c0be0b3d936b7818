// Attention over the cache in 4 bits for few new tokens of a sequence: warp-level products, the context shared out over
// the GPU, and joined.
//
// A unit of work is a record (16 tokens of a head) for a tile of rows (queries of that head's group).  The units of all
// sequences, heads and tiles stand in one row, and every block takes an equal share of it, found on the device from the
// lengths; so a batch of any lengths keeps all SMs reading.  The tokens are the matrix operand (16 rows of m16n8k16) and the
// queries, up to 8 kTiles of them, the other: S^T = K Q^T, then O^T += V^T P^T, whose codes - zero come straight from
// a record's words, exactly, as F16 (whose expansion takes two instructions in eleven fewer than bfloat16's; so queries in bfloat16
// become F16, times a power of two).  A key's scale multiplies its row of S^T, a value's its row of P^T, which a matrix transposition
// within the warp (movmatrix) makes the second operand.  The softmax is one pass: a running maximum, raised (and
// the sums rescaled) only when it is exceeded by more than 2^8, and sums in fp32.
//
// A block: one warp copies records into a ring in shared memory, a thread a stage, and seven warps take every
// seventh unit each; at an item's end (the units of a tile) they add their sums.  An item that lies in
// several blocks' shares leaves partial sums in the workspace, which a second kernel joins.
//
// 64 sequences of 300 to 8192 tokens, 8 heads of 128 with four queries each: 88 us with the join (294 MB, 0.51 of a copy's rate), at
// 2.5 instructions per clock, half of the ALU's: the expansion of the codes and the softmax, 390 instructions a record of 4096 codes.  Single
// tokens of short batches are latency: 5000 tokens 12.9 us with the join.  Two blocks per SM: one of 14 warps took 130 us (they
// meet at every item's end), three spilled, 146.
#include <algorithm>
#include <climits>
#include <type_traits>

#include "kv4_attention.cuh"

namespace xnor {

__device__ int g_status_kv4_few = 0;

namespace {

using namespace umma;

// Seven computing warps and one that copies: 256 threads, so that two blocks have 128 registers a thread.
constexpr int kWarps = 7, kTurns = 4, kStages = kTurns * kWarps;      // kTurns: stages of a warp
constexpr int per_sm(int tiles) { return tiles == 1 ? 2 : 1; }          // blocks: by their registers
constexpr int kMaxWorkers = 2 * 160;         // blocks, at most (a B200 has 148 SMs)
constexpr int kLeastUnits = 3 * kWarps;      // of a block's share, where items are few: us for 14, 21, 28 with one sequence of 1000 tokens, 8 heads, 11.2 12.2 13.0, of 5000 15.2 13.3 14.0

// Shares are cut in a row in which an item has kEnd places more than units, before its first: its end, where the warps meet, and its
// start take a block about as long as so many units.  us for 0, 10, 24, 36, 56: 64 sequences of 300 to 8192 tokens
// 101 99 90.8 89.6 91.8; 16 of up to 1500, whole step, 26.4 23.1 22.2 22.4 23.3; one of 5000 17.1 15.4 15.3 15.5 15.6.
constexpr int kEnd = 32;

// What the threads of a warp know of the row: each the sums over its own run of sequences, and before them, of units and of places.
struct Row {
  int per;                     // sequences of a thread
  long long before, total;     // units
  long long places_before, places;
  long long workers;
  Sequence own;                // with one sequence a thread: that
  __device__ __forceinline__ static long long places_of(const Sequence &s, int kv_heads) { return (long long)kv_heads * s.tiles * (s.units + kEnd); }
  __device__ __forceinline__ Row(const Kv4Where &W, const Tiling &T, int lane, int most) {
    per = (W.d.seqs + 31) / 32;
    long long mine = 0, my_places = 0;
#pragma unroll 4
    for (int i = 0; i < per; ++i) {
      const int b = lane * per + i;
      if (b >= W.d.seqs) break;
      own.load(W, T, b);
      mine += own.all(W.d.kv_heads);
      my_places += places_of(own, W.d.kv_heads);
    }
    long long sum = mine, place_sum = my_places;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
      const long long v = __shfl_up_sync(0xffffffffu, sum, o), w = __shfl_up_sync(0xffffffffu, place_sum, o);
      if (lane >= o) { sum += v; place_sum += w; }
    }
    before = sum - mine;
    total = __shfl_sync(0xffffffffu, sum, 31);
    places_before = place_sum - my_places;
    places = __shfl_sync(0xffffffffu, place_sum, 31);
    workers = max(1ll, min((long long)most, max((places - total) / kEnd, total / kLeastUnits)));      // (a block an item at least: 100 tokens 11.2 -> 8.9 us)
  }
  __device__ __forceinline__ int worker_of(long long place) const { return (int)divide((place + 1) * workers - 1, places); }
  // The places before sequence b; the same for all threads.
  __device__ __forceinline__ long long places_before_sequence(const Kv4Where &W, const Tiling &T, int b, int lane) const {
    long long v = places_before;
    if (per > 1 && lane == b / per)
      for (int i = lane * per; i < b; ++i) {
        Sequence s;
        s.load(W, T, i);
        v += places_of(s, W.d.kv_heads);
      }
    return __shfl_sync(0xffffffffu, v, b / per);
  }
  // The first unit of a worker's share (that worker's first place's, or the next one's that is a unit's), its sequence, and the units before that.
  __device__ __forceinline__ long long first_of(const Kv4Where &W, const Tiling &T, long long worker, int lane, int &b, long long &sum, Sequence &found) const {
    const long long place = divide(worker * places, workers);
    const uint32_t later = __ballot_sync(0xffffffffu, places_before > place);
    const int owner = later == 0 ? 31 : __ffs((int)later) - 2;       // the last thread with no more places before it
    long long u = before, v = places_before;
    b = lane;
    if (per > 1 && lane == owner) {
      for (b = lane * per; b + 1 < W.d.seqs; ++b) {
        Sequence s;
        s.load(W, T, b);
        const long long n = places_of(s, W.d.kv_heads);
        if (v + n > place) break;
        v += n;
        u += s.all(W.d.kv_heads);
      }
    }
    sum = __shfl_sync(0xffffffffu, u, owner);
    v = __shfl_sync(0xffffffffu, v, owner);
    b = __shfl_sync(0xffffffffu, b, owner);
    if (per > 1) found.load(W, T, b);
    else found = own.of(owner);
    const int length = found.units + kEnd;
    const long long item = divide(place - v, length);
    return sum + item * found.units + max(0, (int)(place - v - item * length) - kEnd);
  }
};

// A place in the row: item (sequence, head, tile) and record.
struct Place {
  int b, head, tile, rec;
  Sequence s;
  __device__ __forceinline__ void set(long long in_sequence) {
    const long long item = divide(in_sequence, s.units);
    rec = (int)(in_sequence - item * s.units);
    head = (int)divide(item, s.tiles);
    tile = (int)(item - (long long)head * s.tiles);
  }
};

// ---- shared memory -----------------------------------------------------------------------------------------------
template <int kDim, int kTiles>
struct Layout {
  static constexpr uint32_t kRecord = kv4_record(kDim);
  static constexpr int kRows = 8 * kTiles;
  static constexpr int kSumRow = kDim + 4;                          // floats
  static constexpr uint32_t kFull = 0, kEmpty = 8 * kStages, kValid = 16 * kStages, kAbort = kValid + 4 * kStages, kRead = kAbort + 8;
  static constexpr uint32_t kStats = 1024;                          // [kWarps][kRows] maxima and sums
  static constexpr uint32_t kSums = kStats + 8 * kWarps * kRows;    // [kWarps][kRows][kSumRow]
  static constexpr uint32_t kRing = (kSums + 4u * kWarps * kRows * kSumRow + 127u) & ~127u;
  static constexpr uint32_t kBytes = kRing + kStages * kRecord;
  static_assert(kRead % 8 == 0 && kRead + 8 <= kStats, "control words");
};

__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
// Which token of a record is row i of the products (neighbours are neighbours): keys and values then meet in the fewest banks.
__device__ __forceinline__ int token_of(int i) { return i ^ ((i >> 1) & 1); }

struct Params {
  Kv4Args A;
  Tiling T;
  int workers, q_pieces, out_words;      // q can be read in 16-byte pieces, out written in words
  uint32_t magic;              // W4Type's
};

// Waits of a warp's threads for their own barriers; false: gave up.
__device__ __forceinline__ bool wait_for(uint32_t bar, uint32_t parity, volatile int *abort_flag) {
  return mbar_wait(bar, parity, abort_flag, &g_status_kv4_few);
}

// ---- the copying warp --------------------------------------------------------------------------------------------
// Thread i fills stage i, of every kStages-th unit of the share.  It finds the next unit's record before it waits for the stage.
template <class L>
__device__ __forceinline__ void copy_role(const Params &P, long long u0, long long u1, int b0, const Sequence &s0, long long sum0, uint32_t smem,
                                          volatile int *abort_flag, int lane) {
  const Kv4Where &W = P.A.w;
  Place p;
  p.b = b0;
  p.s = s0;
  long long sum = sum0;
  struct Next { long long record; int valid; };
  auto find = [&](long long u) {
    Next n = {-1, 0};
    if (u >= u1) return n;
    while (u >= sum + p.s.all(W.d.kv_heads)) {
      sum += p.s.all(W.d.kv_heads);
      p.s.load(W, P.T, ++p.b);
    }
    p.set(u - sum);
    n.valid = min(kKvTokens, p.s.len - p.rec * kKvTokens);
    if (n.valid > 0) n.record = kv4_find(W, p.b, p.rec, p.head);
    return n;
  };
  const uint32_t full = smem + L::kFull + 8u * lane, empty = smem + L::kEmpty + 8u * lane;
  const bool mine = lane < kStages;
  Next next = find(mine ? u0 + lane : u1);
  uint32_t parity = 1u;
  bool in_flight = false, alive = true;
#pragma unroll 1
  for (long long u = u0; alive && u < u1; u += kStages, parity ^= 1u) {
    const Next now = next;
    next = find(mine ? u + lane + kStages : u1);
    // a stage of each warp at a time: the others' units stay under way meanwhile (all at once the ring ran empty: 107 us for
    // 64 sequences of up to 8192 tokens)
#pragma unroll 1
    for (int turn = 0; alive && turn < kTurns; ++turn) {
      if (lane / kWarps == turn && mine && u + lane < u1) {
        alive = mbar_wait_relaxed(empty, parity, abort_flag, &g_status_kv4_few, 100);     // (the issue slots are the others')
        if (alive) {
          const bool there = now.record >= 0;
          if (!there && now.valid > 0) record_bounds(&g_status_kv4_few);
          asm volatile("st.shared.b32 [%0], %1;" ::"r"(smem + L::kValid + 4u * lane), "r"(there ? now.valid : 0) : "memory");
          if (there) {
            mbar_arrive_expect_tx(full, L::kRecord);
            bulk_copy_g2s(smem + L::kRing + (uint32_t)lane * L::kRecord, P.A.cache + (size_t)now.record * L::kRecord, L::kRecord, full);
          } else {
            mbar_arrive(full);
          }
          in_flight = there;
        }
      }
      alive = __all_sync(0xffffffffu, alive);
    }
  }
  // gave up: the copies in flight must land before the block's shared memory is released
  if (!alive && in_flight) {
    const long long t0 = clock64();
    while (clock64() - t0 < (1 << 20)) {}
  }
}

// ---- the computing warps -----------------------------------------------------------------------------------------
__device__ __forceinline__ void block_sync() { asm volatile("bar.sync 1, %0;" ::"n"(32 * kWarps) : "memory"); }

// A row of the tile: where its query and its outputs are; -1: none.
struct TileRow {
  long long q, out;
  long long lse;
  int limit;                   // the last token that it sees; below 0: none
  bool in;
  __device__ __forceinline__ TileRow(const Params &P, const Place &p, int rows, int i, int dim) {
    const int r = p.tile * rows + i, token = r / P.T.group, head = p.head * P.T.group + r % P.T.group;
    in = token < p.s.n;
    q = (p.s.start + token) * P.A.r.q_stride + (long long)head * dim;
    out = (p.s.start + token) * P.A.r.out_stride + (long long)head * dim;
    lse = (long long)(p.s.start + token) * P.A.r.q_heads + head;
    limit = p.s.lead + p.s.start + token;
  }
};

// A warp's row of outputs, kDim / 32 columns a thread.
template <class T, int kDim>
__device__ __forceinline__ void store_row(T *row, const float (&acc)[kDim / 32], float inv, bool blind, bool words, int lane) {
#pragma unroll
  for (int c = 0; c < kDim / 64; ++c) {
    const uint32_t v = blind ? 0u : float_to_pair(acc[2 * c] * inv, acc[2 * c + 1] * inv, T());
    T *to = row + lane * (kDim / 32) + 2 * c;
    if (words) {
      *reinterpret_cast<uint32_t *>(to) = v;
    } else {
      reinterpret_cast<uint16_t *>(to)[0] = (uint16_t)v;
      reinterpret_cast<uint16_t *>(to)[1] = (uint16_t)(v >> 16);
    }
  }
}

__host__ __device__ constexpr size_t slot_floats(int rows, int dim) { return (size_t)rows * (dim + 2); }

template <class T, int kDim, int kTiles>
__device__ __forceinline__ void compute_role(const Params &P, int worker, long long u0, long long u1, int b0, const Sequence &s0, long long sum0,
                                             uint32_t smem, uint8_t *smem_ptr, volatile int *abort_flag, int warp, int lane) {
  using L = Layout<kDim, kTiles>;
  constexpr int kRows = L::kRows, kWords = kDim / 32, kVWords = kDim / 64, kMTiles = kDim / 16;      // of a thread: key words, value words of a token; tiles of O^T
  const Kv4Where &W = P.A.w;
  const int g = lane >> 2, t = lane & 3;
  float *stats = reinterpret_cast<float *>(smem_ptr + L::kStats), *sums = reinterpret_cast<float *>(smem_ptr + L::kSums);
  const float scale2 = P.A.r.scale * kLog2e;
  const int tok0 = token_of(g), tok1 = tok0 + 8;                           // this thread's rows of S^T
  const int pair = token_of(2 * t);                                        // and of P^T: this, its neighbour, and eight on
  Place p;
  p.b = b0;
  p.s = s0;
  long long u = u0, sum = sum0;
  bool alive = true;
  uint32_t read = 1u;                                                      // parity of kRead's next phase to wait for; at first there is nothing to
  uint32_t use = 0u;                                                       // units that this warp has had: unit warp + kWarps use of the share is next
  const uint32_t turned = t & 1 ? 0x1054u : 0x5410u;                       // (tokens 2 t and 2 t + 1 are the other way round there)
  while (u < u1) {
    while (u >= sum + p.s.all(W.d.kv_heads)) {
      sum += p.s.all(W.d.kv_heads);
      p.s.load(W, P.T, ++p.b);
    }
    p.set(u - sum);
    const int rec_end = (int)min((long long)p.s.units, p.rec + (u1 - u));
    // Q: thread (g, t) has row g's columns kDim / 4 t .., as its words of keys have them
    uint32_t q[kTiles][kWords][4];
    int limit[kTiles][2], least = 0x7FFFFFFF;
    float row_scale[kTiles][2];                                            // of logits: scale, log2 e and what the query was multiplied by
#pragma unroll
    for (int n = 0; n < kTiles; ++n) {
      const TileRow r(P, p, kRows, 8 * n + g, kDim);
      Chunk<T> c[kWords];
#pragma unroll
      for (int w = 0; w < kWords; ++w) c[w].load(static_cast<const T *>(P.A.q) + r.q + t * (kDim / 4) + 8 * w, P.q_pieces, r.in ? 8 : 0);
      float lifted = 1.0f;
      if constexpr (std::is_same<T, __nv_bfloat16>::value) {
        // bfloat16 as F16, times a power of two that brings the row's largest value to 2^14: exact but for values below 2^-31 of that
        uint32_t top = 0u;                                                 // (bit patterns of magnitudes; infinity and NaN stay what they are)
#pragma unroll
        for (int w = 0; w < kWords; ++w)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t lo = c[w].w[i] & 0x7FFFu, hi = c[w].w[i] >> 16 & 0x7FFFu;
            top = max(top, max(lo < 0x7F80u ? lo : 0u, hi < 0x7F80u ? hi : 0u));
          }
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const int up = min(126, max(-112, 14 - ((int)(top >> 7) - 127)));
        const float f = power_of_two(up);
        lifted = power_of_two(-up);
#pragma unroll
        for (int w = 0; w < kWords; ++w)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float2 v = pair_to_float(c[w].w[i], T());
            q[n][w][i] = float_to_pair(v.x * f, v.y * f, __half());
          }
      } else {
#pragma unroll
        for (int w = 0; w < kWords; ++w)
#pragma unroll
          for (int i = 0; i < 4; ++i) q[n][w][i] = c[w].w[i];
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) row_scale[n][i] = scale2 * __shfl_sync(0xffffffffu, lifted, 4 * (2 * t + i));
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const TileRow s(P, p, kRows, 8 * n + 2 * t + i, kDim);
        limit[n][i] = s.in ? s.limit : 0x7FFFFFFF;                         // (rows that do not exist compute something)
        least = min(least, limit[n][i]);
      }
    }
    least = __reduce_min_sync(0xffffffffu, least);
    // sums, a row's maximum so far, 0 where nothing was seen (`settled`: all of the warp's rows have one), and the sum of its weights
    float o[kTiles][kMTiles][4], m[kTiles][2], l[kTiles][2];
    uint32_t unset = (1u << (2 * kTiles)) - 1u;
    bool settled = false;
    // 2^(kLift - e), 2^e above the scales of the values that the row has seen: of each row, for the tokens behind it may have any (up to
    // the first record that is masked all rows have seen the same); and the least 2^e (0: not known)
    float lift[kTiles][2], largest = 0.0f;
#pragma unroll
    for (int n = 0; n < kTiles; ++n) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        m[n][i] = l[n][i] = 0.0f;
        lift[n][i] = power_of_two(kLift - kLeastScale);
      }
#pragma unroll
      for (int j = 0; j < kMTiles; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[n][j][i] = 0.0f;
    }
    // every kWarps-th unit of the share is this warp's
    const int skip = (int)((warp + kWarps - (u - u0) % kWarps) % kWarps);
#pragma unroll 1
    for (int rec = p.rec + skip; alive && rec < rec_end; rec += kWarps, ++use) {
      const uint32_t stage = (uint32_t)warp + kWarps * (use % kTurns), base = smem + L::kRing + stage * L::kRecord;
      alive = __all_sync(0xffffffffu, wait_for(smem + L::kFull + 8u * stage, (use / kTurns) & 1u, abort_flag));
      if (!alive) break;
      // all of the record that this thread needs
      const int valid = (int)lds32(smem + L::kValid + 4u * stage);
      const uint32_t kw0 = lds32(base + kv4_words(kDim, false) + 4u * tok0), kw1 = lds32(base + kv4_words(kDim, false) + 4u * tok1);
      const uint32_t vw0 = lds32(base + kv4_words(kDim, true) + 4u * tok0), vw1 = lds32(base + kv4_words(kDim, true) + 4u * tok1);
      uint32_t c0[kWords], c1[kWords];
      {
        const uint32_t from = base + (uint32_t)(t * (kDim / 8));
        if constexpr (kWords == 4) {
          lds128(from + tok0 * (kDim / 2), c0);
          lds128(from + tok1 * (kDim / 2), c1);
        } else {
          lds64(from + tok0 * (kDim / 2), c0[0], c0[1]);
          lds64(from + tok1 * (kDim / 2), c1[0], c1[1]);
        }
      }
      // ---- S^T
      // (two chains of products: one waits eight times for a product of 30 cycles and more)
      float s[kTiles][4], s2[kTiles][4];
#pragma unroll
      for (int n = 0; n < kTiles; ++n)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[n][j] = s2[n][j] = 0.0f;
      {
        const W4Type<__half>::Zero z0 = W4Type<__half>::zero(kw0 & 15u), z1 = W4Type<__half>::zero(kw1 & 15u);
#pragma unroll
        for (int w = 0; w < kWords; ++w) {
          uint32_t e0[4], e1[4];
          W4Type<__half>::expand(c0[w], z0, P.magic, e0);
          W4Type<__half>::expand(c1[w], z1, P.magic, e1);
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const uint32_t a[4] = {e0[2 * k], e1[2 * k], e0[2 * k + 1], e1[2 * k + 1]};
#pragma unroll
            for (int n = 0; n < kTiles; ++n) mma16816(k == 0 ? s[n] : s2[n], a, q[n][w][2 * k], q[n][w][2 * k + 1]);
          }
        }
      }
      uint32_t c[2][2][kVWords], zeros[2];                                 // (under way during the softmax)
      {
        const uint32_t codes = base + kv4_codes(kDim, true) + (uint32_t)(g * (kDim / 16));
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int ta = pair + 8 * h, tb = (pair ^ 1) + 8 * h;
          if constexpr (kVWords == 2) {
            lds64(codes + ta * (kDim / 2), c[h][0][0], c[h][0][1]);
            lds64(codes + tb * (kDim / 2), c[h][1][0], c[h][1][1]);
          } else {
            c[h][0][0] = lds32(codes + ta * (kDim / 2));
            c[h][1][0] = lds32(codes + tb * (kDim / 2));
          }
          uint32_t wa, wb;
          lds64(base + kv4_words(kDim, true) + 32u * h + 8u * t, wa, wb);
          zeros[h] = __byte_perm(wa, wb, turned) & 0x000F000Fu;
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(smem + L::kEmpty + 8u * stage);
      // ---- the softmax: s[n][0], [1]: token tok0 for rows 2 t, 2 t + 1; [2], [3]: token tok1
      const float ks0 = kv4_scale(kw0), ks1 = kv4_scale(kw1);
      float vs0 = kv4_scale(vw0), vs1 = kv4_scale(vw1);
      float over = -INFINITY, x[kTiles][4];
      const int p0 = rec * kKvTokens;
      const bool masked = valid < kKvTokens || p0 + kKvTokens - 1 > least;
#pragma unroll
      for (int n = 0; n < kTiles; ++n)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[n][j] = (s[n][j] + s2[n][j]) * row_scale[n][j & 1] * (j < 2 ? ks0 : ks1);
      if (masked) {
#pragma unroll
        for (int n = 0; n < kTiles; ++n)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int tok = j < 2 ? tok0 : tok1;
            if (tok >= valid || p0 + tok > limit[n][j & 1]) s[n][j] = -INFINITY;
          }
      }
#pragma unroll
      for (int n = 0; n < kTiles; ++n)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          x[n][j] = s[n][j] - m[n][j & 1];
          over = fmaxf(over, x[n][j]);
        }
      if (!settled || __any_sync(0xffffffffu, over > kRaise || fmaxf(vs0, vs1) > largest)) {
        const float lift0 = power_of_two(kLift - scale_above(vs0)), lift1 = power_of_two(kLift - scale_above(vs1));
        float most = 0.0f;
#pragma unroll
        for (int n = 0; n < kTiles; ++n)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            float top = fmaxf(s[n][i], s[n][i + 2]), f = 1.0f, now = lift[n][i];
            if (!masked || s[n][i] != -INFINITY) now = fminf(now, lift0);
            if (!masked || s[n][i + 2] != -INFINITY) now = fminf(now, lift1);
#pragma unroll
            for (int y = 4; y < 32; y *= 2) {
              top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, y));
              now = fminf(now, __shfl_xor_sync(0xffffffffu, now, y));
            }
            const float down = now * inverse_power(lift[n][i]);
            lift[n][i] = now;
            most = fmaxf(most, now);
            const uint32_t bit = 1u << (2 * n + i);
            if (unset & bit ? top > -INFINITY : top > m[n][i] + kRaise) {
              f = unset & bit ? 0.0f : exp2_fast(m[n][i] - top);
              m[n][i] = top;
              unset &= ~bit;
            }
            l[n][i] *= f;
#pragma unroll
            for (int j = 0; j < kMTiles; ++j) {
              o[n][j][i] *= f * down;
              o[n][j][i + 2] *= f * down;
            }
            x[n][i] = s[n][i] - m[n][i];
            x[n][i + 2] = s[n][i + 2] - m[n][i];
          }
        largest = power_of_two(kLift) * inverse_power(most);
        settled = __all_sync(0xffffffffu, unset == 0u);
      }
      if (!masked) {
        vs0 *= lift[0][0];
        vs1 *= lift[0][0];
      }
      uint32_t b[kTiles][2], rest[kTiles][2];                              // P^T: tokens 0 .. 7 and 8 .. 15 of the rows; what its rounding left
#pragma unroll
      for (int n = 0; n < kTiles; ++n) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          x[n][j] = exp2_fast(x[n][j]);
          l[n][j & 1] += x[n][j];
          if (!masked) x[n][j] *= j < 2 ? vs0 : vs1;
        }
        if (masked) {                                                      // (a token that is not seen may stand for anything)
#pragma unroll
          for (int j = 0; j < 4; ++j) x[n][j] = s[n][j] == -INFINITY ? 0.0f : x[n][j] * ((j < 2 ? vs0 : vs1) * lift[n][j & 1]);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t w = float_to_pair(x[n][2 * h], x[n][2 * h + 1], __half());
          b[n][h] = transpose8x8(w);
          if constexpr (kTwoParts<T>) {
            const float2 f = pair_to_float(w, __half());
            rest[n][h] = transpose8x8(float_to_pair(x[n][2 * h] - f.x, x[n][2 * h + 1] - f.y, __half()));
          }
        }
      }
      // ---- O^T: thread (g, t) has columns kDim / 8 g .. of tokens 2 t, 2 t + 1 and 8 more
      {
        using V = W4Type<__half>;
        V::Zero z[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) z[h] = {P.magic | zeros[h], 0xD400D400u | zeros[h] << 4};
#pragma unroll
        for (int w = 0; w < kVWords; ++w) {
          uint32_t v[2][2][4];                                             // [half of the tokens][even, odd columns][pairs]
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            V::expand(__byte_perm(c[h][0][w], c[h][1][w], 0x5410), z[h], P.magic, v[h][0]);
            V::expand(__byte_perm(c[h][0][w], c[h][1][w], 0x7632), z[h], P.magic, v[h][1]);
          }
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint32_t a[4] = {v[0][0][k], v[0][1][k], v[1][0][k], v[1][1][k]};
#pragma unroll
            for (int n = 0; n < kTiles; ++n) {
              mma16816(o[n][4 * w + k], a, b[n][0], b[n][1]);
              if constexpr (kTwoParts<T>) mma16816(o[n][4 * w + k], a, rest[n][0], rest[n][1]);
            }
          }
        }
      }
    }
#pragma unroll
    for (int n = 0; n < kTiles; ++n)
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (unset >> (2 * n + i) & 1u) m[n][i] = -INFINITY;
    // ---- the warps' sums together
    // (all have read the last item's; who gives up goes on to the next meeting all the same)
    if (!wait_for(smem + L::kRead, read, abort_flag)) alive = false;
    read ^= 1u;
#pragma unroll
    for (int n = 0; n < kTiles; ++n)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float back = inverse_power(lift[n][i]);
#pragma unroll
        for (int x = 4; x < 32; x *= 2) l[n][i] += __shfl_xor_sync(0xffffffffu, l[n][i], x);
        const int r = 8 * n + 2 * t + i;
        if (g == 0) {
          stats[2 * (warp * kRows + r)] = m[n][i];
          stats[2 * (warp * kRows + r) + 1] = l[n][i];
        }
        float *to = sums + (size_t)(warp * kRows + r) * L::kSumRow + g * (kDim / 8);
#pragma unroll
        for (int w = 0; w < kVWords; ++w)
#pragma unroll
          for (int k = 0; k < 4; k += 2)
            *reinterpret_cast<float4 *>(to + 8 * w + 2 * k) = make_float4(back * o[n][4 * w + k][i], back * o[n][4 * w + k][i + 2], back * o[n][4 * w + k + 1][i], back * o[n][4 * w + k + 1][i + 2]);
      }
    block_sync();
    alive = *abort_flag == 0;
    const bool first = p.rec == 0, last = rec_end == p.s.units;
    float *slot = static_cast<float *>(P.A.work) + (size_t)(2 * worker + (first ? 1 : 0)) * slot_floats(kRows, kDim);
    // a warp's rows; a thread has kDim / 32 columns
#pragma unroll 1
    for (int r = warp; r < kRows; r += kWarps) {
      const TileRow at(P, p, kRows, r, kDim);
      if (!at.in) break;
      float top = -INFINITY, total = 0.0f, f[kWarps], acc[kDim / 32] = {};
#pragma unroll
      for (int i = 0; i < kWarps; ++i) top = fmaxf(top, stats[2 * (i * kRows + r)]);
#pragma unroll
      for (int i = 0; i < kWarps; ++i) {
        f[i] = top == -INFINITY ? 0.0f : exp2_fast(stats[2 * (i * kRows + r)] - top);
        total = fmaf(f[i], stats[2 * (i * kRows + r) + 1], total);
      }
#pragma unroll
      for (int i = 0; i < kWarps; ++i)
#pragma unroll
        for (int c = 0; c < kDim / 32; ++c) acc[c] = fmaf(f[i], sums[(size_t)(i * kRows + r) * L::kSumRow + lane * (kDim / 32) + c], acc[c]);
      if (first && last) {
        const bool blind = total == 0.0f;                    // no token before it, or all of them outside the cache
        const float inv = 1.0f / total;
        store_row<T, kDim>(static_cast<T *>(P.A.out) + at.out, acc, inv, blind, P.out_words, lane);
        if (lane == 0 && P.A.lse) P.A.lse[at.lse] = blind ? -INFINITY : (top + log2f(total)) * kLn2;
      } else {
#pragma unroll
        for (int c = 0; c < kDim / 32; ++c) slot[(size_t)r * kDim + lane * (kDim / 32) + c] = acc[c];
        if (lane == 0) {
          slot[(size_t)kRows * kDim + 2 * r] = top;
          slot[(size_t)kRows * kDim + 2 * r + 1] = total;
        }
      }
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(smem + L::kRead);
    u += rec_end - p.rec;
  }
}

template <class T, int kDim, int kTiles>
__global__ void __launch_bounds__(32 * (kWarps + 1), per_sm(kTiles))
kv4_few_kernel(const Params P) {
  using L = Layout<kDim, kTiles>;
  extern __shared__ __align__(128) uint8_t smem_ptr[];
  const uint32_t smem = smem_u32(smem_ptr);
  volatile int *abort_flag = reinterpret_cast<volatile int *>(smem_ptr + L::kAbort);
  const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(smem + L::kFull + 8u * i, 1);
      mbar_init(smem + L::kEmpty + 8u * i, 1);
    }
    mbar_init(smem + L::kRead, kWarps);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  stream_order();
  const Row row(P.A.w, P.T, lane, P.workers);
  if (threadIdx.x < 32) P.T.check_lengths(P.A.w, lane, &g_status_kv4_few);
  if (row.total == 0 || (long long)blockIdx.x >= row.workers) return;
  long long sum, u1 = row.total;
  Sequence first;
  int b;
  if (blockIdx.x + 1 < row.workers) u1 = row.first_of(P.A.w, P.T, blockIdx.x + 1, lane, b, sum, first);
  const long long u0 = row.first_of(P.A.w, P.T, blockIdx.x, lane, b, sum, first);
  if (warp == kWarps)
    copy_role<L>(P, u0, u1, b, first, sum, smem, abort_flag, lane);
  else
    compute_role<T, kDim, kTiles>(P, blockIdx.x, u0, u1, b, first, sum, smem, smem_ptr, abort_flag, warp, lane);
}

__device__ __forceinline__ float4 load_piece(const float4 *p) { return load_global(p); }
__device__ __forceinline__ float2 load_piece(const float2 *p) {
  const uint2 v = load_global(reinterpret_cast<const uint2 *>(p));
  return make_float2(__uint_as_float(v.x), __uint_as_float(v.y));
}

// Joins the partial sums of items that lie in several blocks' shares: a warp has a row (token and head).  limit > 0: it has row
// i < limit of a sequence and head of the cache instead, which are fewer where most tokens belong to long prompts (two of 4096
// tokens, none of them this kernel's, took 33 us).
constexpr int kJoinWarps = 4;
template <class T, int kDim>
__global__ void __launch_bounds__(32 * kJoinWarps)
kv4_join_kernel(const Params P, int rows, int limit) {
  const int lane = threadIdx.x & 31;
  const uint32_t item = blockIdx.x * kJoinWarps + threadIdx.x / 32;        // (up to 2^30)
  stream_order();
  const Kv4Where &W = P.A.w;
  int token, head, b;
  Sequence s;
  long long before;
  if (limit > 0) {
    const uint32_t of_sequence = (uint32_t)W.d.kv_heads * (uint32_t)limit, rest = item % of_sequence;
    b = (int)(item / of_sequence);
    if (b >= W.d.seqs) return;
    s.load(W, P.T, b);
    const int r = (int)(rest % (uint32_t)limit);
    if (r >= s.n * P.T.group) return;
    token = s.start + r / P.T.group;
    head = (int)(rest / (uint32_t)limit) * P.T.group + r % P.T.group;
  } else {
    token = (int)(item / (uint32_t)P.A.r.q_heads);
    head = (int)(item % (uint32_t)P.A.r.q_heads);
    if (token >= P.A.r.rows) return;
  }
  const Row row(W, P.T, lane, P.workers);
  if (limit > 0) {
    before = row.places_before_sequence(W, P.T, b, lane);
  } else if (row.per == 1) {                               // (a thread has read all of a sequence's numbers)
    const uint32_t has = __ballot_sync(0xffffffffu, lane < W.d.seqs && token >= row.own.start && token - row.own.start < row.own.n);
    if (has == 0u) return;
    b = __ffs((int)has) - 1;
    s = row.own.of(b);
    before = __shfl_sync(0xffffffffu, row.places_before, b);
  } else {
    int place;
    if (!find_sequence(W, token, lane, b, place)) return;
    s.load(W, P.T, b);
    if (s.n == 0) return;
    before = row.places_before_sequence(W, P.T, b, lane);
  }
  const long long r = (long long)(token - s.start) * P.T.group + head % P.T.group;
  const int tile = (int)divide(r, rows), at = (int)(r - (long long)tile * rows);
  const long long first = before + ((long long)(head / P.T.group) * s.tiles + tile) * (s.units + kEnd) + kEnd;
  const int w0 = row.worker_of(first), w1 = row.worker_of(first + s.units - 1);
  if (w0 == w1) return;
  const float *work = static_cast<const float *>(P.A.work);
  auto slot = [&](int w) { return work + (size_t)(2 * w + (w == w0 ? 1 : 0)) * slot_floats(rows, kDim); };
  // eight shares' loads under way at a time, the first before the maximum is known
  using Piece = std::conditional_t<kDim == 128, float4, float2>;
  Piece v[8];
  float ml[8][2], top = -INFINITY;
  auto fetch = [&](int w) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float *from = slot(min(w + i, w1));
      ml[i][0] = load_global(from + (size_t)rows * kDim + 2 * at);
      ml[i][1] = load_global(from + (size_t)rows * kDim + 2 * at + 1);
      v[i] = load_piece(reinterpret_cast<const Piece *>(from + (size_t)at * kDim) + lane);
    }
  };
  fetch(w0);
  if (w1 - w0 < 8) {
#pragma unroll
    for (int i = 0; i < 8; ++i) top = fmaxf(top, ml[i][0]);
  } else {
    for (int w = w0 + lane; w <= w1; w += 32) top = fmaxf(top, load_global(slot(w) + (size_t)rows * kDim + 2 * at));
#pragma unroll
    for (int x = 16; x > 0; x /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
  }
  float total = 0.0f, acc[kDim / 32] = {};
  for (int w = w0; w <= w1; w += 8) {
    if (w > w0) fetch(w);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (w + i > w1) continue;
      // (a share that saw nothing has zeros; one whose sums are NaN has them whatever its maximum is, which NaN does not raise)
      const float f = top == -INFINITY ? 0.0f : exp2_fast(ml[i][0] - top);
      total = fmaf(f, ml[i][1], total);
#pragma unroll
      for (int c = 0; c < kDim / 32; ++c) acc[c] = fmaf(f, reinterpret_cast<const float *>(&v[i])[c], acc[c]);
    }
  }
  const bool blind = total == 0.0f;                        // no token before it, or all of them outside the cache
  const float inv = 1.0f / total;
  store_row<T, kDim>(static_cast<T *>(P.A.out) + token * P.A.r.out_stride + (long long)head * kDim, acc, inv, blind, P.out_words, lane);
  if (lane == 0 && P.A.lse) P.A.lse[(long long)token * P.A.r.q_heads + head] = blind ? -INFINITY : (top + log2f(total)) * kLn2;
}

// Rows of a tile, in eights.  Up to eight rows: 23.5 us with one eight, 28.4 with two (16 sequences of 2000 tokens, 8 heads); 16 rows: 47 and 28.9.
int tiles_for(const xnor_kv4_desc &d, const xnor_kv4_rows &r) { return kv4_most_rows(d, r) <= 8 ? 1 : 2; }

template <class T, int kDim, int kTiles>
cudaError_t run(const Kv4Args &a, int most_rows, cudaStream_t st) {
  using L = Layout<kDim, kTiles>;
  static bool flags[64] = {};
  cudaError_t e = allow_shared(kv4_few_kernel<T, kDim, kTiles>, L::kBytes, flags);
  if (e != cudaSuccess) return e;
  const int workers = std::min(kMaxWorkers, per_sm(kTiles) * sm_count_of_current_device());
  const Params P = {a, {a.r.q_heads / a.w.d.kv_heads, L::kRows, kKvTokens, a.r.rows, 0, most_rows}, workers, rows_in_pieces(a.q, a.r.q_stride, kDim, 2), a.r.out_stride % 2 == 0, W4Type<__half>::kMagic};
  e = launch_kernel(kv4_few_kernel<T, kDim, kTiles>, dim3((unsigned)workers), 32 * (kWarps + 1), L::kBytes, st, 1, P);
  if (e != cudaSuccess) return e;
  // (by most_rows, which the kernel holds to, not by what the caller says)
  const long long rows = (long long)a.r.rows * a.r.q_heads, places = most_rows == INT_MAX ? rows : (long long)most_rows * a.w.d.kv_heads * a.w.d.seqs;
  return launch_kernel(kv4_join_kernel<T, kDim>, dim3((unsigned)((std::min(rows, places) + kJoinWarps - 1) / kJoinWarps)), 32 * kJoinWarps, 0, st, 1, P, L::kRows,
                       places < rows ? most_rows : 0);
}
template <class T>
cudaError_t run_type(const Kv4Args &a, int most_rows, cudaStream_t st) {
  const int tiles = tiles_for(a.w.d, a.r);
  if (a.w.d.dim == 64) return tiles == 1 ? run<T, 64, 1>(a, most_rows, st) : run<T, 64, 2>(a, most_rows, st);
  return tiles == 1 ? run<T, 128, 1>(a, most_rows, st) : run<T, 128, 2>(a, most_rows, st);
}

}  // namespace

size_t kv4_few_work_bytes(const xnor_kv4_desc &d, const xnor_kv4_rows &r) {
  return 2 * (size_t)kMaxWorkers * slot_floats(8 * tiles_for(d, r), d.dim) * sizeof(float);
}

cudaError_t read_status_kv4_few(int *status) {
  cudaError_t e = cudaMemcpyFromSymbol(status, g_status_kv4_few, sizeof(int));
  if (e == cudaSuccess && *status != 0) {
    const int zero = 0;
    e = cudaMemcpyToSymbol(g_status_kv4_few, &zero, sizeof(int));
  }
  return e;
}

cudaError_t launch_kv4_few(const Kv4Args &a, int most_rows, cudaStream_t st) {
  return a.r.type == XNOR_BF16 ? run_type<__nv_bfloat16>(a, most_rows, st) : run_type<__half>(a, most_rows, st);
}

}  // namespace xnor
