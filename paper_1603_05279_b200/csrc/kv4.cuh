// The layout of the cache in 4 bits, and the sequences in it (internal).
//
// 16 tokens of a head are a record: the keys' codes, 16 rows of dim / 2 bytes, the values', and a word for each row, 16
// of keys, 16 of values: its scale, whose last four bits are its zero point.  Records lie together by page and
// head, so that one bulk copy brings 16 tokens, whatever a page holds; and a token is written without reading.
// Codes lie in a word as those of 4-bit weights do (w4.cuh): a mask brings neighbours to where two 16-bit values have them.
#pragma once
#include "heads.cuh"
#include "w4.cuh"

namespace xnor {

constexpr int kKvTokens = 16;                // of a record
__host__ __device__ constexpr uint32_t kv4_record(int dim) { return (uint32_t)(kKvTokens * (dim + 8)); }
__host__ __device__ constexpr uint32_t kv4_codes(int dim, bool values) { return values ? (uint32_t)(8 * dim) : 0u; }
__host__ __device__ constexpr uint32_t kv4_words(int dim, bool values) { return (uint32_t)(16 * dim + (values ? 64 : 0)); }

__device__ __forceinline__ float kv4_scale(uint32_t word) { return __uint_as_float(word & ~15u); }

// What says where tokens lie.
struct Kv4Where {
  const int *starts, *lens, *table;
  xnor_kv4_desc d;
};

__device__ __forceinline__ int load_int(const int *p) { return (int)load_global(reinterpret_cast<const uint32_t *>(p)); }

// Record `rec` of sequence b (16 of its tokens), head h: its number in the cache.  -1: outside the table or the cache.
__device__ __forceinline__ long long kv4_find(const Kv4Where &W, int b, int rec, int h) {
  const int per_page = W.d.page / kKvTokens, at = rec / per_page;
  if (at >= W.d.table_cols) return -1;
  const int page = load_int(W.table + (size_t)b * W.d.table_cols + at);
  if (page < 0 || page >= W.d.pages) return -1;
  return ((long long)page * W.d.kv_heads + h) * per_page + (rec - at * per_page);
}

// The sequence of a row and the row's token in it (below 0: before its first), for all threads of a warp; false: it belongs to
// none.  Thirty-two threads look at once, and in the last round each at a whole sequence, so that up to 32 of them take one load's latency.
__device__ __forceinline__ bool find_sequence(const Kv4Where &W, int row, int lane, int &b, int &place) {
  int lo = 0, hi = W.d.seqs;                  // the first sequence that ends behind the row is in lo .. hi (hi: none)
  while (hi - lo > 32) {
    const int step = (hi - lo + 31) / 32, i = lo + (lane + 1) * step - 1;
    const bool before = i < hi && load_int(W.starts + i + 1) <= row;
    const int k = __popc(__ballot_sync(0xffffffffu, before));
    hi = min(hi, lo + (k + 1) * step - 1);
    lo = min(hi, lo + k * step);
  }
  const int i = min(lo + lane, W.d.seqs - 1);
  const int start = load_int(W.starts + i), end = load_int(W.starts + i + 1), len = max(0, load_int(W.lens + i));
  const uint32_t has = __ballot_sync(0xffffffffu, lo + lane <= hi && lo + lane < W.d.seqs && start <= row && end > row);
  // (it is one of lo .. hi; where 32 lie before hi, hi itself has no thread and is looked at by all)
  if (has == 0u) {
    if (hi - lo < 32 || hi >= W.d.seqs) return false;
    const int s = load_int(W.starts + hi), e = load_int(W.starts + hi + 1);
    b = hi;
    place = max(0, load_int(W.lens + hi)) - (e - row);
    return s <= row && e > row;
  }
  const int who = __ffs((int)has) - 1;
  b = lo + who;
  place = __shfl_sync(0xffffffffu, len - (end - row), who);
  return true;
}

struct Kv4AppendArgs {
  HeadsArgs h;                // pos is not used
  const void *v;
  Kv4Where w;
  uint8_t *cache;
};
cudaError_t launch_kv4_append(const Kv4AppendArgs &a, cudaStream_t st);
struct Kv4ReadArgs {
  const uint8_t *cache;
  Kv4Where w;
  int type, rows;
  void *k, *v;
  long long k_stride, v_stride;
};
cudaError_t launch_kv4_read(const Kv4ReadArgs &a, cudaStream_t st);
struct Kv4Args {
  const void *q;
  const uint8_t *cache;
  Kv4Where w;
  xnor_kv4_rows r;
  void *out;
  float *lse;
  void *work;
};
cudaError_t launch_kv4_attention(const Kv4Args &a, cudaStream_t st);
size_t kv4_work_bytes(const xnor_kv4_desc &d, const xnor_kv4_rows &r);
cudaError_t read_status_kv4(int *status);
// Its two kernels: of sequences with at most so many rows (new tokens x queries of a head), and of those with more.
cudaError_t launch_kv4_few(const Kv4Args &a, int most_rows, cudaStream_t st);
size_t kv4_few_work_bytes(const xnor_kv4_desc &d, const xnor_kv4_rows &r);
cudaError_t read_status_kv4_few(int *status);
cudaError_t launch_kv4_prompt(const Kv4Args &a, int least_rows, cudaStream_t st);
size_t kv4_prompt_work_bytes(const xnor_kv4_desc &d, const xnor_kv4_rows &r);
cudaError_t read_status_kv4_prompt(int *status);
// Rows of a sequence, at most, as far as the caller knows.
inline long long kv4_most_rows(const xnor_kv4_desc &d, const xnor_kv4_rows &r) {
  return (long long)(r.most > 0 && r.most < r.rows ? r.most : r.rows) * (r.q_heads / d.kv_heads);
}

}  // namespace xnor
