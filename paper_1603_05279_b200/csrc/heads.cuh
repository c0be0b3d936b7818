// Rows of heads [rows][heads][dim]: their root-mean-square norm and the rotation by position (internal).
//
// A head's pairs: with the halves paired, value i of the first `rot` with value i + rot / 2, or neighbours, 2 i with
// 2 i + 1; pair i turns by the angle whose cosine and sine are entries i and rot / 2 + i of the position's row of the table.
// Values from `rot` on stay.
//
// A thread has eight pairs, as two chunks of eight values that lie together in memory, and 2^k threads a head; so the
// partner of a value is in the same thread, and only the sum of squares crosses threads.  A thread whose pairs are
// behind the rotated ones has values of the rest.
#pragma once
#include "rows.cuh"

namespace xnor {

constexpr int kHeadsMaxDim = 512;

struct HeadsArgs {
  const void *q, *k, *q_weight, *k_weight;
  const int *pos;
  const float *table;
  void *q_out, *k_out;
  const void *dq_out, *dk_out;          // backward pass: q_out and k_out are the gradients at q and k
  float *dq_weight, *dk_weight, *work;
  xnor_heads_desc d;
};
cudaError_t launch_heads(const HeadsArgs &a, cudaStream_t st);
cudaError_t launch_heads_backward(const HeadsArgs &a, cudaStream_t st);
int heads_parts(int rows, int q_heads, int k_heads);      // rows of partial sums in the workspace
cudaError_t read_status_heads(int *status);

// Heads whose threads have whole chunks: 64, 128 or 256 values, rotated and other values in whole chunks, rows anywhere
// that 16-byte pieces can be read.
inline bool heads_in_chunks(const xnor_heads_desc &d) { return (d.dim == 64 || d.dim == 128 || d.dim == 256) && d.rot % 16 == 0; }

// a / b of numbers that are not negative, for the most part below 2^32 (in 64 bits it takes 100 instructions).
__device__ __forceinline__ long long divide(long long a, long long b) {
  return ((a | b) >> 32) == 0 ? (long long)((uint32_t)a / (uint32_t)b) : a / b;
}

template <int kDim>
struct HeadLane {
  static constexpr int kLanes = kDim / 16, kHeads = 32 / kLanes;      // threads of a head, heads of a warp
  int sub, which;                       // this thread's head of the warp's, its place in it
  int a, b;                             // the chunks' first columns
  bool turns;
  __device__ __forceinline__ HeadLane(int lane, int rot, int pairs) {
    sub = lane / kLanes;
    which = lane % kLanes;
    const int p = 8 * which, rest = p - rot / 2;
    turns = rest < 0;
    if (pairs) { a = 2 * p; b = a + 8; }
    else if (turns) { a = p; b = rot / 2 + p; }
    else { a = rot + rest; b = a + (kDim - rot) / 2; }
  }
  // Sum over the threads of a head.
  template <class V>
  __device__ __forceinline__ V sum(V v) const {
#pragma unroll
    for (int o = kLanes / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
  }
};

// A thread's values of a head.  Loads have no condition, so that nothing waits for them before their values are used: what
// does not exist is read elsewhere.
template <class T>
struct TwoChunks {
  Chunk<T> a, b;
  template <bool kPieces = true, class Lane>
  __device__ __forceinline__ void load(const T *head, const Lane &lane) {
    a.load(head + lane.a, kPieces, 8);
    b.load(head + lane.b, kPieces, 8);
  }
  template <bool kPieces = true, class Lane>
  __device__ __forceinline__ void store(T *head, const Lane &lane) const {
    a.store(head + lane.a, kPieces, 8);
    b.store(head + lane.b, kPieces, 8);
  }
  __device__ __forceinline__ void to_float(float (&v)[16]) const {
    a.to_float(*reinterpret_cast<float (*)[8]>(v));
    b.to_float(*reinterpret_cast<float (*)[8]>(v + 8));
  }
  __device__ __forceinline__ void from_float(const float (&v)[16]) {
    a.from_float(*reinterpret_cast<const float (*)[8]>(v));
    b.from_float(*reinterpret_cast<const float (*)[8]>(v + 8));
  }
};

// Cosines and sines of a thread's eight pairs.
struct Angles {
  float c[8], s[8];
  __device__ __forceinline__ void load(const float *row, int rot, int which) {
    const float4 *p = reinterpret_cast<const float4 *>(row + 8 * which), *q = reinterpret_cast<const float4 *>(row + rot / 2 + 8 * which);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float4 u = load_global(p + i), v = load_global(q + i);
      c[4 * i] = u.x; c[4 * i + 1] = u.y; c[4 * i + 2] = u.z; c[4 * i + 3] = u.w;
      s[4 * i] = v.x; s[4 * i + 1] = v.y; s[4 * i + 2] = v.z; s[4 * i + 3] = v.w;
    }
  }
};

// x: chunk a, then chunk b.  kSign = -1: backwards.
template <bool kPairs, int kSign, class V>
__device__ __forceinline__ void turn(V (&x)[16], const Angles &t) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    V &u = kPairs ? x[2 * i] : x[i], &v = kPairs ? x[2 * i + 1] : x[8 + i];
    const V c = (V)t.c[i], s = kSign > 0 ? (V)t.s[i] : -(V)t.s[i], w = u * c - v * s;
    v = v * c + u * s;
    u = w;
  }
}

// Weights of a chunk: of the rows' type, in 32 bits or (null) ones.
template <class T>
__device__ __forceinline__ void load_head_weights(const void *w, bool f32, int column, float *v) {
  if (w == nullptr) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 1.0f;
  } else if (f32) {
    Chunk<float> c;
    c.load(static_cast<const float *>(w) + column, true, 8);
    c.to_float(*reinterpret_cast<float (*)[8]>(v));
  } else {
    Chunk<T> c;
    c.load(static_cast<const T *>(w) + column, true, 8);
    c.to_float(*reinterpret_cast<float (*)[8]>(v));
  }
}

}  // namespace xnor
