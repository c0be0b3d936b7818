// New tokens' keys and values into the cache in 4 bits, with norm and rotation on the way; and out of it.
//
// Read once, written once; a token's place is two dependent loads away (its sequence, its page), its angles three, and its keys are
// worked out in 64 bits.  16 prompts of up to 1000 tokens, 32 and 8 heads of 64 in F16: 29 us in and 10 us out again (floor of both 18.5), 122
// registers and 22 % of the warps a SM can have, 1.9 instructions per clock.  (With loads that had conditions, and so were waited for
// one by one, 49 in; three blocks per SM spilled, 73 for both.)  64 tokens, one of a sequence each: 7.3 us, latency.
#include <algorithm>

#include "kv4.cuh"

namespace xnor {

__device__ int g_status_kv4 = 0;

namespace {

constexpr int kWarps = 8;

// Sixteen values of a thread, chunks at lane.a and lane.b of a head, into its record.  The head's threads share its scale.
template <int kDim>
__device__ __forceinline__ void store_codes(const float (&v)[16], const HeadLane<kDim> &lane, uint8_t *record, int slot, bool values, bool in) {
  float lo = 0.0f, hi = 0.0f, odd = 0.0f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    lo = fminf(lo, v[i]);
    hi = fmaxf(hi, v[i]);
    odd = fmaf(v[i], 0.0f, odd);                     // NaN if any is NaN or infinite
  }
#pragma unroll
  for (int o = HeadLane<kDim>::kLanes / 2; o > 0; o >>= 1) {
    lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    odd += __shfl_xor_sync(0xffffffffu, odd, o);
  }
  // a fifteenth in 64 bits, the quotient mended by its rest (Markstein): a division by a variable takes 100 instructions
  const double range = (double)hi - (double)lo, fifteenth = range * (1.0 / 15.0);
  const uint32_t bits = __float_as_uint((float)fma(fma(-15.0, fifteenth, range), 1.0 / 15.0, fifteenth)) & ~15u;
  const float s = __uint_as_float(bits);
  const bool sound = odd == 0.0f && s > 0.0f;
  const float inv = sound && s > 1e-37f ? 1.0f / s : 0.0f;        // 0: it would overflow
  float z = 8.0f, q[16];
  if (sound) {
    z = fminf(15.0f, fmaxf(0.0f, inv == 0.0f ? round_quotient(-lo, s) : mend_quotient(rintf(-lo * inv), -lo, s)));
    round_quotients(v, s, inv, z, q);
#pragma unroll
    for (int i = 0; i < 16; ++i) q[i] = fminf(15.0f, fmaxf(0.0f, q[i] + z));
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) q[i] = 8.0f;
  }
  if (!in) return;
  uint8_t *codes = record + kv4_codes(kDim, values) + slot * (kDim / 2);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const float *c = q + 8 * h;
    const uint32_t even = __float_as_uint(four_codes(8388608.0f + c[0], c[2], c[4], c[6])), other = __float_as_uint(four_codes(8388608.0f + c[1], c[3], c[5], c[7]));
    *reinterpret_cast<uint32_t *>(codes + (h == 0 ? lane.a : lane.b) / 2) = __byte_perm(even, other, 0x5410);
  }
  if (lane.which == 0)
    *reinterpret_cast<uint32_t *>(record + kv4_words(kDim, values) + 4 * slot) = (odd == 0.0f ? bits : 0x7FFFFFF0u) | (uint32_t)z;
}

// As the kernel of norms and rotations (heads.cu): a warp has a token, and its units of queries, then of keys, then of values,
// every parts-th of the three together.  The first of each kind are under way while the token's place is looked up.
template <class T, int kDim, bool kPairs, bool kPieces>
__global__ void __launch_bounds__(32 * kWarps, 2)
kv4_append_kernel(const Kv4AppendArgs A, int parts) {
  using Lane = HeadLane<kDim>;
  const xnor_heads_desc &d = A.h.d;
  const int id = threadIdx.x & 31;
  const Lane lane(id, d.rot, kPairs);
  const bool f32 = d.weight_type == XNOR_F32;
  const int q_units = (d.q_heads + Lane::kHeads - 1) / Lane::kHeads, k_units = (d.k_heads + Lane::kHeads - 1) / Lane::kHeads;
  const int per_page = A.w.d.page / kKvTokens, step = parts * Lane::kHeads;
  const int items = d.rows * parts;                          // (rows, or a few thousand)
  stream_order();
  for (int item = (int)blockIdx.x * kWarps + (int)threadIdx.x / 32; item < items; item += (int)gridDim.x * kWarps) {
    const int t = item / parts, first = item - t * parts;
    const int first_k = first >= q_units ? first - q_units : (parts - (q_units - first) % parts) % parts;
    const int first_v = first >= q_units + k_units ? first - q_units - k_units : (parts - (q_units + k_units - first) % parts) % parts;
    const T *k = static_cast<const T *>(A.h.k) + t * d.k_stride, *v_row = static_cast<const T *>(A.v) + t * d.v_stride;
    const T *q = d.q_heads > 0 ? static_cast<const T *>(A.h.q) + t * d.q_stride : k;      // (read, but not used)
    auto fetch = [&](const T *from, int heads, int h, TwoChunks<T> &x) { x.template load<kPieces>(from + (h < heads ? h : 0) * kDim, lane); };
    TwoChunks<T> x_q, x_k, x_v;
    fetch(q, d.q_heads, first * Lane::kHeads + lane.sub, x_q);
    fetch(k, d.k_heads, first_k * Lane::kHeads + lane.sub, x_k);
    fetch(v_row, d.k_heads, first_v * Lane::kHeads + lane.sub, x_v);
    int b, place;
    if (!find_sequence(A.w, t, id, b, place) || place < 0) continue;
    const bool angles_there = d.rot == 0 || place < d.positions;
    Angles angles;
    if (lane.turns && angles_there) angles.load(A.h.table + (size_t)place * d.rot, d.rot, lane.which);
    const long long record = kv4_find(A.w, b, place / kKvTokens, 0);
    if ((record < 0 || !angles_there) && id == 0) atomicMax(&g_status_kv4, (int)XNOR_ERR_BOUNDS);
    if (!angles_there) continue;
    // units first, first + parts, .. of one kind, the next one's values under way
    auto run = [&](const T *from, int units, int heads, int first, TwoChunks<T> &x, auto finish) {
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
    float w[16];
    auto weights = [&](const void *weight) {
      if (!d.norm) return;
      load_head_weights<T>(weight, f32, lane.a, w);
      load_head_weights<T>(weight, f32, lane.b, w + 8);
    };
    if (first < q_units) {
      T *q_out = static_cast<T *>(A.h.q_out) + t * d.q_out_stride;
      weights(A.h.q_weight);
      run(q, q_units, d.q_heads, first, x_q, [&](int h, TwoChunks<T> &x) {
        float v[16];
        x.to_float(v);
        if (d.norm) {
          float s = 0.0f;
#pragma unroll
          for (int i = 0; i < 16; ++i) s = fmaf(v[i], v[i], s);
          const float r = __frsqrt_rn(lane.sum(s) * (1.0f / kDim) + d.eps);
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i] *= r * w[i];
        }
        if (lane.turns) turn<kPairs, 1>(v, angles);
        x.from_float(v);
        if (h < d.q_heads) x.template store<kPieces>(q_out + h * kDim, lane);
      });
    }
    if (record < 0) continue;
    auto record_of = [&](int h) { return A.cache + (size_t)(record + (long long)(h < d.k_heads ? h : 0) * per_page) * kv4_record(kDim); };
    if (first_k < k_units) {
      weights(A.h.k_weight);
      run(k, k_units, d.k_heads, first_k, x_k, [&](int h, TwoChunks<T> &c) {
        float v[16];
        c.to_float(v);
        if (d.norm || d.rot > 0) {
          // Keys in 64 bits: a code is that of the exact key, wherever it lies next to a border.
          double x[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) x[i] = (double)v[i];
          if (d.norm) {
            double s = 0.0;
#pragma unroll
            for (int i = 0; i < 16; ++i) s = fma(x[i], x[i], s);
            const double r = 1.0 / sqrt(lane.sum(s) * (1.0 / kDim) + (double)d.eps);
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = x[i] * r * (double)w[i];
          }
          if (lane.turns) turn<kPairs, 1>(x, angles);
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i] = (float)x[i];
        }
        store_codes<kDim>(v, lane, record_of(h), place % kKvTokens, false, h < d.k_heads);
      });
    }
    run(v_row, k_units, d.k_heads, first_v, x_v, [&](int h, TwoChunks<T> &c) {
      float v[16];
      c.to_float(v);
      store_codes<kDim>(v, lane, record_of(h), place % kKvTokens, true, h < d.k_heads);
    });
  }
}

// A warp has a token, and its units of keys, then of values.
template <class T, int kDim>
__global__ void __launch_bounds__(32 * kWarps)
kv4_read_kernel(const Kv4ReadArgs A, uint32_t magic, int parts, int pieces) {
  using Lane = HeadLane<kDim>;
  const int id = threadIdx.x & 31, heads = A.w.d.kv_heads, k_units = (heads + Lane::kHeads - 1) / Lane::kHeads;
  const Lane lane(id, 0, 0);
  const int per_page = A.w.d.page / kKvTokens;
  const int items = A.rows * parts;
  stream_order();
  for (int item = (int)blockIdx.x * kWarps + (int)threadIdx.x / 32; item < items; item += (int)gridDim.x * kWarps) {
    const int t = item / parts;
    int b, place;
    if (!find_sequence(A.w, t, id, b, place) || place < 0) continue;
    const long long record = kv4_find(A.w, b, place / kKvTokens, 0);
    if (record < 0) {
      if (id == 0) atomicMax(&g_status_kv4, (int)XNOR_ERR_BOUNDS);
      continue;
    }
    const int slot = place % kKvTokens;
    for (int u = item - t * parts; u < 2 * k_units; u += parts) {
      const bool values = u >= k_units;
      const int head = (values ? u - k_units : u) * Lane::kHeads + lane.sub;
      if (head >= heads) continue;
      const uint8_t *from = A.cache + (size_t)(record + (long long)head * per_page) * kv4_record(kDim);
      const uint32_t word = load_global(reinterpret_cast<const uint32_t *>(from + kv4_words(kDim, values)) + slot);
      const float s = kv4_scale(word);
      const W4Type<__nv_bfloat16>::Zero z = W4Type<__nv_bfloat16>::zero(word & 15u);
      T *to = static_cast<T *>(values ? A.v : A.k) + t * (values ? A.v_stride : A.k_stride) + head * kDim;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int column = h == 0 ? lane.a : lane.b;
        uint32_t pair[4];
        W4Type<__nv_bfloat16>::expand(load_global(reinterpret_cast<const uint32_t *>(from + kv4_codes(kDim, values) + slot * (kDim / 2) + column / 2)), z, magic, pair);
        float v[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 f = pair_to_float(pair[i], __nv_bfloat16());
          v[2 * i] = f.x * s;
          v[2 * i + 1] = f.y * s;
        }
        Chunk<T> c;
        c.from_float(v);
        c.store(to + column, pieces, 8);
      }
    }
  }
}

unsigned blocks_for(long long items) { return (unsigned)std::min<long long>((items + kWarps - 1) / kWarps, 1 << 20); }
int parts_for(int units, int rows) { return (int)std::min<long long>(units, std::max<long long>(1, 32ll * kSms / rows)); }

template <class T, int kDim>
cudaError_t append(const Kv4AppendArgs &a, cudaStream_t st) {
  constexpr int kHeads = HeadLane<kDim>::kHeads;
  const xnor_heads_desc &d = a.h.d;
  const bool pieces = rows_in_pieces(a.h.q, d.q_stride, kDim, sizeof(T)) && rows_in_pieces(a.h.k, d.k_stride, kDim, sizeof(T)) &&
                     rows_in_pieces(a.v, d.v_stride, kDim, sizeof(T)) && rows_in_pieces(a.h.q_out, d.q_out_stride, kDim, sizeof(T));
  const int parts = parts_for((d.q_heads + kHeads - 1) / kHeads + 2 * ((d.k_heads + kHeads - 1) / kHeads), d.rows);
  const dim3 grid(blocks_for((long long)d.rows * parts));
  auto *kernel = d.pairs ? (pieces ? kv4_append_kernel<T, kDim, true, true> : kv4_append_kernel<T, kDim, true, false>)
                         : (pieces ? kv4_append_kernel<T, kDim, false, true> : kv4_append_kernel<T, kDim, false, false>);
  return launch_kernel(kernel, grid, 32 * kWarps, 0, st, 1, a, parts);
}
template <class T>
cudaError_t append_type(const Kv4AppendArgs &a, cudaStream_t st) { return a.h.d.dim == 64 ? append<T, 64>(a, st) : append<T, 128>(a, st); }

template <class T, int kDim>
cudaError_t read(const Kv4ReadArgs &a, cudaStream_t st) {
  const int pieces = rows_in_pieces(a.k, a.k_stride, kDim, sizeof(T)) && rows_in_pieces(a.v, a.v_stride, kDim, sizeof(T));
  constexpr int kHeads = HeadLane<kDim>::kHeads;
  const int parts = parts_for(2 * ((a.w.d.kv_heads + kHeads - 1) / kHeads), a.rows);
  return launch_kernel(kv4_read_kernel<T, kDim>, dim3(blocks_for((long long)a.rows * parts)), 32 * kWarps, 0, st, 1, a, W4Type<__nv_bfloat16>::kMagic, parts, pieces);
}
template <class T>
cudaError_t read_type(const Kv4ReadArgs &a, cudaStream_t st) { return a.w.d.dim == 64 ? read<T, 64>(a, st) : read<T, 128>(a, st); }

}  // namespace

cudaError_t read_status_kv4(int *status) {
  cudaError_t e = cudaMemcpyFromSymbol(status, g_status_kv4, sizeof(int));
  if (e == cudaSuccess && *status != 0) {
    const int zero = 0;
    e = cudaMemcpyToSymbol(g_status_kv4, &zero, sizeof(int));
  }
  return e;
}

cudaError_t launch_kv4_append(const Kv4AppendArgs &a, cudaStream_t st) {
  if (a.h.d.rows == 0) return cudaSuccess;
  if (a.h.d.type == XNOR_F32) return append_type<float>(a, st);
  return a.h.d.type == XNOR_BF16 ? append_type<__nv_bfloat16>(a, st) : append_type<__half>(a, st);
}

cudaError_t launch_kv4_read(const Kv4ReadArgs &a, cudaStream_t st) {
  if (a.rows == 0) return cudaSuccess;
  if (a.type == XNOR_F32) return read_type<float>(a, st);
  return a.type == XNOR_BF16 ? read_type<__nv_bfloat16>(a, st) : read_type<__half>(a, st);
}

}  // namespace xnor
