// New tokens' keys and values into the cache in 4 bits, with norm and rotation on the way; and out of it.
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

// As the kernel of norms and rotations (heads.cu): a warp has a token, and its units of queries, then of keys, then of values.
template <class T, int kDim, bool kPairs>
__global__ void __launch_bounds__(32 * kWarps, 2)
kv4_append_kernel(const Kv4AppendArgs A, int parts, int pieces) {
  using Lane = HeadLane<kDim>;
  const xnor_heads_desc &d = A.h.d;
  const int id = threadIdx.x & 31;
  const Lane lane(id, d.rot, kPairs);
  const bool f32 = d.weight_type == XNOR_F32;
  const int q_units = (d.q_heads + Lane::kHeads - 1) / Lane::kHeads, k_units = (d.k_heads + Lane::kHeads - 1) / Lane::kHeads;
  const int per_page = A.w.d.page / kKvTokens;
  const long long items = (long long)d.rows * parts;
  stream_order();
  for (long long item = (long long)blockIdx.x * kWarps + threadIdx.x / 32; item < items; item += (long long)gridDim.x * kWarps) {
    const int t = (int)(item / parts);
    const T *q = static_cast<const T *>(A.h.q) + t * d.q_stride, *k = static_cast<const T *>(A.h.k) + t * d.k_stride;
    const T *v_row = static_cast<const T *>(A.v) + t * d.v_stride;
    auto kind_of = [&](int u) { return u < q_units ? 0 : u < q_units + k_units ? 1 : 2; };
    auto head_of = [&](int u) { return (u < q_units ? u : u < q_units + k_units ? u - q_units : u - q_units - k_units) * Lane::kHeads + lane.sub; };
    auto fetch = [&](int u, Chunk<T> &ca, Chunk<T> &cb) {
      const int kind = kind_of(u), head = head_of(u);
      const bool in = u < q_units + 2 * k_units && head < (kind == 0 ? d.q_heads : d.k_heads);
      const T *from = (kind == 0 ? q : kind == 1 ? k : v_row) + (in ? head : 0) * kDim;
      ca.load(from + lane.a, pieces, in ? 8 : 0);
      cb.load(from + lane.b, pieces, in ? 8 : 0);
    };
    // (the first values are under way while the token's place is looked up, then the next ones while these are worked on)
    const int first = (int)(item % parts);
    Chunk<T> xa, xb, ya, yb;
    fetch(first, xa, xb);
    int b, place;
    if (!find_sequence(A.w, t, id, b, place) || place < 0) continue;
    const bool angles_there = d.rot == 0 || place < d.positions;
    Angles angles;
    if (lane.turns && angles_there) angles.load(A.h.table + (size_t)place * d.rot, d.rot, lane.which);
    const long long record = kv4_find(A.w, b, place / kKvTokens, 0);
    if ((record < 0 || !angles_there) && id == 0) atomicMax(&g_status_kv4, (int)XNOR_ERR_BOUNDS);
    if (!angles_there) continue;
    T *q_out = static_cast<T *>(A.h.q_out) + t * d.q_out_stride;
    auto finish = [&](int u, Chunk<T> &ca, Chunk<T> &cb) {
      const int kind = kind_of(u), head = head_of(u);
      if (kind > 0 && record < 0) return;
      const bool in = head < (kind == 0 ? d.q_heads : d.k_heads);
      float v[16];
      ca.to_float(*reinterpret_cast<float (*)[8]>(v));
      cb.to_float(*reinterpret_cast<float (*)[8]>(v + 8));
      float w[16];
      if (kind < 2 && d.norm) {
        const void *weight = kind == 0 ? A.h.q_weight : A.h.k_weight;
        load_head_weights<T>(weight, f32, lane.a, w);
        load_head_weights<T>(weight, f32, lane.b, w + 8);
      }
      if (kind == 0) {
        if (d.norm) {
          float s = 0.0f;
#pragma unroll
          for (int i = 0; i < 16; ++i) s = fmaf(v[i], v[i], s);
          const float r = __frsqrt_rn(lane.sum(s) * (1.0f / kDim) + d.eps);
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i] *= r * w[i];
        }
        if (lane.turns) turn<kPairs, 1>(v, angles);
        ca.from_float(*reinterpret_cast<const float (*)[8]>(v));
        cb.from_float(*reinterpret_cast<const float (*)[8]>(v + 8));
        if (in) {
          ca.store(q_out + head * kDim + lane.a, pieces, 8);
          cb.store(q_out + head * kDim + lane.b, pieces, 8);
        }
        return;
      }
      if (kind == 1 && (d.norm || d.rot > 0)) {
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
      uint8_t *to = A.cache + (size_t)(record + (long long)(in ? head : 0) * per_page) * kv4_record(kDim);
      store_codes<kDim>(v, lane, to, place % kKvTokens, kind == 2, in);
    };
#pragma unroll 1
    for (int u = first; u < q_units + 2 * k_units; u += 2 * parts) {
      fetch(u + parts, ya, yb);
      finish(u, xa, xb);
      if (u + parts >= q_units + 2 * k_units) break;
      fetch(u + 2 * parts, xa, xb);
      finish(u + parts, ya, yb);
    }
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
  const long long items = (long long)A.rows * parts;
  stream_order();
  for (long long item = (long long)blockIdx.x * kWarps + threadIdx.x / 32; item < items; item += (long long)gridDim.x * kWarps) {
    const int t = (int)(item / parts);
    int b, place;
    if (!find_sequence(A.w, t, id, b, place) || place < 0) continue;
    const long long record = kv4_find(A.w, b, place / kKvTokens, 0);
    if (record < 0) {
      if (id == 0) atomicMax(&g_status_kv4, (int)XNOR_ERR_BOUNDS);
      continue;
    }
    const int slot = place % kKvTokens;
    for (int u = (int)(item % parts); u < 2 * k_units; u += parts) {
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
  const int pieces = rows_in_pieces(a.h.q, d.q_stride, kDim, sizeof(T)) && rows_in_pieces(a.h.k, d.k_stride, kDim, sizeof(T)) &&
                     rows_in_pieces(a.v, d.v_stride, kDim, sizeof(T)) && rows_in_pieces(a.h.q_out, d.q_out_stride, kDim, sizeof(T));
  const int parts = parts_for((d.q_heads + kHeads - 1) / kHeads + 2 * ((d.k_heads + kHeads - 1) / kHeads), d.rows);
  const dim3 grid(blocks_for((long long)d.rows * parts));
  return d.pairs ? launch_kernel(kv4_append_kernel<T, kDim, true>, grid, 32 * kWarps, 0, st, 1, a, parts, pieces)
                 : launch_kernel(kv4_append_kernel<T, kDim, false>, grid, 32 * kWarps, 0, st, 1, a, parts, pieces);
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
