// New tokens into the cache: rotary positions on q and k, k and v to their pages.
#pragma once

#include "kv_common.hpp"

namespace saki {

struct KvStrides {
  char* data;
  int64_t token, head;  // bytes
};

struct KvAppendParams {
  KvTable t;
  KvPool p;  // bases of the layer
  KvTokens n;
  const double* freq;
  int pairs;  // rotary_dim / 2
  float amplitude;
  int n_q_heads;
  KvStrides q, q_out, k, v;
};

constexpr int KV_APPEND_NT = 256;
constexpr int KV_MAX_PAIRS = 128;

__device__ __forceinline__ float kv_to_f32(uint16_t x) { return __uint_as_float(static_cast<uint32_t>(x) << 16); }
__device__ __forceinline__ float kv_to_f32(float x) { return x; }
// to the nearest bf16, ties to even (a NaN stays one)
__device__ __forceinline__ uint16_t kv_to_bf16(float x) {
  return __builtin_bit_cast(uint16_t, static_cast<__bf16>(x));
}
__device__ __forceinline__ void kv_put(uint16_t* p, float x) { *p = kv_to_bf16(x); }
__device__ __forceinline__ void kv_put(float* p, float x) { *p = x; }

// Eight consecutive elements of a head.
template <typename T>
struct Kv8 {
  T x[8];
};
template <typename T>
__device__ __forceinline__ Kv8<T> kv_load8(const T* p) {
  Kv8<T> r;
  const uint4* s = reinterpret_cast<const uint4*>(p);
  uint4 u[sizeof(T) / 2];
#pragma unroll
  for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i) u[i] = s[i];
  __builtin_memcpy(&r, u, sizeof(r));
  return r;
}
template <typename T>
__device__ __forceinline__ void kv_store8(T* p, const Kv8<T>& r) {
  uint4 u[sizeof(T) / 2];
  __builtin_memcpy(u, &r, sizeof(r));
  uint4* d = reinterpret_cast<uint4*>(p);
#pragma unroll
  for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i) d[i] = u[i];
}

// The sequence whose rows hold `row`: the largest b with offsets[b] <= row, found
// by the whole workgroup in steps of 256 candidates.
__device__ __forceinline__ int kv_find_sequence(const KvTokens& T, int n_seq, int row) {
  int lo = 0, n = n_seq;  // among lo .. lo + n - 1
  while (n > 1) {
    const int step = (n + KV_APPEND_NT - 1) / KV_APPEND_NT;
    const int at = static_cast<int>(threadIdx.x) * step;
    const int below = __syncthreads_count(at < n && T.offsets[lo + at] <= row);
    if (below == 0) return lo;
    lo += (below - 1) * step;
    n = n - (below - 1) * step < step ? n - (below - 1) * step : step;
  }
  return lo;
}

// One workgroup per token.  The angles of the token's pairs are formed once, in
// 64 bits (at position 2^20 an angle in 32 bits would be off by up to 0.06),
// reduced to a fraction of a turn, and their cosines and sines shared by all heads.
// A thread takes 8 consecutive elements of a head, or the two runs of 8 whose
// elements pair up, so that a row may be rotated in place.  VEC: runs of 8 pair
// up whole (half layout: rotary_dim / 2 a multiple of 8; interleaved: rotary_dim a
// multiple of 8); else a thread takes single pairs.
template <typename T, bool INTERLEAVED, bool VEC>
__global__ __launch_bounds__(KV_APPEND_NT) void kv_append_kernel(KvAppendParams P) {
  __shared__ float cs[KV_MAX_PAIRS], sn[KV_MAX_PAIRS];
  const int row = blockIdx.x, tid = threadIdx.x;
  const int b = P.n.offsets ? kv_find_sequence(P.n, P.t.n_seq, row) : row / P.n.n_new;
  int first, count;
  kv_rows(P.n, b, &first, &count);
  if (row < first || row >= first + count) return;  // the whole workgroup
  const int64_t pos = static_cast<int64_t>(P.t.length[b]) + P.n.shift + (row - first);
  const int64_t slot_page = pos >> P.t.shift;
  int page = -1;
  if (pos >= 0 && slot_page < kv_held(P.t, b)) page = P.t.pages[static_cast<int64_t>(b) * P.t.max_pages + slot_page];
  // (a page that other sequences hold too is not written: they would see the token)
  const bool fine = page >= 0 && page < P.t.n_pages && P.t.refs[page] <= 1;
  const int R2 = P.pairs, D = P.p.dim;
  for (int i = tid; i < R2; i += KV_APPEND_NT) {
    const double turns = static_cast<double>(pos) * P.freq[i];
    float s, c;
    sincospif(2.0f * static_cast<float>(turns - rint(turns)), &s, &c);
    cs[i] = P.amplitude * c;
    sn[i] = P.amplitude * s;
  }
  __syncthreads();
  const int64_t in_page = (pos & ((1 << P.t.shift) - 1)) * P.p.token_stride;
  const int64_t cell = fine ? page * P.p.page_stride + in_page : 0;
  const int Hq = P.n_q_heads, Hk = P.p.n_heads;
  const float nan = __builtin_nanf("");
  // runs (or pairs) of a head that turn, and runs of 8 that are copied
  const int turning = VEC ? (INTERLEAVED ? R2 / 4 : R2 / 8) : R2;
  const int plain = VEC ? D / 8 - R2 / 4 : D - 2 * R2;
  const int per_head = turning + plain;
  const int rotated = (Hq + Hk) * per_head;
  const int total = rotated + (fine ? Hk * (D / 8) : 0);
  for (int u = tid; u < total; u += KV_APPEND_NT) {
    if (u >= rotated) {
      const int w = u - rotated, h = w / (D / 8), c = w - h * (D / 8);
      const T* src = reinterpret_cast<const T*>(P.v.data + row * P.v.token + h * P.v.head) + 8 * c;
      kv_store8(reinterpret_cast<T*>(P.p.v + cell + h * P.p.head_stride) + 8 * c, kv_load8(src));
      continue;
    }
    const int hh = u / per_head, e = u - hh * per_head;
    const bool is_q = hh < Hq;
    const int h = is_q ? hh : hh - Hq;
    if (!is_q && !fine) continue;
    const KvStrides& in = is_q ? P.q : P.k;
    const T* src = reinterpret_cast<const T*>(in.data + row * in.token + h * in.head);
    T* dst = is_q ? reinterpret_cast<T*>(P.q_out.data + row * P.q_out.token + h * P.q_out.head)
                  : reinterpret_cast<T*>(P.p.k + cell + h * P.p.head_stride);
    if constexpr (VEC) {
      if (e >= turning) {
        const int at = 2 * R2 + 8 * (e - turning);
        Kv8<T> x = kv_load8(src + at);
        if (!fine)
#pragma unroll
          for (int i = 0; i < 8; ++i) kv_put(&x.x[i], nan);
        kv_store8(dst + at, x);
      } else if constexpr (INTERLEAVED) {
        Kv8<T> x = kv_load8(src + 8 * e);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float a = kv_to_f32(x.x[2 * i]), z = kv_to_f32(x.x[2 * i + 1]), c = cs[4 * e + i], s = sn[4 * e + i];
          kv_put(&x.x[2 * i], fine ? a * c - z * s : nan);
          kv_put(&x.x[2 * i + 1], fine ? z * c + a * s : nan);
        }
        kv_store8(dst + 8 * e, x);
      } else {
        Kv8<T> x = kv_load8(src + 8 * e), y = kv_load8(src + R2 + 8 * e);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float a = kv_to_f32(x.x[i]), z = kv_to_f32(y.x[i]), c = cs[8 * e + i], s = sn[8 * e + i];
          kv_put(&x.x[i], fine ? a * c - z * s : nan);
          kv_put(&y.x[i], fine ? z * c + a * s : nan);
        }
        kv_store8(dst + 8 * e, x);
        kv_store8(dst + R2 + 8 * e, y);
      }
    } else {
      if (e >= turning) {
        const int at = 2 * R2 + (e - turning);
        const T x = src[at];
        if (fine)
          dst[at] = x;
        else
          kv_put(&dst[at], nan);
      } else {
        const int i0 = INTERLEAVED ? 2 * e : e, i1 = INTERLEAVED ? 2 * e + 1 : e + R2;
        const float a = kv_to_f32(src[i0]), z = kv_to_f32(src[i1]), c = cs[e], s = sn[e];
        kv_put(&dst[i0], fine ? a * c - z * s : nan);
        kv_put(&dst[i1], fine ? z * c + a * s : nan);
      }
    }
  }
}

}  // namespace saki
