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

// The sequence whose rows hold `row`, or -1, and its first row, found by the whole workgroup: the largest b with
// offsets[b] <= row, in steps of 256 candidates.  That is the one if the offsets are in order; where its range
// does not hold the row (a row of no sequence, or a range somewhere that is out of order and counts as
// empty), every range is looked at.
__device__ __forceinline__ int kv_find_sequence(const KvTokens& T, int n_seq, int row, int* first) {
  int lo = 0, n = n_seq;  // among lo .. lo + n - 1
  while (n > 1) {
    const int step = (n + KV_APPEND_NT - 1) / KV_APPEND_NT;
    const int at = static_cast<int>(threadIdx.x) * step;
    const int below = __syncthreads_count(at < n && T.offsets[lo + at] <= row);
    if (below == 0) break;
    lo += (below - 1) * step;
    n = n - (below - 1) * step < step ? n - (below - 1) * step : step;
  }
  auto holds = [&](int b, int* first) {
    int count;
    kv_rows(T, b, first, &count);
    return row >= *first && row - *first < count;
  };
  if (holds(lo, first)) return lo;
  __shared__ int found;
  if (threadIdx.x == 0) found = -1;
  __syncthreads();
  for (int b = threadIdx.x; b < n_seq; b += KV_APPEND_NT)
    if (holds(b, first)) atomicMax(&found, b);  // (one b, unless ranges overlap, which they may not)
  __syncthreads();
  const int b = found;
  if (b >= 0) *first = T.offsets[b];
  return b;
}

// One workgroup per token.  The angles of the token's pairs are formed once, in
// 64 bits (at position 2^20 an angle in 32 bits would be off by up to 0.06),
// reduced to a fraction of a turn, and their cosines and sines shared by all heads.
// A thread takes 8 consecutive elements of a head, or the two runs of 8 whose
// elements pair up, so that a row may be rotated in place.  VEC: runs of 8 pair
// up whole (half layout: rotary_dim / 2 a multiple of 8; interleaved: rotary_dim a
// multiple of 8); else a thread takes single pairs.
// The cosine, the sine and the rotation itself are in 32 bits, for 32-bit rows too: an element is then off by 2^-20 of
// its pair's size at most (rms 5.6e-8, of which the row's own rounding is 2.5e-8).  64 bits take 7% to 13% more where that
// is not hidden behind memory (a verification of 8 sequences 11.4 us -> 12.3, 33,000 tokens in single pairs 563 -> 637).
// What bounds it: memory, and for few tokens the chain of lookups (the row's sequence, its length,
// page and the page's count); a thread's first KV_AHEAD loads are under way meanwhile (32 ragged
// prompts, 33,000 tokens of 32 + 8 heads of 128 bf16 elements: 203 us without, 188 with:
// 4.3 TB/s of the 4.8 that a large copy reaches; in f32 346 us, 4.7).  Single pairs: accesses of one element
// (heads of 96 elements, 24 of them rotated: bf16 446 us, 1.4 TB/s, f32 563, 2.2; of 80, 20 rotated, bf16 376, 1.4).
constexpr int KV_AHEAD = 3;

template <typename T, bool INTERLEAVED, bool VEC>
__global__ __launch_bounds__(KV_APPEND_NT) void kv_append_kernel(KvAppendParams P) {
  __shared__ float cs[KV_MAX_PAIRS], sn[KV_MAX_PAIRS];
  const int row = blockIdx.x, tid = threadIdx.x;
  const int R2 = P.pairs, D = P.p.dim, Hq = P.n_q_heads, Hk = P.p.n_heads;
  // a token's work: units of q's and k's heads (runs or pairs that turn, then what is copied), then
  // runs of v
  const int turning = VEC ? (INTERLEAVED ? R2 / 4 : R2 / 8) : R2;
  const int per_head = turning + (VEC ? D / 8 - R2 / 4 : D - 2 * R2);
  const int rotated = (Hq + Hk) * per_head, total = rotated + Hk * (D / 8);
  constexpr bool TWO = VEC && !INTERLEAVED;  // a unit that turns is two runs
  struct Unit {
    Kv8<T> x, y;
  };
  auto head_of = [&](int u, int* e) {
    const int h = u / per_head;
    *e = u - h * per_head;
    return h;
  };
  auto load = [&](int u) {
    Unit w;
    if (u >= rotated) {
      const int v = u - rotated, h = v / (D / 8), c = v - h * (D / 8);
      w.x = kv_load8(reinterpret_cast<const T*>(P.v.data + row * P.v.token + h * P.v.head) + 8 * c);
      return w;
    }
    int e;
    const int h = head_of(u, &e);
    const T* src = reinterpret_cast<const T*>(h < Hq ? P.q.data + row * P.q.token + h * P.q.head
                                                     : P.k.data + row * P.k.token + (h - Hq) * P.k.head);
    if constexpr (VEC) {
      const bool turns = e < turning;
      w.x = kv_load8(src + (turns ? 8 * e : 2 * R2 + 8 * (e - turning)));
      if (TWO && turns) w.y = kv_load8(src + R2 + 8 * e);
    } else {
      const bool turns = e < turning;
      w.x.x[0] = src[!turns ? 2 * R2 + (e - turning) : INTERLEAVED ? 2 * e : e];
      if (turns) w.y.x[0] = src[INTERLEAVED ? 2 * e + 1 : e + R2];
    }
    return w;
  };
  Unit ahead[KV_AHEAD];
#pragma unroll
  for (int i = 0; i < KV_AHEAD; ++i)
    if (tid + i * KV_APPEND_NT < total) ahead[i] = load(tid + i * KV_APPEND_NT);

  int b, first;
  if (P.n.offsets) {
    b = kv_find_sequence(P.n, P.t.n_seq, row, &first);
    if (b < 0) return;  // the whole workgroup
  } else {
    b = row / P.n.n_new;
    first = b * P.n.n_new;
  }
  const int64_t pos = static_cast<int64_t>(P.t.length[b]) + P.n.shift + (row - first);
  const int64_t slot_page = pos >> P.t.shift;
  int page = -1;
  if (pos >= 0 && slot_page < kv_held(P.t, b)) page = P.t.pages[static_cast<int64_t>(b) * P.t.max_pages + slot_page];
  // (a page that other sequences hold too is not written: they would see the token)
  const bool fine = page >= 0 && page < P.t.n_pages && P.t.refs[page] <= 1;
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
  const float nan = __builtin_nanf("");
  // where the token has no page of its own, q's row becomes NaN and k and v are not written
  auto turn = [&](T* a, T* b2, int i) {
    const float x = kv_to_f32(*a), z = kv_to_f32(*b2), c = cs[i], s = sn[i];
    kv_put(a, fine ? x * c - z * s : nan);
    kv_put(b2, fine ? z * c + x * s : nan);
  };
  auto store = [&](int u, Unit w) {
    if (u >= rotated) {
      const int v = u - rotated, h = v / (D / 8), c = v - h * (D / 8);
      if (fine) kv_store8(reinterpret_cast<T*>(P.p.v + cell + h * P.p.head_stride) + 8 * c, w.x);
      return;
    }
    int e;
    const int h = head_of(u, &e);
    if (h >= Hq && !fine) return;
    T* dst = reinterpret_cast<T*>(h < Hq ? P.q_out.data + row * P.q_out.token + h * P.q_out.head
                                         : P.p.k + cell + (h - Hq) * P.p.head_stride);
    const bool turns = e < turning;
    if constexpr (VEC) {
      if (!turns) {
        if (!fine)
#pragma unroll
          for (int i = 0; i < 8; ++i) kv_put(&w.x.x[i], nan);
        kv_store8(dst + 2 * R2 + 8 * (e - turning), w.x);
      } else if constexpr (INTERLEAVED) {
#pragma unroll
        for (int i = 0; i < 4; ++i) turn(&w.x.x[2 * i], &w.x.x[2 * i + 1], 4 * e + i);
        kv_store8(dst + 8 * e, w.x);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) turn(&w.x.x[i], &w.y.x[i], 8 * e + i);
        kv_store8(dst + 8 * e, w.x);
        kv_store8(dst + R2 + 8 * e, w.y);
      }
    } else if (turns) {
      turn(&w.x.x[0], &w.y.x[0], e);
      dst[INTERLEAVED ? 2 * e : e] = w.x.x[0];
      dst[INTERLEAVED ? 2 * e + 1 : e + R2] = w.y.x[0];
    } else {
      if (!fine) kv_put(&w.x.x[0], nan);
      dst[2 * R2 + (e - turning)] = w.x.x[0];
    }
  };
#pragma unroll
  for (int i = 0; i < KV_AHEAD; ++i)
    if (tid + i * KV_APPEND_NT < total) store(tid + i * KV_APPEND_NT, ahead[i]);
  for (int u = tid + KV_AHEAD * KV_APPEND_NT; u < total; u += KV_APPEND_NT) store(u, load(u));
}

}  // namespace saki
