// The k largest logits of a row, best first, and the log-sum-exp of the others.
//
// One pass over the row.  Every wave keeps a list of candidates in LDS and a threshold L: the
// k-th largest entry it knows (-infinity before it knows k).  An entry above L joins the
// list; any other is not among the row's k largest and is added at once to the sum
//   R = sum 2^((x - L) c),   c = log2(e) / tau,
// whose terms are at most 1.  When the list is full, its k-th largest entry becomes L, the entries
// below it go to R, and R is brought to the new reference.  So R holds exactly the entries that
// are not listed: nothing is subtracted, and a rest of 1e-30 of the row is as exact as one of half
// of it.  Equal entries: a candidate is the number (order-preserving image of the logit, ~index), so
// all differ; an entry of a later chunk has to be above L, not at it, since a wave sees its chunks by
// ascending index, and inside a chunk, where it does not, the numbers are compared.
// Terms below 2^-126 are lost in 32 bits: where R ends below TOP_RESCAN (everything else lies far
// below the list, as with masked tokens), the row is read again with the reference at the largest
// entry that is not listed.
//
// What bounds it: for whole rows HBM and VALU issue together, see top_kernel.
#pragma once

#include "common.hpp"

namespace saki {

struct TopPart {
  double rest;  // sum over the part of 2^((x - ref) c), without its listed entries
  float ref;
  int bad;  // an entry is not finite
};

struct TopParams {
  const void* x;
  int64_t n_rows;
  int64_t stride;
  int V;
  int k;
  int parts;      // a row's parts (TOP_PART, TOP_MERGE)
  int part_len;   // entries of a part, whole chunks
  float c;        // log2(e) / tau
  float* top_logit;
  int32_t* top_token;
  int64_t top_stride;
  float* rest_logit;
  uint8_t* row_status;
  uint64_t* keys;  // [n_rows, parts, k], 0: no entry
  TopPart* info;   // [n_rows, parts]
};

enum TopMode { TOP_WHOLE, TOP_PART, TOP_MERGE };

constexpr int TOP_NT = 256;
constexpr int TOP_NW = TOP_NT / WAVE;
constexpr int TOP_CAP = 512;  // candidates of a wave: more than SAKI_MAX_TOP_K + WAVE
static_assert(TOP_CAP >= SAKI_MAX_TOP_K + 2 * WAVE, "a list that was shortened takes another 64 entries");

// The order-preserving image of a logit: BITS bits, never 0; -0 and +0 are alike.
template <typename T>
struct TopKey {
  static constexpr int BITS = sizeof(T) * 8;
  static __device__ __forceinline__ uint32_t of(float x) {
    const uint32_t u = x == 0.0f ? 0u : __float_as_uint(x);
    return ((u >> 31) ? ~u : (u | 0x80000000u)) >> (32 - BITS);
  }
  static __device__ __forceinline__ float value(uint32_t key) {
    const uint32_t u = key << (32 - BITS);
    return __uint_as_float((u >> 31) ? (u & 0x7fffffffu) : (BITS == 32 ? ~u : ~u & 0xffff0000u));
  }
};

struct TopShared {
  uint64_t list[TOP_NW][TOP_CAP];
  uint64_t best[SAKI_MAX_TOP_K];  // the block's k largest, then in order
  uint64_t sorted[SAKI_MAX_TOP_K];
  int count[TOP_NW];
  int n_best;
  double red_d[TOP_NW][RED_MAX];
  float red_f[TOP_NW][4];
  int red_i[TOP_NW][4];
};

__device__ __forceinline__ int lanes_below(uint64_t m) {
  return __builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(m >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(m), 0));
}

// The k-th largest of the candidates u[i] (0: none) of a wave's lanes, of which there are at
// least k: bit by bit from the top, the largest number that k of them reach.  Every lane gets it.  The
// index is only searched where more entries tie at the k-th value than are taken.
template <typename T, int N>
__device__ __forceinline__ uint64_t top_threshold(const uint64_t (&u)[N], int k) {
  auto reach = [&](auto at_least) {
    int n = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) n += __popcll(__ballot(at_least(u[i])));
    return n;
  };
  uint32_t hi = 0;
  for (int b = TopKey<T>::BITS - 1; b >= 0; --b) {
    const uint32_t t = hi | (1u << b);
    if (reach([&](uint64_t v) { return static_cast<uint32_t>(v >> 32) >= t; }) >= k) hi = t;
  }
  const uint64_t whole = static_cast<uint64_t>(hi) << 32;
  if (reach([&](uint64_t v) { return v >= whole; }) == k) return whole;
  uint64_t low = whole;
  for (int b = 31; b >= 0; --b) {
    const uint64_t t = low | (1ull << b);
    if (reach([&](uint64_t v) { return v >= t; }) >= k) low = t;
  }
  return low;
}

// A wave's candidates.
template <typename T>
struct WaveTop {
  uint64_t* list;  // LDS
  int lane, k;
  float c;
  int n;        // candidates in the list (the same in all lanes)
  float L;      // the k-th largest entry so far, and the number of its candidate
  uint64_t t;
  double rest;  // this lane's part of R, relative to L

  __device__ __forceinline__ void init(uint64_t* lds, int l, int kk, float cc) {
    list = lds;
    lane = l;
    k = kk;
    c = cc;
    n = 0;
    L = -finf();
    t = 0ull;
    rest = 0.0;
  }

  static __device__ __forceinline__ uint64_t number(float x, int index) {
    return static_cast<uint64_t>(TopKey<T>::of(x)) << 32 | static_cast<uint32_t>(~index);
  }

  // Keeps the k largest candidates; the others go to the rest.
  __device__ __forceinline__ void shorten() {
    constexpr int N = TOP_CAP / WAVE;
    uint64_t u[N];
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < N; ++i) u[i] = i * WAVE + lane < n ? list[i * WAVE + lane] : 0ull;
    t = top_threshold<T, N>(u, k);
    const float to = TopKey<T>::value(static_cast<uint32_t>(t >> 32));
    rest *= static_cast<double>(fexp2((L - to) * c));  // (0 stays 0: L = -infinity has no rest)
    L = to;
    int m = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const bool keep = u[i] >= t;
      const uint64_t who = __ballot(keep);
      if (keep) list[m + lanes_below(who)] = u[i];
      else if (u[i] != 0ull)
        rest += static_cast<double>(fexp2((TopKey<T>::value(static_cast<uint32_t>(u[i] >> 32)) - L) * c));
      m += __popcll(who);
    }
    n = m;
    __builtin_amdgcn_wave_barrier();
  }

  // One entry of each lane that has one (`there`).
  __device__ __forceinline__ void push(bool there, float x, int index) {
    if (n + WAVE > TOP_CAP) shorten();
    const uint64_t u = number(x, index);
    const bool in = there && u > t && x == x;
    const uint64_t who = __ballot(in);
    if (in) list[n + lanes_below(who)] = u;
    n += __popcll(who);
    if (there && !in) rest += static_cast<double>(fexp2((x - L) * c));
  }

  // A lane's 16 entries of a chunk behind all chunks before, those with their bit in vm; base: the
  // chunk's first index.
  __device__ __forceinline__ void push_chunk(const float (&x)[EPL], uint32_t vm, int base) {
    int more = 0;
#pragma unroll
    for (int e = 0; e < EPL; ++e) more += __popcll(__ballot(((vm >> e) & 1u) && x[e] > L));
    if (n + more <= TOP_CAP) {
      float s = 0.0f;
#pragma unroll
      for (int e = 0; e < EPL; ++e) {
        const bool there = (vm >> e) & 1u, in = there && x[e] > L;
        const uint64_t who = __ballot(in);
        if (who != 0ull) {
          if (in) list[n + lanes_below(who)] = number(x[e], base + elem_offset(lane, e));
          n += __popcll(who);
        }
        s += there && !in ? fexp2((x[e] - L) * c) : 0.0f;
      }
      rest += static_cast<double>(s);
    } else {
#pragma unroll 1
      for (int e = 0; e < EPL; ++e) {
        float xe = x[0];
#pragma unroll
        for (int i = 1; i < EPL; ++i) xe = i == e ? x[i] : xe;
        push((vm >> e) & 1u, xe, base + elem_offset(lane, e));
      }
    }
  }
};

// R below this is computed again.
constexpr double TOP_RESCAN = 0x1p-100;

// TOP_WHOLE: a workgroup a row.  Few rows: TOP_PART, a workgroup for each part of a row, whose list
// and rest go to the workspace, and TOP_MERGE, a workgroup a row that joins the parts.
template <typename T, int MODE>
__global__ __launch_bounds__(TOP_NT) void top_kernel(TopParams P) {
  __shared__ TopShared sh;
  Block<TOP_NT, TopShared> B(sh);
  const int k = P.k, lane = B.lane;
  const int wave = __builtin_amdgcn_readfirstlane(B.wave);
  const int64_t items = MODE == TOP_PART ? P.n_rows * P.parts : P.n_rows;
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int64_t r = MODE == TOP_PART ? it / P.parts : it;
    const int part = MODE == TOP_PART ? static_cast<int>(it - r * P.parts) : 0;
    WaveTop<T> W;
    W.init(sh.list[wave], lane, k, P.c);
    float lo = finf(), hi = -finf();
    bool bad = false;
    float ref = -finf();      // TOP_MERGE: the parts' largest reference, which is no more than the
    double parts_rest = 0.0;  // row's k-th largest entry, and their rests relative to it
    if constexpr (MODE == TOP_MERGE) {
      for (int p = B.tid; p < P.parts; p += TOP_NT) ref = fmaxf(ref, P.info[r * P.parts + p].ref);
      ref = B.max(ref);
      for (int p = B.tid; p < P.parts; p += TOP_NT) {
        const TopPart f = P.info[r * P.parts + p];
        bad |= f.bad != 0;
        if (f.rest != 0.0) parts_rest += f.rest * exp2((static_cast<double>(f.ref) - ref) * P.c);
      }
      for (int p = wave; p < P.parts; p += TOP_NW)
        for (int i0 = 0; i0 < k; i0 += WAVE) {
          const int i = i0 + lane;
          const uint64_t u = i < k ? P.keys[(r * P.parts + p) * k + i] : 0ull;
          W.push(u != 0ull, TopKey<T>::value(static_cast<uint32_t>(u >> 32)), static_cast<int>(~static_cast<uint32_t>(u)));
        }
    } else {
      const int first = MODE == TOP_PART ? part * P.part_len : 0;
      const int len = MODE == TOP_PART ? min(P.part_len, P.V - first) : P.V;
      const T* row = static_cast<const T*>(P.x) + r * P.stride + first;
      const int chunks = (len + CHUNK - 1) / CHUNK, full = len / CHUNK;
      Frag<T> next;
      if (wave < full) frag_load<true>(next, row, wave, lane);
      for (int ch = wave; ch < chunks; ch += TOP_NW) {
        float x[EPL];
        uint32_t vm = 0xffffu;
        if (ch < full) {
          frag_unpack(next, x);
          if (ch + TOP_NW < full) frag_load<true>(next, row, ch + TOP_NW, lane);
        } else {
          load_lane<T, true>(row, ch, lane, len, x, &vm);
        }
        float lm = -finf();
        if (ch < full) {
#pragma unroll
          for (int e = 0; e < EPL; e += 2) {
            lm = max3_raw(lm, x[e], x[e + 1]);
            lo = min3_raw(lo, x[e], x[e + 1]);
          }
        } else {
#pragma unroll
          for (int e = 0; e < EPL; ++e)
            if ((vm >> e) & 1u) {
              lm = fmaxf(lm, x[e]);
              lo = fminf(lo, x[e]);
            }
        }
        hi = fmaxf(hi, lm);
        if (ch < full && !wave_any(lm > W.L)) {
          float s = 0.0f;
#pragma unroll
          for (int e = 0; e < EPL; ++e) s += fexp2((x[e] - W.L) * P.c);
          W.rest += static_cast<double>(s);
        } else {
          W.push_chunk(x, vm, first + ch * CHUNK);
        }
      }
    }
    if (W.n > k) W.shorten();
    // the block: its k largest of at most TOP_NW k
    if (lane == 0) sh.count[wave] = W.n;
    if (B.tid == 0) sh.n_best = 0;
    __syncthreads();
    int total = 0;
#pragma unroll
    for (int w = 0; w < TOP_NW; ++w) total += sh.count[w];
    uint64_t t = 1ull;
    float to;
    auto threshold = [&](auto entries) {
      constexpr int N = decltype(entries)::value;
      uint64_t u[N];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int w = i / (N / TOP_NW), j = (i % (N / TOP_NW)) * WAVE + lane;
        u[i] = j < sh.count[w] ? sh.list[w][j] : 0ull;
      }
      return top_threshold<T, N>(u, k);
    };
    if (total > k) {
      t = k <= WAVE ? threshold(std::integral_constant<int, TOP_NW>())
                    : threshold(std::integral_constant<int, TOP_NW * SAKI_MAX_TOP_K / WAVE>());
      to = TopKey<T>::value(static_cast<uint32_t>(t >> 32));
    } else {
      to = B.max(fmaxf(W.L, ref));  // (one wave, or one part, has all that there is)
    }
    // this wave's entries: to the block's list, or to the rest
    double rest = W.rest != 0.0 ? W.rest * exp2((static_cast<double>(W.L) - to) * P.c) : 0.0;
    for (int i0 = 0; i0 < W.n; i0 += WAVE) {
      const int i = i0 + lane;
      const uint64_t u = i < W.n ? sh.list[wave][i] : 0ull;
      if (u >= t) {
        sh.best[atomicAdd(&sh.n_best, 1)] = u;
      } else if (u != 0ull) {
        rest += static_cast<double>(fexp2((TopKey<T>::value(static_cast<uint32_t>(u >> 32)) - to) * P.c));
      }
    }
    if (MODE == TOP_MERGE && parts_rest != 0.0) rest += parts_rest * exp2((static_cast<double>(ref) - to) * P.c);
    double v[2];
    v[0] = rest;
    v[1] = (MODE != TOP_MERGE && !(lo > -finf() && hi < finf())) || bad ? 1.0 : 0.0;
    B.sum(v);
    const int n = sh.n_best;
    const bool wrong = v[1] != 0.0 || !(v[0] < __builtin_huge_val());
    if constexpr (MODE == TOP_PART) {
      uint64_t* keys = P.keys + it * k;
      for (int i = B.tid; i < k; i += TOP_NT) keys[i] = i < n ? sh.best[i] : 0ull;
      if (B.tid == 0) P.info[it] = TopPart{v[0], to, wrong ? 1 : 0};
    } else {
      // ranks by counting: all keys differ
      if (B.tid < n) {
        const uint64_t mine = sh.best[B.tid];
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += sh.best[j] > mine ? 1 : 0;
        sh.sorted[rank] = mine;
      }
      __syncthreads();
      if (B.tid < k) {
        const uint64_t u = B.tid < n ? sh.sorted[B.tid] : 0ull;
        const bool none = wrong || u == 0ull;
        P.top_logit[r * P.top_stride + B.tid] = none ? nanf_() : TopKey<T>::value(static_cast<uint32_t>(u >> 32));
        P.top_token[r * P.top_stride + B.tid] = none ? -1 : static_cast<int32_t>(~static_cast<uint32_t>(u));
      }
      double other = static_cast<double>(to) + log2(v[0]) / P.c;
      if (P.rest_logit && !wrong && v[0] < TOP_RESCAN && n < P.V) {
        const T* row = static_cast<const T*>(P.x) + r * P.stride;
        const uint64_t least = sh.sorted[n - 1];
        float m = -finf();
        auto others = [&](auto&& take) {
          for_chunks1<T, TOP_NW>(row, P.V, wave, lane, [&](auto tail, const float* x, uint32_t vm, int ch) {
            constexpr bool TAIL = decltype(tail)::value;
#pragma unroll
            for (int e = 0; e < EPL; ++e)
              if ((!TAIL || ((vm >> e) & 1u)) && WaveTop<T>::number(x[e], ch * CHUNK + elem_offset(lane, e)) < least) take(x[e]);
          });
        };
        others([&](float x) { m = fmaxf(m, x); });
        m = B.max(m);
        double s[1] = {0.0};
        others([&](float x) { s[0] += static_cast<double>(fexp2((x - m) * P.c)); });
        B.sum(s);
        other = static_cast<double>(m) + log2(s[0]) / P.c;
      }
      if (B.tid == 0) {
        if (P.rest_logit) P.rest_logit[r] = wrong ? nanf_() : n < P.V ? static_cast<float>(other) : -finf();
        if (P.row_status) P.row_status[r] = wrong ? SAKI_ROW_NONFINITE : SAKI_ROW_OK;
      }
    }
    __syncthreads();
  }
}

}  // namespace saki
