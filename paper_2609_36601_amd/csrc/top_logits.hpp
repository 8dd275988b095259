// The k largest logits of a row, best first, and the log-sum-exp of the others.
//
// One pass over the row.  Every wave keeps a list of candidates in LDS and a threshold L below which no
// entry is among the row's k largest.  An entry above L joins the list; any other is added at once to
//   R = sum 2^(x c - Lc),   c = log2(e) / tau,  Lc = L c rounded,
// whose terms are at most 1.  When a list is full, its k-th largest entry becomes L, the entries below it go to
// R, and R is brought to the new reference.  So R holds exactly the entries that are not listed: nothing is
// subtracted, and a rest of 1e-20 of the row is as exact as one of half of it.
//
// The first L is a guess: from the maxima of a sample of the row, so low that the entries above it are
// more than k with three standard deviations' certainty in a row without an order (some 200 to 600 of
// 151,936 at k of 20 to 256; without a guess each wave would see k (1 + log(entries / k)) candidates).  A row that has fewer
// than k entries above the guess is done again from L = -infinity.
//
// Candidates are rare in every lane and, k of them in 149 chunks, common in a wave: so a chunk costs the same with
// and without.  A lane whose largest entry is above L leaves its sum out and puts its 16 entries as they are
// into a queue in LDS; 64 such groups are looked into at a time.
//
// Equal entries: a candidate is the number (order-preserving image of the logit, ~index), so all differ.  An entry of a
// later chunk has to be above L, not at it; inside a chunk, and in the queue, the numbers are compared.
//
// Terms below 2^-126 are lost in 32 bits: where R ends below TOP_RESCAN (everything else lies far
// below the list, as with masked tokens), the row is read again with the reference at the largest
// entry that is not listed.
//
// What bounds it: many rows, memory (4,096 of 151,936 bf16, k 64: 242 us, 5.2 TB/s, VALU busy 0.75 of the CUs' cycles); few rows,
// the steps one behind the other (16 rows in 8 parts: 13 us, and 7 to join them).
#pragma once

#include "common.hpp"

namespace saki {

struct TopPart {
  double rest;  // sum over the part of 2^(x c - reference(L)), without its listed entries
  float L;
  int bad;  // an entry is not finite
};

struct TopParams {
  const void* x;
  int64_t n_rows;
  int64_t stride;
  int V;
  int k;
  int parts;     // a row's parts (TOP_PART, TOP_MERGE)
  float c;       // log2(e) / tau
  float* top_logit;
  int32_t* top_token;
  int64_t top_stride;
  float* rest_logit;
  uint8_t* row_status;
  uint64_t* keys;  // [n_rows, parts, k], 0: no entry
  TopPart* info;   // [n_rows, parts]
};

constexpr int TOP_NT = 256;
constexpr int TOP_NW = TOP_NT / WAVE;
// The sample of a row (or part) of `full` whole chunks: so many chunks of each wave.  Which of the 256 lanes' maxima is the
// guess: the q-th has about q len / sample entries above it, give or take a standard deviation of that for sqrt(q), and
// k <= (q - 3 sqrt(q)) len / sample.
__device__ __forceinline__ int top_sample(int full) { return full >= 64 ? 2 : full >= TOP_NW ? 1 : 0; }
__device__ __forceinline__ int top_rank(int k, int sample, int len) {
  const float want = static_cast<float>(k) * static_cast<float>(sample * TOP_NW * CHUNK) / static_cast<float>(len);
  const float root = 0.5f * (3.0f + __builtin_sqrtf(9.0f + 4.0f * want));
  return static_cast<int>(root * root) + 1;
}

enum TopMode { TOP_WHOLE, TOP_PART, TOP_MERGE };

constexpr int TOP_CAP = 384;   // candidates of a wave
constexpr int TOP_BEST = SAKI_MAX_TOP_K;
static_assert(TOP_CAP >= SAKI_MAX_TOP_K + 2 * WAVE, "a list that was shortened takes another 64 entries");
// R below this is computed again.
constexpr double TOP_RESCAN = 0x1p-100;

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

// Lc.  Where the product leaves the range: -3e38 keeps all terms at or below 1, +infinity makes them 0 (and the row is
// read again).
__device__ __forceinline__ float top_reference(float L, float c) {
  const float r = L * c;
  return r < -3.0e38f && L > -finf() ? -3.0e38f : r;
}

template <typename T>
struct TopShared {
  // Groups of the queue: TAKE at least (and 64 at most) are taken out at a time, 64 more come at most before that.
  // (f32: so that four workgroups fit a CU)
  static constexpr int TAKE = sizeof(T) == 2 ? 64 : 32, QUEUE = TAKE + WAVE;
  uint64_t list[TOP_NW][TOP_CAP];
  union {
    struct {
      uint4 group[TOP_NW][sizeof(T) == 2 ? 2 : 4][QUEUE];
      int place[TOP_NW][QUEUE];
    };
    struct {  // when the queues are empty
      uint64_t best[TOP_BEST];
      uint64_t sorted[TOP_BEST];
    };
    float maxima[TOP_NT];
  };
  int count[TOP_NW];
  int n_best;
  double red_d[TOP_NW][RED_MAX];
  float red_f[TOP_NW][4];
  int red_i[TOP_NW][4];
};

__device__ __forceinline__ int lanes_below(uint64_t m) {
  return __builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(m >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(m), 0));
}

// frag_unpack's inverse.
__device__ __forceinline__ void frag_pack(Frag<uint16_t>& f, const float (&x)[EPL]) {
  uint32_t w[EPL / 2];
#pragma unroll
  for (int i = 0; i < EPL / 2; ++i) w[i] = __float_as_uint(x[2 * i]) >> 16 | (__float_as_uint(x[2 * i + 1]) & 0xffff0000u);
  f.q[0] = make_uint4(w[0], w[1], w[2], w[3]);
  f.q[1] = make_uint4(w[4], w[5], w[6], w[7]);
}
__device__ __forceinline__ void frag_pack(Frag<float>& f, const float (&x)[EPL]) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    f.q[i] = make_uint4(__float_as_uint(x[4 * i]), __float_as_uint(x[4 * i + 1]), __float_as_uint(x[4 * i + 2]), __float_as_uint(x[4 * i + 3]));
}

// How many of a wave's numbers u reach t.
template <typename U, int N>
__device__ __forceinline__ int top_reach(const U (&u)[N], U t) {
  int n = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) n += __popcll(__ballot(u[i] >= t));
  return n;
}

// The largest number that k of a wave's u reach, bit by bit from `bit` down.
template <typename U, int N>
__device__ __forceinline__ U top_search(const U (&u)[N], int k, int bit, U found = 0) {
  for (int b = bit; b >= 0; --b) {
    const U t = found | (U{1} << b);
    if (top_reach(u, t) >= k) found = t;
  }
  return found;
}

// A wave's candidates.
template <typename T>
struct WaveTop {
  static constexpr int PIECES = sizeof(T) == 2 ? 2 : 4;  // 16-byte pieces of a lane's 16 entries
  uint64_t* list;  // LDS
  int lane, k;
  float c;
  int n;        // candidates in the list (the same in all lanes)
  float L, Lc;  // the threshold, and R's reference
  uint64_t t;   // a candidate's number is above it
  double rest;  // this lane's part of R

  __device__ __forceinline__ void start(float L_, uint64_t t_) {
    n = 0;
    L = L_;
    Lc = top_reference(L, c);
    t = t_;
    rest = 0.0;
  }

  static __device__ __forceinline__ uint64_t number(float x, int index) {
    return static_cast<uint64_t>(TopKey<T>::of(x)) << 32 | static_cast<uint32_t>(~index);
  }
  static __device__ __forceinline__ float value(uint64_t u) { return TopKey<T>::value(static_cast<uint32_t>(u >> 32)); }
  __device__ __forceinline__ float term(float x) const { return fexp2(__builtin_fmaf(x, c, -Lc)); }

  // Keeps the k largest candidates; the others go to the rest.
  __device__ __forceinline__ void shorten() {
    constexpr int N = TOP_CAP / WAVE;
    uint32_t hi[N], lo[N];
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint64_t u = i * WAVE + lane < n ? list[i * WAVE + lane] : 0ull;
      hi[i] = static_cast<uint32_t>(u >> 32);
      lo[i] = static_cast<uint32_t>(u);
    }
    const uint32_t th = top_search(hi, k, TopKey<T>::BITS - 1);
    uint32_t tl = 0u;
    const int above = top_reach(hi, th + 1u);
    if (top_reach(hi, th) > k) {  // those at the k-th value with the lowest indices
      uint32_t w[N];
#pragma unroll
      for (int i = 0; i < N; ++i) w[i] = hi[i] == th ? lo[i] : 0u;
      tl = top_search(w, k - above, 31);
    }
    t = static_cast<uint64_t>(th) << 32 | tl;
    const float before = Lc;
    L = TopKey<T>::value(th);
    Lc = top_reference(L, c);
    rest = rest != 0.0 ? rest * static_cast<double>(fexp2(before - Lc)) : 0.0;
    int m = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const bool keep = hi[i] > th || (hi[i] == th && lo[i] >= tl);
      const uint64_t who = __ballot(keep);
      if (keep) list[m + lanes_below(who)] = static_cast<uint64_t>(hi[i]) << 32 | lo[i];
      else if (hi[i] != 0u) rest += static_cast<double>(term(TopKey<T>::value(hi[i])));
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
    if (there && !in) rest += static_cast<double>(term(x));
  }

  // 16 entries of each lane in `mine` (-infinity: none), that of e at index base + elem_offset(0, e).
  __device__ __forceinline__ void push_group(bool mine, const float (&x)[EPL], int base) {
    int more = 0;
#pragma unroll
    for (int e = 0; e < EPL; ++e) more += __popcll(__ballot(mine && x[e] >= L));
    // all lanes, or where the list might overflow, so few at a time that a list that was shortened holds theirs
    constexpr int FEW = (TOP_CAP - SAKI_MAX_TOP_K) / EPL;
    const int step = n + more <= TOP_CAP ? WAVE : FEW;
#pragma unroll 1
    for (int l0 = 0; l0 < WAVE; l0 += step) {
      if (step < WAVE && n + FEW * EPL > TOP_CAP) shorten();
      const bool now = mine && lane >= l0 && lane < l0 + step;
      float s = 0.0f;
#pragma unroll
      for (int e = 0; e < EPL; ++e) {
        const bool there = now && x[e] != -finf();
        bool in = there && x[e] >= L;
        if (__ballot(in) != 0ull) {
          const uint64_t u = number(x[e], base + elem_offset(0, e));
          in = in && u > t;
          const uint64_t who = __ballot(in);
          if (in) list[n + lanes_below(who)] = u;
          n += __popcll(who);
        }
        s += there && !in ? term(x[e]) : 0.0f;
      }
      rest += static_cast<double>(s);
    }
  }
};

// 2^d to 32 bits' precision, of any size.
__device__ __forceinline__ double top_exp2(double d) {
  const double whole = rint(fmax(d, -2000.0));
  return ldexp(static_cast<double>(fexp2(static_cast<float>(d - whole))), static_cast<int>(whole));
}
// log2 of x > 0, off by some 2^-23.
__device__ __forceinline__ double top_log2(double x) {
  int e;
  const double m = frexp(x, &e);
  return static_cast<double>(flog2(static_cast<float>(m))) + e;
}

// TOP_WHOLE: a workgroup a row.  Few rows: TOP_PART, a workgroup for each part of a row, whose list
// and rest go to the workspace, and TOP_MERGE, a workgroup a row that joins the parts.
template <typename T, int MODE>
__global__ __launch_bounds__(TOP_NT, 4) void top_kernel(TopParams P) {
  __shared__ TopShared<T> sh;
  Block<TOP_NT, TopShared<T>> B(sh);
  constexpr int PIECES = WaveTop<T>::PIECES;
  const int k = P.k, lane = B.lane;
  const int wave = __builtin_amdgcn_readfirstlane(B.wave);
  const int64_t items = MODE == TOP_PART ? P.n_rows * P.parts : P.n_rows;
  WaveTop<T> W;
  W.list = sh.list[wave];
  W.lane = lane;
  W.k = k;
  W.c = P.c;
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int64_t r = MODE == TOP_PART ? it / P.parts : it;
    const int part = MODE == TOP_PART ? static_cast<int>(it - r * P.parts) : 0;
    // (parts of whole chunks, as even as they can be)
    const int all_chunks = (P.V + CHUNK - 1) / CHUNK;
    const int first = MODE == TOP_PART ? part * all_chunks / P.parts * CHUNK : 0;
    const int len = MODE == TOP_PART ? min((part + 1) * all_chunks / P.parts * CHUNK, P.V) - first : P.V;
    const T* row = static_cast<const T*>(P.x) + r * P.stride + first;
    const int chunks = (len + CHUNK - 1) / CHUNK, full = len / CHUNK;
    float lo = finf(), hi = -finf();
    bool bad = false;
    float ref = -finf();      // TOP_MERGE: the parts' largest reference, and their rests relative to it
    double parts_rest = 0.0;
    int total;
    W.start(-finf(), 0ull);
    if constexpr (MODE == TOP_MERGE) {
      // the parts' largest threshold is the row's
      float L = -finf();
      for (int p = B.tid; p < P.parts; p += TOP_NT) L = fmaxf(L, P.info[r * P.parts + p].L);
      L = B.max(L);
      ref = top_reference(L, P.c);
      for (int p = B.tid; p < P.parts; p += TOP_NT) {
        const TopPart f = P.info[r * P.parts + p];
        bad |= f.bad != 0;
        if (f.rest != 0.0) parts_rest += f.rest * top_exp2(static_cast<double>(top_reference(f.L, P.c)) - ref);
      }
      if (L > -finf()) W.start(L, static_cast<uint64_t>(TopKey<T>::of(L)) << 32);
      for (int p = wave; p < P.parts; p += TOP_NW)
        for (int i0 = 0; i0 < k; i0 += WAVE) {
          const int i = i0 + lane;
          const uint64_t u = i < k ? P.keys[(r * P.parts + p) * k + i] : 0ull;
          W.push(u != 0ull, WaveTop<T>::value(u), static_cast<int>(~static_cast<uint32_t>(u)));
        }
    } else if (const int sample = top_sample(full), rank = top_rank(k, sample, len); sample > 0 && rank <= TOP_NT / 2) {
      // the guess (of more maxima it would be no better than a wave's own threshold)
      float m = -finf();
      for (int s = 0; s < sample; ++s) {
        Frag<T> f;
        float x[EPL];
        frag_load<false>(f, row, static_cast<int>(static_cast<int64_t>(s * TOP_NW + wave) * full / (TOP_NW * sample)), lane);
        frag_unpack(f, x);
#pragma unroll
        for (int e = 0; e < EPL; e += 2) m = max3_raw(m, x[e], x[e + 1]);
      }
      sh.maxima[B.tid] = m;
      __syncthreads();
      uint32_t u[TOP_NW];
#pragma unroll
      for (int w = 0; w < TOP_NW; ++w) u[w] = TopKey<T>::of(sh.maxima[w * WAVE + lane]);
      const uint32_t g = top_search(u, rank, TopKey<T>::BITS - 1);
      const float L = TopKey<T>::value(g);
      if (L > -finf() && L < finf()) W.start(L, static_cast<uint64_t>(g) << 32 | 0xffffffffu);
      __syncthreads();
    }
    for (int attempt = 0;; ++attempt) {
      if constexpr (MODE != TOP_MERGE) {
        int queued = 0, ch = wave;
        // looks into 64 groups of the queue (the last ones)
        auto take = [&]() __attribute__((always_inline)) {
          __builtin_amdgcn_wave_barrier();
          const int from = max(queued - WAVE, 0), at = min(from + lane, queued - 1);
          const bool mine = from + lane < queued;
          Frag<T> f;
#pragma unroll
          for (int i = 0; i < PIECES; ++i) f.q[i] = sh.group[wave][i][at];
          const int place = sh.place[wave][at];
          float x[EPL];
          frag_unpack(f, x);
          __builtin_amdgcn_wave_barrier();
          W.push_group(mine, x, first + place);
          queued = from;
        };
        // a chunk of which lanes in `some` have entries
        auto chunk = [&](const Frag<T>& f, const float (&x)[EPL], bool some, int c) __attribute__((always_inline)) {
          float lm = max3_raw(x[0], x[1], x[2]), s = 0.0f;
          lm = max3_raw(lm, x[3], x[3]);
#pragma unroll
          for (int e = 4; e < EPL; e += 2) lm = max3_raw(lm, x[e], x[e + 1]);
#pragma unroll
          for (int e = 0; e < EPL; ++e) s += W.term(x[e]);
          hi = fmaxf(hi, lm);
          const bool in = lm > W.L;
          W.rest += static_cast<double>(in || !some ? 0.0f : s);
          const uint64_t who = __ballot(in);
          if (who != 0ull) {
            if (in) {
              const int at = queued + lanes_below(who);
#pragma unroll
              for (int i = 0; i < PIECES; ++i) sh.group[wave][i][at] = f.q[i];
              sh.place[wave][at] = c * CHUNK + 8 * lane;
            }
            queued += __popcll(who);
          }
        };
        auto whole = [&](const Frag<T>& f, int c) __attribute__((always_inline)) {
          float x[EPL];
          frag_unpack(f, x);
#pragma unroll
          for (int e = 0; e < EPL; e += 2) lo = min3_raw(lo, x[e], x[e + 1]);
          chunk(f, x, true, c);
        };
        // two buffers in turn, loads on every path (see for_chunks)
        if (ch < full) {
          Frag<T> a, b;
          frag_load<false>(a, row, ch, lane);
          frag_load<false>(b, row, ch + TOP_NW < full ? ch + TOP_NW : ch, lane);
          for (;;) {
            whole(a, ch);
            frag_load<false>(a, row, ch + 2 * TOP_NW < full ? ch + 2 * TOP_NW : ch, lane);
            if (queued >= TopShared<T>::TAKE) take();
            ch += TOP_NW;
            if (ch >= full) break;
            whole(b, ch);
            frag_load<false>(b, row, ch + 2 * TOP_NW < full ? ch + 2 * TOP_NW : ch, lane);
            if (queued >= TopShared<T>::TAKE) take();
            ch += TOP_NW;
            if (ch >= full) break;
          }
        }
        if (ch == full && ch < chunks) {  // the last entries; -infinity where there are none
          float x[EPL];
          uint32_t vm;
          load_lane<T, true>(row, ch, lane, len, x, &vm);
#pragma unroll
          for (int e = 0; e < EPL; ++e) {
            const bool there = (vm >> e) & 1u;
            lo = there ? fminf(lo, x[e]) : lo;
            x[e] = there ? x[e] : -finf();
          }
          Frag<T> f;
          frag_pack(f, x);
          chunk(f, x, vm != 0u, ch);
        }
        while (queued > 0) take();
      }
      if (lane == 0) sh.count[wave] = W.n;
      if (B.tid == 0) sh.n_best = 0;
      __syncthreads();
      total = 0;
#pragma unroll
      for (int w = 0; w < TOP_NW; ++w) total += sh.count[w];
      // fewer than there are: the guess was too high
      if (MODE == TOP_MERGE || attempt > 0 || uniform(total >= min(k, len))) break;
      W.start(-finf(), 0ull);
      __syncthreads();
    }
    // the block's k largest: those that reach the k-th value, or where more than LDS holds tie at it, those
    // with the lowest indices
    uint64_t t = 1ull;
    float to;
    auto threshold = [&](auto entries) {
      constexpr int N = decltype(entries)::value;
      uint32_t v[N], low[N];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int w = i / (N / TOP_NW), j = (i % (N / TOP_NW)) * WAVE + lane;
        const uint64_t u = j < sh.count[w] ? sh.list[w][j] : 0ull;
        v[i] = static_cast<uint32_t>(u >> 32);
        low[i] = static_cast<uint32_t>(u);
      }
      const uint32_t th = top_search(v, k, TopKey<T>::BITS - 1);
      uint32_t tl = 0u;
      if (top_reach(v, th) > TOP_BEST) {
        const int above = top_reach(v, th + 1u);
#pragma unroll
        for (int i = 0; i < N; ++i) low[i] = v[i] == th ? low[i] : 0u;
        tl = top_search(low, k - above, 31);
      }
      return static_cast<uint64_t>(th) << 32 | tl;
    };
    if (total > k) {
      const bool few = max(max(sh.count[0], sh.count[1]), max(sh.count[2], sh.count[3])) <= 2 * WAVE;
      t = uniform(few) ? threshold(std::integral_constant<int, 2 * TOP_NW>())
                       : threshold(std::integral_constant<int, TOP_NW * TOP_CAP / WAVE>());
      to = WaveTop<T>::value(t);
    } else {
      to = B.max(W.L);  // (one wave, or one part, has all that there is)
    }
    // this wave's entries: to the block's list, or to the rest
    const float to_c = top_reference(to, P.c);
    double rest = W.rest != 0.0 ? W.rest * top_exp2(static_cast<double>(W.Lc) - to_c) : 0.0;
    for (int i0 = 0; i0 < W.n; i0 += WAVE) {
      const int i = i0 + lane;
      const uint64_t u = i < W.n ? sh.list[wave][i] : 0ull;
      if (u >= t) {
        sh.best[atomicAdd(&sh.n_best, 1)] = u;
      } else if (u != 0ull) {
        rest += static_cast<double>(fexp2(__builtin_fmaf(WaveTop<T>::value(u), P.c, -to_c)));
      }
    }
    if (MODE == TOP_MERGE && parts_rest != 0.0) rest += parts_rest * top_exp2(static_cast<double>(ref) - to_c);
    double v[2];
    v[0] = rest;
    v[1] = (MODE != TOP_MERGE && !(lo > -finf() && hi < finf())) || bad ? 1.0 : 0.0;
    B.sum(v);
    const int found = sh.n_best, n = min(found, k);
    // ranks by counting: all numbers differ; what ties behind the k-th place is at `to`, a term of 1 (or of what the
    // rounding of the reference leaves)
    if (B.tid < found) {
      const uint64_t mine = sh.best[B.tid];
      int rank = 0;
      for (int j = 0; j < found; ++j) rank += sh.best[j] > mine ? 1 : 0;
      sh.sorted[rank] = mine;
    }
    __syncthreads();
    if (found > n) v[0] += static_cast<double>(found - n) * static_cast<double>(fexp2(__builtin_fmaf(to, P.c, -to_c)));
    const bool wrong = v[1] != 0.0 || !(v[0] < __builtin_huge_val());
    if constexpr (MODE == TOP_PART) {
      uint64_t* keys = P.keys + it * k;
      for (int i = B.tid; i < k; i += TOP_NT) keys[i] = i < n ? sh.sorted[i] : 0ull;
      if (B.tid == 0) P.info[it] = TopPart{v[0], to, wrong ? 1 : 0};
    } else {
      if (B.tid < k) {
        const uint64_t u = B.tid < n ? sh.sorted[B.tid] : 0ull;
        const bool none = wrong || u == 0ull;
        P.top_logit[r * P.top_stride + B.tid] = none ? nanf_() : WaveTop<T>::value(u);
        P.top_token[r * P.top_stride + B.tid] = none ? -1 : static_cast<int32_t>(~static_cast<uint32_t>(u));
      }
      double other = (static_cast<double>(to_c) + top_log2(v[0])) / P.c;
      if (P.rest_logit && uniform(!wrong && v[0] < TOP_RESCAN && n < P.V)) {
        const T* whole = static_cast<const T*>(P.x) + r * P.stride;
        const uint64_t least = sh.sorted[n - 1];
        float m = -finf();
        double s[1] = {0.0};
#pragma unroll 1
        for (int pass = 0; pass < 2; ++pass) {
          for (int ch = wave; ch < (P.V + CHUNK - 1) / CHUNK; ch += TOP_NW) {
            float x[EPL];
            uint32_t vm;
            load_lane<T, true>(whole, ch, lane, P.V, x, &vm);
            float sum = 0.0f;
#pragma unroll
            for (int e = 0; e < EPL; ++e)
              if (((vm >> e) & 1u) && WaveTop<T>::number(x[e], ch * CHUNK + elem_offset(lane, e)) < least) {
                if (pass == 0) m = fmaxf(m, x[e]);
                sum += fexp2((x[e] - m) * P.c);
              }
            s[0] += static_cast<double>(sum);
          }
          if (pass == 0) {
            m = B.max(m);
            s[0] = 0.0;
          }
        }
        B.sum(s);
        other = static_cast<double>(m) + top_log2(s[0]) / P.c;
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
