// Attention of new tokens over the pages of a key-value cache.
//
// Rows.  The query heads that share a key head are rows of one product: row
// r = j * group + g of sequence b and key head h is token j, query head h * group + g.
// A unit is a tile of rows of one sequence and key head; its keys may be split over
// several items (workgroups), whose results kv_join_kernel puts together.
//
// Products.  S^T = K Q^T and O^T = V^T P^T on the matrix cores, with 16 x 16
// tiles: a lane then holds the scores of one row (its column) for the same tokens that
// it needs of P as the second product's operand, so P never leaves the registers.
// The order of the summed index is free in both products, and is chosen so that every
// lane reads 16 consecutive bytes: of a key (the row's elements), and of eight tokens'
// values, whose 8 x 8 block the lane transposes itself (bf16).
//
// Softmax.  One pass with the running maximum m and sum l of each row.  m only moves
// when a score passes it by more than 2^8: P is then at most 256 times what it
// would be, which 32-bit sums and bf16's exponent hold alike, and most blocks need no
// exchange between lanes and no rescaling of O.
#pragma once

#include <type_traits>

#include "kv_append.hpp"

namespace saki {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int KV_ATT_NT = 256;
constexpr int KV_ATT_WAVES = KV_ATT_NT / KV_WAVE;
constexpr int KV_ATT_ROWS = 64;    // most rows of a tile
constexpr int KV_ATT_ITEMS = 1024; // items that a call is split into where it has fewer units
constexpr float KV_LOG2E = 1.44269504088896340736f;
constexpr float KV_LN2 = 0.693147180559945309417f;

struct KvAttnParams {
  KvTable t;
  KvPool p;  // bases of the layer
  KvTokens n;
  KvStrides q, out;
  float* lse;
  int n_q_heads, group;
  float scale2;  // scale * log2 e
  int window, sinks;
  int items;     // target of the split
  float* part;   // [slots][rows][DP] partial sums, then
  float* part_ml;  // [slots][rows][2] their maximum and sum
  int slots;
  unsigned* split_units;  // how many units are split, for kv_join_kernel
};

// Blocks of BLK tokens that the rows of tokens [j0, j1) (positions p0 .. p1 - 1) see:
// the first `sink` blocks, then those from token `lo` on.
struct KvSpan {
  int lo;     // first token of the main part, a multiple of BLK
  int sinks;  // blocks of the sinks
  int blocks; // of both
};
template <int BLK>
__device__ __forceinline__ KvSpan kv_span(int64_t p0, int64_t p1, int window, int sinks) {
  KvSpan s{0, 0, 0};
  if (window > 0) {
    const int64_t lo = p0 - window + 1;
    s.lo = lo > 0 ? static_cast<int>(lo / BLK) * BLK : 0;
    const int n = sinks < s.lo ? sinks : s.lo;
    s.sinks = (n + BLK - 1) / BLK;
  }
  s.blocks = s.sinks + static_cast<int>((p1 - s.lo + BLK - 1) / BLK);
  return s;
}

// A sequence's share of the call: its tiles, and the blocks of its largest tile.
struct KvLoad {
  int first, count;  // token rows
  int64_t start;     // position of the first
  int tiles;
  int blocks;
  bool fine;
};
template <int ROWS, int BLK>
__device__ __forceinline__ KvLoad kv_load_of(const KvAttnParams& P, int b) {
  KvLoad s;
  kv_rows(P.n, b, &s.first, &s.count);
  s.start = static_cast<int64_t>(P.t.length[b]) + P.n.shift;
  s.tiles = static_cast<int>((static_cast<int64_t>(s.count) * P.group + ROWS - 1) / ROWS);
  const int64_t end = s.start + s.count;
  s.fine = P.t.length[b] >= 0 && end <= (static_cast<int64_t>(kv_held(P.t, b)) << P.t.shift);
  s.blocks = 1;
  if (s.fine && s.count > 0) {
    if (P.window > 0) {
      // the widest tile: at most ROWS rows, which span so many tokens
      const int span = s.count < (ROWS + P.group - 2) / P.group + 1 ? s.count : (ROWS + P.group - 2) / P.group + 1;
      const KvSpan a = kv_span<BLK>(end - span, end, P.window, P.sinks);
      s.blocks = a.blocks + (span < s.count ? 1 : 0);
    } else {
      s.blocks = static_cast<int>((end + BLK - 1) / BLK);
    }
  }
  return s;
}

// Where an item stands in the call.
struct KvItem {
  int b, first, count;
  int start;
  int tile, head, split, splits, slot;
  int fine;
};

// Finds item `item` of the call, or (JOIN) split unit `item`; every workgroup derives the
// split from the lengths by itself, which spares a launch.  Items of a sequence are
// ordered by tile (last first: with causal rows those are the longest), split, key
// head, so that the workgroups of one key head, which read the same keys, tend to
// one XCD.  False: there is no such item.
template <int ROWS, int BLK, bool JOIN>
__device__ __forceinline__ bool kv_find_item(const KvAttnParams& P, int64_t item, KvItem* out) {
  __shared__ long long part[KV_ATT_WAVES];
  __shared__ KvItem found;
  __shared__ int is_found;
  const int tid = threadIdx.x;
  const int Hk = P.p.n_heads;
  const int per = (P.t.n_seq + KV_ATT_NT - 1) / KV_ATT_NT;
  const int b0 = tid * per, b1 = b0 + per < P.t.n_seq ? b0 + per : P.t.n_seq;
  if (tid == 0) is_found = 0;
  long long blocks = 0, all = 0;
  KvLoad keep;  // the thread's only sequence where it has one
  for (int b = b0; b < b1; ++b) {
    keep = kv_load_of<ROWS, BLK>(P, b);
    blocks += static_cast<long long>(keep.tiles) * keep.blocks;
  }
  kv_block_scan<KV_ATT_NT, long long>(blocks, part, &all);
  // blocks an item takes: what gives the call P.items of them, and at least one
  // block for each wave twice
  long long len = (all * Hk + P.items - 1) / P.items;
  if (len < 2 * KV_ATT_WAVES) len = 2 * KV_ATT_WAVES;
  auto splits_of = [&](const KvLoad& s) { return static_cast<int>((s.blocks + len - 1) / len); };
  long long items = 0, slots = 0, split_units = 0;
  for (int b = b0; b < b1; ++b) {
    const KvLoad s = per == 1 ? keep : kv_load_of<ROWS, BLK>(P, b);
    const int n = splits_of(s);
    if (n > 1) split_units += static_cast<long long>(s.tiles) * Hk;
    items += static_cast<long long>(s.tiles) * Hk * (JOIN ? n > 1 : n);
    if (n > 1) slots += static_cast<long long>(s.tiles) * Hk * n;
  }
  // (both sums in one scan: at most 2^31 items, as the grid is)
  long long sums = 0;
  const long long before = kv_block_scan<KV_ATT_NT, long long>((slots << 32) | items, part, &sums);
  if (!JOIN && blockIdx.x == 0) {
    long long n = 0;
    kv_block_scan<KV_ATT_NT, long long>(split_units, part, &n);
    if (tid == 0) *P.split_units = n < P.items ? static_cast<unsigned>(n) : static_cast<unsigned>(P.items);
  }
  long long at = before & 0xffffffffll, slot = before >> 32;
  if (item >= at && item < at + items) {
    for (int b = b0; b < b1; ++b) {
      const KvLoad s = per == 1 ? keep : kv_load_of<ROWS, BLK>(P, b);
      const int n = splits_of(s);
      const long long mine = static_cast<long long>(s.tiles) * Hk * (JOIN ? n > 1 : n);
      if (item < at + mine) {
        int i = static_cast<int>(item - at);
        KvItem f;
        f.head = i % Hk;
        i /= Hk;
        f.split = JOIN ? 0 : i % n;
        const int tile_back = JOIN ? i : i / n;
        f.tile = s.tiles - 1 - tile_back;
        f.b = b;
        f.first = s.first;
        f.count = s.count;
        f.start = static_cast<int>(s.start);
        f.fine = s.fine;
        f.splits = n;
        // slots of a unit are consecutive
        f.slot = static_cast<int>(slot) + (tile_back * Hk + f.head) * n + f.split;
        found = f;
        is_found = 1;
        break;
      }
      at += mine;
      if (n > 1) slot += static_cast<long long>(s.tiles) * Hk * n;
    }
  }
  __syncthreads();
  // (the same for the whole workgroup: in scalar registers)
  const int* f = reinterpret_cast<const int*>(&found);
  int* o = reinterpret_cast<int*>(out);
#pragma unroll
  for (int i = 0; i < static_cast<int>(sizeof(KvItem) / 4); ++i) o[i] = __builtin_amdgcn_readfirstlane(f[i]);
  return __builtin_amdgcn_readfirstlane(is_found) != 0;
}

// Workgroups that the registers of a CU hold (one wave of each on every SIMD).
template <typename T>
constexpr int kv_groups_per_cu(int dp, int r) {
  return dp * r <= 64 ? 4 : dp * r <= 128 ? 3 : dp * r <= 256 ? 2 : 1;
}

template <typename T>
struct KvBlk {
  static constexpr int N = sizeof(T) == 2 ? 32 : 16;  // tokens of a wave's step
};

// Parts of a value (a pair of them in bf16): SIGN 0, the value if it is finite, else 0;
// SIGN 1 (-1), one where it is +infinity (-infinity) or NaN, else 0.
template <typename T, int SIGN>
__device__ __forceinline__ uint32_t kv_select(uint32_t v) {
  constexpr uint32_t EXP = sizeof(T) == 2 ? 0x7f80u : 0x7f800000u, MAG = EXP | (EXP - 1);
  constexpr uint32_t ONE = sizeof(T) == 2 ? 0x3f80u : 0x3f800000u, SIGN_BIT = MAG + 1;
  auto one = [](uint32_t x) -> uint32_t {
    const bool finite = (x & EXP) != EXP, nan = (x & MAG) > EXP, minus = (x & SIGN_BIT) != 0;
    if (SIGN == 0) return finite ? x : 0u;
    return !finite && (nan || minus == (SIGN < 0)) ? ONE : 0u;
  };
  if constexpr (sizeof(T) == 4) return one(v);
  return one(v & 0xffffu) | one(v >> 16) << 16;
}

// One item: ROWS = 16 R rows, the blocks of its split dealt to the four waves.
template <typename T, int DP, int R>
__global__ __launch_bounds__(KV_ATT_NT, kv_groups_per_cu<T>(DP, R)) void kv_attention_kernel(KvAttnParams P) {
  constexpr bool BF = sizeof(T) == 2;
  constexpr int BLK = KvBlk<T>::N;
  constexpr int ROWS = 16 * R;
  constexpr int NT = DP / 16;              // 16-wide tiles of the head: a lane's elements of a value row
  constexpr int QC = BF ? DP / 32 : DP / 16;  // 16-byte pieces of a lane's share of a key row
  constexpr int TOK = BF ? 8 : 4;          // tokens of a lane in a block
  constexpr int VW = NT * sizeof(T) / 4;   // 32-bit words of a lane's share of a value row
  using VPiece = typename std::conditional<(VW >= 4), uint4, uint2>::type;
  constexpr int VC = VW * 4 / sizeof(VPiece), VE = sizeof(VPiece) / sizeof(T);  // its loads, elements of a load
  __shared__ float join_o[KV_ATT_WAVES][16][DP + 4];
  __shared__ float join_m[KV_ATT_WAVES][ROWS], join_l[KV_ATT_WAVES][ROWS];

  KvItem it;
  if (!kv_find_item<ROWS, BLK, false>(P, blockIdx.x, &it)) return;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / KV_WAVE), lane = tid & (KV_WAVE - 1);
  const int c = lane & 15, g = lane >> 4;
  const int D = P.p.dim, G = P.group;
  const int row0 = it.tile * ROWS, rows = it.count * G;
  const int n_rows = rows - row0 < ROWS ? rows - row0 : ROWS;
  const int j0 = row0 / G, j1 = (row0 + n_rows - 1) / G + 1;
  const int p0 = it.start + j0, p1 = it.start + j1;  // positions of the tile's tokens
  bool bad = !it.fine;

  // this lane's rows
  int pos[R];
  uint4 qf[R][QC];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int row = 16 * r + c;
    const bool real = row < n_rows;
    const int rr = row0 + (real ? row : n_rows - 1);
    const int j = rr / G, head = it.head * G + rr - j * G;
    pos[r] = it.start + j;
    const char* src = P.q.data + (it.first + j) * P.q.token + head * P.q.head;
#pragma unroll
    for (int i = 0; i < QC; ++i) {
      const int d = i * (BF ? 32 : 16) + g * (BF ? 8 : 4);
      qf[r][i] = d < D ? *reinterpret_cast<const uint4*>(src + d * sizeof(T)) : uint4{0, 0, 0, 0};
    }
  }

  f32x4 acc[R][NT];
  float m[R], l[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    m[r] = -INFINITY;
    l[r] = 0.0f;
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[r][t] = f32x4{0, 0, 0, 0};
  }

  if (it.fine) {
    const KvSpan span = kv_span<BLK>(p0, p1, P.window, P.sinks);
    const int from = static_cast<int>(static_cast<int64_t>(span.blocks) * it.split / it.splits);
    const int to = static_cast<int>(static_cast<int64_t>(span.blocks) * (it.split + 1) / it.splits);
    const int32_t* row_pages = P.t.pages + static_cast<int64_t>(it.b) * P.t.max_pages;
    const int mask = (1 << P.t.shift) - 1;
    const char* kb = P.p.k + it.head * P.p.head_stride;
    const char* vb = P.p.v + it.head * P.p.head_stride;
    const int last = p1 - 1;  // no lane reads behind the tile's last token
    // first token of block i
    auto token_of = [&](int i) { return i < span.sinks ? i * BLK : span.lo + (i - span.sinks) * BLK; };
    // The runs of 8 tokens that hold this lane's keys and values in the block at t0 (runs behind the
    // last token: that token's); a run lies in one page, whose id is looked up once.
    auto run_of = [&](int tok) { return tok <= last ? tok & ~7 : last & ~7; };
    const int k_in = BF ? (c >> 2) * 8 : c, v_in = g * TOK;
    int k_id = 0, v_id = 0;
    auto load_ids = [&](int t0) {
      k_id = row_pages[run_of(t0 + k_in) >> P.t.shift];
      v_id = row_pages[run_of(t0 + v_in) >> P.t.shift];
    };
    auto page_at = [&](int id) {
      const bool in = id >= 0 && id < P.t.n_pages;
      bad |= !in;
      return static_cast<int64_t>(in ? id : 0) * P.p.page_stride;
    };
    uint4 kf[BF ? 2 : 1][QC];
    uint32_t vr[TOK][VW];
    const int token_stride = static_cast<int>(P.p.token_stride);
    auto load_keys = [&](int t0) {
      const int run = run_of(t0 + k_in);
      const char* src = kb + page_at(k_id) + (g * 16);
#pragma unroll
      for (int s = 0; s < (BF ? 2 : 1); ++s) {
        int tok = BF ? run + (c & 3) + 4 * s : run + (c & 7);
        tok = tok < last ? tok : last;
        const char* at = src + static_cast<int64_t>(tok & mask) * token_stride;
#pragma unroll
        for (int e = 0; e < QC; ++e)
          kf[s][e] = e * 64 + g * 16 < D * static_cast<int>(sizeof(T)) ? *reinterpret_cast<const uint4*>(at + e * 64)
                                                                       : uint4{0, 0, 0, 0};
      }
    };
    auto load_values = [&](int t0) {
      const int run = run_of(t0 + v_in);
      const char* src = vb + page_at(v_id) + c * NT * static_cast<int>(sizeof(T));
#pragma unroll
      for (int e = 0; e < TOK; ++e) {
        int tok = run + (BF ? 0 : v_in & 7) + e;
        tok = tok < last ? tok : last;
        const char* at = src + static_cast<int64_t>(tok & mask) * token_stride;
#pragma unroll
        for (int w = 0; w < VC; ++w) {
          const VPiece x = c * NT + w * VE < D ? reinterpret_cast<const VPiece*>(at)[w] : VPiece{};
          __builtin_memcpy(&vr[e][w * sizeof(VPiece) / 4], &x, sizeof(x));
        }
      }
    };
    // The next block's keys are loaded once this block's are multiplied, and its values
    // once this block's are: both are under way while the rest of a block is computed.
    int i = from + wave;
    if (i < to) {
      load_ids(token_of(i));
      load_keys(token_of(i));
      load_values(token_of(i));
    }
    while (i < to) {
      const int t0 = token_of(i), vt0 = t0 + v_in;
      const int next = i + KV_ATT_WAVES;
      const int t_next = token_of(next);
      if (next < to) load_ids(t_next);
      // scores
      f32x4 s[R][BF ? 2 : 1];
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int u = 0; u < (BF ? 2 : 1); ++u) {
          f32x4 x{0, 0, 0, 0};
#pragma unroll
          for (int e = 0; e < QC; ++e) {
            if constexpr (BF) {
              x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf[u][e]),
                                                          __builtin_bit_cast(bf16x8, qf[r][e]), x, 0, 0, 0);
            } else {
              const f32x4 a = __builtin_bit_cast(f32x4, kf[u][e]), z = __builtin_bit_cast(f32x4, qf[r][e]);
#pragma unroll
              for (int w = 0; w < 4; ++w) x = __builtin_amdgcn_mfma_f32_16x16x4f32(a[w], z[w], x, 0, 0, 0);
            }
          }
          s[r][u] = x;
        }
      if (next < to) load_keys(t_next);
      // whole block visible to every row of the tile?
      const bool whole = t0 + BLK - 1 <= p0 && (P.window <= 0 || t0 > p1 - 1 - P.window || t0 + BLK <= P.sinks);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float top = -INFINITY;
#pragma unroll
        for (int u = 0; u < (BF ? 2 : 1); ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float x = s[r][u][e] * P.scale2;
            if (!whole) {
              const int tok = vt0 + 4 * u + e;
              const bool seen = tok <= pos[r] && (P.window <= 0 || tok > pos[r] - P.window || tok < P.sinks);
              x = seen ? x : -INFINITY;
            }
            s[r][u][e] = x;
            top = fmaxf(top, x);
          }
        if (__any(top > m[r] + 8.0f)) {
          top = fmaxf(top, __shfl_xor(top, 16));
          top = fmaxf(top, __shfl_xor(top, 32));
          const float to_m = fmaxf(m[r], top);
          const float f = to_m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m[r] - to_m);
          m[r] = to_m;
          l[r] *= f;
#pragma unroll
          for (int t = 0; t < NT; ++t) acc[r][t] *= f;
        }
        const float ref = m[r] == -INFINITY ? 0.0f : m[r];
#pragma unroll
        for (int u = 0; u < (BF ? 2 : 1); ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float x = __builtin_amdgcn_exp2f(s[r][u][e] - ref);
            s[r][u][e] = x;
            l[r] += x;
          }
      }
      // a value that is not finite would reach rows that do not see its token (0 times
      // infinity): such blocks are multiplied in three parts
      bool odd = false;
      if (!whole) {
        bool mine = false;
#pragma unroll
        for (int e = 0; e < TOK; ++e)
#pragma unroll
          for (int w = 0; w < VW; ++w) {
            mine |= (vr[e][w] & 0x7f800000u) == 0x7f800000u;
            if constexpr (BF) mine |= (vr[e][w] & 0x7f80u) == 0x7f80u;
          }
        odd = __any(mine);
      }
      bf16x8 pf[R];
      if constexpr (BF)
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int e = 0; e < 8; ++e) pf[r][e] = static_cast<__bf16>(s[r][e >> 2][e & 3]);
      // O += V^T P^T with tile t of the values, or with `f` of each of its elements
      auto multiply = [&](int t, auto f, f32x4(&to_add)[R]) {
        if constexpr (BF) {
          uint4 a;  // element t of the lane's eight value rows
          uint32_t w[4];
#pragma unroll
          for (int e = 0; e < 4; ++e)
            w[e] = f(__builtin_amdgcn_perm(vr[2 * e + 1][t >> 1], vr[2 * e][t >> 1], t & 1 ? 0x07060302u : 0x05040100u));
          __builtin_memcpy(&a, w, 16);
#pragma unroll
          for (int r = 0; r < R; ++r)
            to_add[r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), pf[r], to_add[r], 0, 0, 0);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float a = __uint_as_float(f(vr[e][t]));
#pragma unroll
            for (int r = 0; r < R; ++r) to_add[r] = __builtin_amdgcn_mfma_f32_16x16x4f32(a, s[r][0][e], to_add[r], 0, 0, 0);
          }
        }
      };
      if (!odd) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          f32x4 x[R];
#pragma unroll
          for (int r = 0; r < R; ++r) x[r] = acc[r][t];
          multiply(t, [](uint32_t v) { return v; }, x);
#pragma unroll
          for (int r = 0; r < R; ++r) acc[r][t] = x[r];
        }
      } else {
        // the finite values as they are; then how much weight lies on values of
        // +infinity or NaN, and of -infinity or NaN
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          f32x4 x[R], up[R], down[R];
#pragma unroll
          for (int r = 0; r < R; ++r) {
            x[r] = acc[r][t];
            up[r] = down[r] = f32x4{0, 0, 0, 0};
          }
          multiply(t, [](uint32_t v) { return kv_select<T, 0>(v); }, x);
          multiply(t, [](uint32_t v) { return kv_select<T, 1>(v); }, up);
          multiply(t, [](uint32_t v) { return kv_select<T, -1>(v); }, down);
#pragma unroll
          for (int r = 0; r < R; ++r)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              acc[r][t][e] = x[r][e] + (up[r][e] > 0.0f ? INFINITY : 0.0f) - (down[r][e] > 0.0f ? INFINITY : 0.0f);
        }
      }
      if (next < to) load_values(t_next);
      i = next;
    }
  }

  // the four waves' sums
  bad = __any(bad);
#pragma unroll
  for (int r = 0; r < R; ++r) {
    l[r] += __shfl_xor(l[r], 16);
    l[r] += __shfl_xor(l[r], 32);
    if (bad) l[r] = __builtin_nanf("");
    if (g == 0) {
      join_m[wave][16 * r + c] = m[r];
      join_l[wave][16 * r + c] = l[r];
    }
  }
  const bool split = it.splits > 1;
  const int jr = tid >> 4, jc = tid & 15;  // this thread's row of 16 and its NT elements
#pragma unroll
  for (int r = 0; r < R; ++r) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int t = 0; t < NT; t += 4)
        *reinterpret_cast<f32x4*>(&join_o[wave][c][(g * 4 + i) * NT + t]) =
            f32x4{acc[r][t][i], acc[r][t + 1][i], acc[r][t + 2][i], acc[r][t + 3][i]};
    __syncthreads();
    const int row = 16 * r + jr;
    if (row >= n_rows) continue;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < KV_ATT_WAVES; ++w) top = fmaxf(top, join_m[w][row]);
    const float ref = top == -INFINITY ? 0.0f : top;
    float sum = 0.0f, o[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) o[t] = 0.0f;
#pragma unroll
    for (int w = 0; w < KV_ATT_WAVES; ++w) {
      const float f = __builtin_amdgcn_exp2f(join_m[w][row] - ref);
      sum += f * join_l[w][row];
#pragma unroll
      for (int t = 0; t < NT; ++t) o[t] += f * join_o[w][jr][jc * NT + t];
    }
    if (split) {
      if (it.slot >= 0 && it.slot < P.slots) {
        float* dst = P.part + (static_cast<int64_t>(it.slot) * ROWS + row) * DP + jc * NT;
#pragma unroll
        for (int t = 0; t < NT; t += 4) *reinterpret_cast<f32x4*>(dst + t) = f32x4{o[t], o[t + 1], o[t + 2], o[t + 3]};
        if (jc == 0) {
          float* ml = P.part_ml + (static_cast<int64_t>(it.slot) * ROWS + row) * 2;
          ml[0] = top;
          ml[1] = sum;
        }
      }
    } else {
      const int rr = row0 + row, j = rr / G, head = it.head * G + rr - j * G;
      const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
      T* dst = reinterpret_cast<T*>(P.out.data + (it.first + j) * P.out.token + head * P.out.head);
#pragma unroll
      for (int t = 0; t < NT; ++t)
        if (jc * NT + t < D) kv_put(dst + jc * NT + t, o[t] * inv);
      if (P.lse && jc == 0)
        P.lse[static_cast<int64_t>(it.first + j) * P.n_q_heads + head] = (ref + log2f(sum)) * KV_LN2;
    }
  }
}

// Joins the partial sums of the split units, of which there are fewer than P.items
// (each has more blocks than an item takes).  A workgroup takes JR rows of a unit; 16
// threads hold a row's elements, and the splits are dealt to the 16 / JR groups of them.
template <typename T, int DP, int R, int JR>
__global__ __launch_bounds__(KV_ATT_NT) void kv_join_kernel(KvAttnParams P) {
  constexpr int ROWS = 16 * R, NT = DP / 16, PER = ROWS / JR, GROUPS = 16 / JR;
  __shared__ float sum_o[KV_ATT_NT][NT + 1];
  __shared__ float sum_m[16], sum_l[16];
  if (blockIdx.x / PER >= *P.split_units) return;
  KvItem it;
  if (!kv_find_item<ROWS, KvBlk<T>::N, true>(P, blockIdx.x / PER, &it)) return;
  const int tid = threadIdx.x, jc = tid & 15, jr = (tid >> 4) % JR, grp = (tid >> 4) / JR;
  const int D = P.p.dim, G = P.group;
  const int row0 = it.tile * ROWS, rows = it.count * G;
  const int row = static_cast<int>(blockIdx.x % PER) * JR + jr;
  const bool real = row0 + row < rows && it.slot >= 0 && it.slot + it.splits <= P.slots;
  float m = -INFINITY, l = 0.0f, o[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) o[t] = 0.0f;
  if (real) {
    const float* ml = P.part_ml + (static_cast<int64_t>(it.slot) * ROWS + row) * 2;
    const float* po = P.part + (static_cast<int64_t>(it.slot) * ROWS + row) * DP + jc * NT;
    for (int s = grp; s < it.splits; s += GROUPS) m = fmaxf(m, ml[static_cast<int64_t>(s) * ROWS * 2]);
    const float ref = m == -INFINITY ? 0.0f : m;
#pragma unroll 4
    for (int s = grp; s < it.splits; s += GROUPS) {
      const float f = __builtin_amdgcn_exp2f(ml[static_cast<int64_t>(s) * ROWS * 2] - ref);
      l += f * ml[static_cast<int64_t>(s) * ROWS * 2 + 1];
      const float* x = po + static_cast<int64_t>(s) * ROWS * DP;
#pragma unroll
      for (int t = 0; t < NT; t += 4) {
        const f32x4 y = *reinterpret_cast<const f32x4*>(x + t);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[t + e] += f * y[e];
      }
    }
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) sum_o[tid][t] = o[t];
  if (jc == 0) {
    sum_m[tid >> 4] = m;
    sum_l[tid >> 4] = l;
  }
  __syncthreads();
  if (grp != 0 || !real) return;
  float top = -INFINITY;
#pragma unroll
  for (int w = 0; w < GROUPS; ++w) top = fmaxf(top, sum_m[w * JR + jr]);
  const float ref = top == -INFINITY ? 0.0f : top;
  float sum = 0.0f;
#pragma unroll
  for (int t = 0; t < NT; ++t) o[t] = 0.0f;
#pragma unroll
  for (int w = 0; w < GROUPS; ++w) {
    const float f = __builtin_amdgcn_exp2f(sum_m[w * JR + jr] - ref);
    sum += f * sum_l[w * JR + jr];
#pragma unroll
    for (int t = 0; t < NT; ++t) o[t] += f * sum_o[(w * JR + jr) * 16 + jc][t];
  }
  const int rr = row0 + row, j = rr / G, head = it.head * G + rr - j * G;
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  T* dst = reinterpret_cast<T*>(P.out.data + (it.first + j) * P.out.token + head * P.out.head);
#pragma unroll
  for (int t = 0; t < NT; ++t)
    if (jc * NT + t < D) kv_put(dst + jc * NT + t, o[t] * inv);
  if (P.lse && jc == 0)
    P.lse[static_cast<int64_t>(it.first + j) * P.n_q_heads + head] = (ref + log2f(sum)) * KV_LN2;
}

// Most tiles of 16 rows that a workgroup takes: what the registers of its waves hold
// (O and Q of each row tile beside a block's keys and values).
template <typename T>
constexpr int kv_row_tiles(int dp) {
  return sizeof(T) == 2 ? (dp <= 64 ? 4 : dp <= 128 ? 2 : 1) : (dp <= 128 ? 2 : 1);
}

// Launches for heads of up to DP elements, `row_tiles` of 16 rows a workgroup; `units`
// bounds the units of the call.
template <typename T, int DP>
hipError_t launch_kv_attention(const KvAttnParams& P, int row_tiles, int64_t units, bool join, hipStream_t st);

}  // namespace saki
