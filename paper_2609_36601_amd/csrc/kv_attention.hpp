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

#include <stddef.h>

#include <type_traits>

#include "kv_append.hpp"

namespace saki {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int KV_ATT_NT = 256;
constexpr int KV_ATT_WAVES = KV_ATT_NT / KV_WAVE;
constexpr int KV_ATT_ROWS = 64;  // most rows of a tile of kv_attention_kernel
constexpr float KV_LOG2E = 1.44269504088896340736f;
constexpr float KV_LN2 = 0.693147180559945309417f;

constexpr int KV_PROMPT_ROWS = 128;

// Workgroups of kv_attention_kernel that a CU takes (one wave of each on every SIMD), by the
// registers of a wave: O and Q of its R row tiles, a block's keys and values.  More waves that
// spill are slower: 512 drafts x 4,480 keys at three a CU with 68 bytes spilled 1,672 us,
// at two without 1,527.
template <typename T>
constexpr int kv_groups_per_cu(int dp, int r) {
  const int q = r > 1 ? 0 : sizeof(T) == 2 ? dp / 8 : dp / 4;  // (in LDS for more than one row tile)
  const int regs = dp / 4 * r + q + dp / 2 + (sizeof(T) == 2 ? 16 : 32) * (r - 1);
  return regs <= 64 ? 4 : regs <= 80 ? 3 : regs <= 160 ? 2 : 1;
}

// Items that a call with fewer units is split into: what the card takes at once.  More, so that
// the last ones to end are short, gives the join more to do than it saves (128 verifications of
// 1,800 to 7,200 keys 475 -> 487 us with four times as many, of 4,100 keys each 391 -> 431).
constexpr int KV_CUS = 256;
template <typename T, int DP, int ROWS>
constexpr int KV_ITEMS = KV_CUS * (ROWS == KV_PROMPT_ROWS ? 2 : kv_groups_per_cu<T>(DP, ROWS / 16));

struct KvItem;

struct KvAttnParams {
  KvTable t;
  KvPool p;  // bases of the layer
  KvTokens n;
  KvStrides q, out;
  float* lse;
  int n_q_heads, group;
  float scale2;  // |scale| log2 e
  uint32_t flip;  // sign bits of a pair of elements (one, in f32) where the scale is negative
  int zero;       // the scale is 0 (scale2 is 1 then)
  int window, sinks;
  float* part;     // [slots][rows][DP] partial sums, then
  float* part_ml;  // [slots][rows][2] their maximum and sum
  int slots;
  float share;     // blocks an item takes, of each block of the sequences' tiles
  float per_tile;  // 1 / tiles of the sequences
  int span;        // tokens that a tile's rows span at most
  int* n_split;           // how many units are split, and which: for kv_join_kernel
  KvItem* split;   // [items]
};

// Blocks of BLK tokens that the rows of tokens [j0, j1) (positions p0 .. p1 - 1) see:
// the first `sinks` blocks, then those from token `lo` on.
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
  int start;         // position of the first
  int tiles;
  int blocks;
  bool fine;
};
template <int ROWS, int BLK>
__device__ __forceinline__ KvLoad kv_load_of(const KvAttnParams& P, int b) {
  KvLoad s;
  kv_rows(P.n, b, &s.first, &s.count);
  const int L = P.t.length[b], held = kv_held(P.t, b);
  // (the host has seen to it that all rows together are fewer than 2^31)
  s.tiles = (s.count * P.group + ROWS - 1) / ROWS;
  const int64_t end = static_cast<int64_t>(L) + P.n.shift + s.count;
  s.fine = L >= 0 && end <= (static_cast<int64_t>(held) << P.t.shift);
  s.start = L + P.n.shift;
  s.blocks = 1;
  if (s.fine && s.count > 0) {
    s.blocks = (static_cast<int>(end) + BLK - 1) / BLK;
    if (P.window > 0) {
      // the widest tile: P.span tokens at most, which may begin anywhere in a block (and no tile
      // has more blocks than the sequence: where those are few, the host leaves out the join)
      const int span = s.count < P.span ? s.count : P.span;
      s.blocks = min(s.blocks, kv_span<BLK>(end - span, end, P.window, P.sinks).blocks + (span < s.count ? 1 : 0));
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

// The same item for the whole workgroup, in scalar registers.
__device__ __forceinline__ KvItem kv_uniform(const KvItem& x) {
  KvItem r;
#define KV_FIELD(f) r.f = __builtin_amdgcn_readfirstlane(x.f)
  KV_FIELD(b), KV_FIELD(first), KV_FIELD(count), KV_FIELD(start), KV_FIELD(tile), KV_FIELD(head), KV_FIELD(split),
      KV_FIELD(splits), KV_FIELD(slot), KV_FIELD(fine);
#undef KV_FIELD
  return r;
}

// The blocks of a split: whole blocks, spread evenly.
__device__ __forceinline__ int kv_split_at(int blocks, int splits, int split) {
  const int q = blocks / splits, r = blocks - q * splits;
  return q * split + (split < r ? split : r);
}

// Finds the workgroup's item; every workgroup derives the split from the lengths by
// itself, which spares a launch.  The sequences whose tiles are longer than the mean come
// first, so that the last workgroups to start are short.  Items of a sequence are ordered by
// tile (last first: with causal rows those are the longest), split, key head, so that the
// workgroups of one key head, which read the same keys, tend to one XCD.  False: there is
// no such item.  Every workgroup pays for this before it begins: sums in 32 bits, no divisions but
// in the one thread that holds the item (4.1 us with 64-bit sums and divisions in every thread, 2.9
// without, 16 sequences).
template <int ROWS, int BLK, int ITEMS>
__device__ __forceinline__ bool kv_find_item(const KvAttnParams& P, KvItem* out) {
  __shared__ int part_blocks[KV_ATT_WAVES];
  __shared__ int4 part[KV_ATT_WAVES];
  __shared__ KvItem found;
  __shared__ int is_found;
  const int tid = threadIdx.x, wave = tid / KV_WAVE;
  const bool last_lane = (tid & (KV_WAVE - 1)) == KV_WAVE - 1;
  const int Hk = P.p.n_heads;
  const int per = (P.t.n_seq + KV_ATT_NT - 1) / KV_ATT_NT;
  const int b0 = tid * per, b1 = b0 + per < P.t.n_seq ? b0 + per : P.t.n_seq;
  if (tid == 0) is_found = 0;
  // all blocks; 2^22 a thread stands for more than can be counted (then nothing is split)
  long long blocks = 0;
  KvLoad keep;  // the thread's only sequence where it has one
  for (int b = b0; b < b1; ++b) {
    keep = kv_load_of<ROWS, BLK>(P, b);
    blocks += static_cast<long long>(keep.tiles) * keep.blocks;
  }
  const int sum = kv_wave_scan(static_cast<int>(blocks < (1 << 22) ? blocks : 1 << 22));
  if (last_lane) part_blocks[wave] = sum;
  __syncthreads();
  int all = 0;
  bool many = false;
#pragma unroll
  for (int w = 0; w < KV_ATT_WAVES; ++w) {
    all += part_blocks[w];
    many |= part_blocks[w] >= 1 << 22;
  }
  // blocks an item takes: its share (rounded up, and at least 8)
  int len = static_cast<int>(static_cast<float>(all) * P.share) + 1;
  len = many ? 1 << 30 : len < 8 ? 8 : len;
  const int mean = static_cast<int>(static_cast<float>(all) * P.per_tile);
  const float inv = 1.0f / static_cast<float>(len);
  auto splits_of = [&](const KvLoad& s) {
    int n = static_cast<int>(static_cast<float>(s.blocks) * inv);  // exact but for one
    n = n < 1 ? 1 : n;
    n += n * len < s.blocks;
    return n - ((n - 1) * len >= s.blocks);
  };
  // Sums over the sequences: items of long ones and of the others; slots of the split units'
  // items, fewer than twice the items aimed at, and (upper half) split units, fewer than
  // those (each has more blocks than an item).
  auto add = [&](const KvLoad& s, int4* x) {
    const int n = splits_of(s), units = s.tiles * Hk;
    (s.blocks > mean ? x->x : x->y) += units * n;
    x->z += n > 1 ? units * (n + (1 << 16)) : 0;
  };
  int4 mine{0, 0, 0, 0};
  for (int b = b0; b < b1; ++b) {
    if (per > 1) keep = kv_load_of<ROWS, BLK>(P, b);
    add(keep, &mine);
  }
  int4 at{kv_wave_scan(mine.x), kv_wave_scan(mine.y), kv_wave_scan(mine.z), 0};
  if (last_lane) part[wave] = at;
  at.x -= mine.x, at.y -= mine.y, at.z -= mine.z;
  __syncthreads();
  int4 total{0, 0, 0, 0};
#pragma unroll
  for (int w = 0; w < KV_ATT_WAVES; ++w) {
    const int4 p = part[w];
    if (w < wave) at.x += p.x, at.y += p.y, at.z += p.z;
    total.x += p.x, total.z += p.z;
  }
  at.y += total.x;
  const int item = static_cast<int>(blockIdx.x);
  // (the bound only matters for token ranges that overlap, whose sums may pass their fields)
  if (item == 0 && tid == 0) *P.n_split = min(total.z >> 16 & 0xffff, ITEMS);
  if ((item >= at.x && item < at.x + mine.x) || (item >= at.y && item < at.y + mine.y)) {
    for (int b = b0; b < b1; ++b) {
      if (per > 1) keep = kv_load_of<ROWS, BLK>(P, b);
      const int n = splits_of(keep), i = item - (keep.blocks > mean ? at.x : at.y);
      if (i >= 0 && i < keep.tiles * Hk * n) {
        KvItem f;
        const int q = i / Hk;
        f.head = i - q * Hk;
        const int back = n == 1 ? q : q / n;
        f.split = q - back * n;
        f.tile = keep.tiles - 1 - back;
        f.first = keep.first;
        f.count = keep.count;
        f.start = keep.start;
        f.fine = keep.fine;
        f.splits = n;
        f.b = b;
        // a unit's slots are consecutive
        f.slot = (at.z & 0xffff) + (back * Hk + f.head) * n + f.split;
        found = f;
        is_found = 1;
        const int unit = (at.z >> 16 & 0xffff) + back * Hk + f.head;
        if (n > 1 && f.split == 0 && unit < ITEMS) P.split[unit] = f;
        break;
      }
      add(keep, &at);
    }
  }
  __syncthreads();
  *out = kv_uniform(found);
  return __builtin_amdgcn_readfirstlane(is_found) != 0;
}

// Token and query head of a tile's rows.  Row r of the tile is row rem + r of those from token j0 on; below
// 2^21 the quotient by the group is exact as a product with its reciprocal (a half is added: the
// quotient is then at least 1 / 2 group from a whole number).
struct KvRowMap {
  int j0, rem, group;
  float inv;
  __device__ __forceinline__ KvRowMap(int row0, int group) : group(group), inv(1.0f / static_cast<float>(group)) {
    j0 = row0 / group;
    rem = row0 - j0 * group;
  }
  __device__ __forceinline__ int token(int r) const {
    return j0 + static_cast<int>((static_cast<float>(rem + r) + 0.5f) * inv);
  }
  __device__ __forceinline__ int member(int r, int j) const { return rem + r - (j - j0) * group; }
};

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

template <int SIGN>
__device__ __forceinline__ uint4 kv_part(uint4 v) {
  return uint4{kv_select<uint16_t, SIGN>(v.x), kv_select<uint16_t, SIGN>(v.y), kv_select<uint16_t, SIGN>(v.z),
               kv_select<uint16_t, SIGN>(v.w)};
}

// Largest magnitudes so far of pairs of bf16 values, as unsigned numbers: those that are not finite are
// the largest ones, and a block's are looked through two instructions a word.
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t kv_largest(uint32_t top, uint32_t v) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, top),
                                                                __builtin_bit_cast(u16x2, v & 0x7fff7fffu)));
}
__device__ __forceinline__ bool kv_not_finite(uint32_t top) { return top >= 0x7f800000u || (top & 0xffffu) >= 0x7f80u; }

__device__ __forceinline__ uint4 kv_flip(uint4 x, uint32_t f) { return uint4{x.x ^ f, x.y ^ f, x.z ^ f, x.w ^ f}; }

// A query's elements where the scale is 0: they are, too, and scale2 is 1, so that scores are 0 from products of any size
// and a hidden one stays -infinity.  (NaN for those that are not finite: 0 times them is.)  Behind one branch
// for all of a lane's: a branch for each took the window in f32 from 82 us to 85, 512 drafts from 1,554 to 1,566.
template <typename T>
__device__ __forceinline__ uint4 kv_zero_query(uint4 x) {
  auto word = [](uint32_t v) {
    const uint32_t ones = kv_select<T, 1>(v) | kv_select<T, -1>(v);
    return ones | ones << 1 | ones >> 1;  // 0x3f80 -> 0x7fc0
  };
  return uint4{word(x.x), word(x.y), word(x.z), word(x.w)};
}

// Hides the scores (a lane's 4 U of a block, of tokens tok + 4 u + e) that the row at `pos` does not see.
template <int U>
__device__ __forceinline__ void kv_mask(f32x4 (&s)[U], int tok, int pos, int window, int sinks) {
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int e = 0; e < 4; ++e) s[u][e] = tok + 4 * u + e <= pos ? s[u][e] : -INFINITY;
  if (window > 0)
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int t = tok + 4 * u + e;
        s[u][e] = t > pos - window || t < sinks ? s[u][e] : -INFINITY;
      }
}

// Scores of a row to weights relative to the running maximum m, with l their sum; where the
// maximum moves, O and l are scaled.  scale2 > 0.
template <int U, int NT>
__device__ __forceinline__ void kv_soften(f32x4 (&s)[U], f32x4 (&acc)[NT], float* m, float* l, float scale2) {
  float top = -INFINITY;
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int e = 0; e < 4; ++e) top = fmaxf(top, s[u][e]);
  if (__any(top * scale2 > *m + 8.0f)) {
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    const float to = fmaxf(*m, top * scale2);
    const float f = to == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(*m - to);
    *m = to;
    *l *= f;
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[t] *= f;
  }
  const float ref = *m == -INFINITY ? 0.0f : *m;
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][e], scale2, -ref));
      s[u][e] = x;
      *l += x;
    }
}

// A lane's eight weights (>= 0, or NaN) as sums of two bf16 numbers: the largest bf16 number below a weight, and the rest,
// which is rounded, 2^-17 of the weight at most.  Both parts of a weight that is not 0 are above 0, so that their products
// with an infinite value are that infinity, and not the NaN of 0 or of opposite signs.
__device__ __forceinline__ void kv_halves(const f32x4 (&s)[2], bf16x8* high, bf16x8* low) {
  uint32_t h[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t x = __float_as_uint(s[e >> 2][e & 3]);
    h[e] = (x > 1u ? x : 1u) - 1u;
    (*low)[e] = static_cast<__bf16>(s[e >> 2][e & 3] - __uint_as_float(h[e] & 0xffff0000u));
  }
  uint32_t w[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = __builtin_amdgcn_perm(h[2 * e + 1], h[2 * e], 0x07060302u);
  *high = __builtin_bit_cast(bf16x8, uint4{w[0], w[1], w[2], w[3]});
}

// N elements o[i] / sum of a row, of which those below `left` are there (a multiple of 8); 0 for a row without
// any weight (o may still not be finite: 0 times a value that is not).
template <typename T, int N>
__device__ __forceinline__ void kv_put_row(T* dst, const float (&o)[N], float sum, int left) {
  const bool none = sum == 0.0f;
  const float f = 1.0f / sum;
#pragma unroll
  for (int t = 0; t < N; t += 4)
    if (t < left) {
      T y[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) kv_put(&y[e], none ? 0.0f : o[t + e] * f);
      __builtin_memcpy(__builtin_assume_aligned(dst + t, 4 * sizeof(T)), y, sizeof(y));
    }
}

// One item: ROWS = 16 R rows, the blocks of its split dealt to the four waves, each of which has a
// running maximum and sum of its own until the end: no barrier between blocks, and every wave's
// loads, a block ahead, go from memory straight to the registers that the products read.
// What bounds it: reading the keys and values (512 drafts over 4,480 keys, 8 + 8 heads of 128 bf16
// elements: 1,560 us, 6.0 TB/s, what a large read reaches; 128 verifications of 8 tokens by 4 query
// heads a key head, R = 2: 444 us, 5.3); for one long sequence that and the join's launch behind
// it (131,072 keys: 44 and 7 us); for few short ones the way to the first product (16 drafts 16 us,
// of which the keys' bytes take 14 only if all are under way at once); in f32 the matrix products, at
// a sixteenth of bf16's rate, and the blocks at both ends of a row's window (ragged tokens behind a
// window of 500: 82 us, 38 TFLOP/s over what the rows see).
template <typename T, int DP, int R>
__global__ __launch_bounds__(KV_ATT_NT, kv_groups_per_cu<T>(DP, R)) void kv_attention_kernel(KvAttnParams P) {
  constexpr bool BF = sizeof(T) == 2;
  constexpr int BLK = KvBlk<T>::N;
  constexpr int ROWS = 16 * R;
  constexpr int NT = DP / 16;              // 16-wide tiles of the head: a lane's elements of a value row
  constexpr int QC = BF ? DP / 32 : DP / 16;  // 16-byte pieces of a lane's share of a key row
  constexpr int TOK = BF ? 8 : 4;          // tokens of a lane in a block
  // Weights as two bf16 numbers: their second products are free where memory bounds the kernel (16 rows: 0 to 1%, 32 rows
  // 0 to 3%), not with four row tiles (64 rows of 64-element heads 53 -> 60 us).
  constexpr bool HALVES = BF && R <= 2;
  constexpr int VW = NT * sizeof(T) / 4;   // 32-bit words of a lane's share of a value row
  using VPiece = typename std::conditional<(VW >= 4), uint4, uint2>::type;
  constexpr int VC = VW * 4 / sizeof(VPiece), VE = sizeof(VPiece) / sizeof(T);  // its loads, elements of a load
  __shared__ __align__(16) float join_o[KV_ATT_WAVES][16][DP + 4];
  __shared__ float join_m[KV_ATT_WAVES][ROWS], join_l[KV_ATT_WAVES][ROWS];

  KvItem it;
  if (!kv_find_item<ROWS, BLK, KV_ITEMS<T, DP, ROWS>>(P, &it)) return;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / KV_WAVE), lane = tid & (KV_WAVE - 1);
  const int c = lane & 15, g = lane >> 4;
  const int D = P.p.dim, G = P.group;
  const int row0 = it.tile * ROWS, rows = it.count * G;
  const int n_rows = rows - row0 < ROWS ? rows - row0 : ROWS;
  const KvRowMap map(row0, G);
  const int p0 = it.start + map.j0, p1 = it.start + map.token(n_rows - 1) + 1;  // positions of the tile's tokens
  bool bad = !it.fine;

  // this lane's rows; their queries stay in registers for one row tile, else in LDS, where every wave
  // reads them again for each block
  constexpr bool Q_LDS = R > 1;
  __shared__ uint4 q_lds[Q_LDS ? R * QC : 1][KV_WAVE];
  int pos[R];
  uint4 qf[Q_LDS ? 1 : R][QC];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int row = 16 * r + c;
    const bool real = row < n_rows;
    const int in = real ? row : n_rows - 1, j = map.token(in), head = it.head * G + map.member(in, j);
    pos[r] = it.start + j;
    const char* src = P.q.data + (it.first + j) * P.q.token + head * P.q.head;
#pragma unroll
    for (int i = 0; i < QC; ++i) {
      const int d = i * (BF ? 32 : 16) + g * (BF ? 8 : 4);
      const uint4 x = kv_flip(d < D ? *reinterpret_cast<const uint4*>(src + d * sizeof(T)) : uint4{0, 0, 0, 0}, P.flip);
      if constexpr (Q_LDS) {
        if ((r * QC + i) % KV_ATT_WAVES == wave) q_lds[r * QC + i][lane] = x;
      } else {
        qf[r][i] = x;
      }
    }
  }
  if constexpr (Q_LDS) {
    if (P.zero)
#pragma unroll
      for (int i = 0; i < R * QC; ++i)
        if (i % KV_ATT_WAVES == wave) q_lds[i][lane] = kv_zero_query<T>(q_lds[i][lane]);
    __syncthreads();
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
    const int from = kv_split_at(span.blocks, it.splits, it.split), to = kv_split_at(span.blocks, it.splits, it.split + 1);
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
    // (page ids are looked up two blocks ahead: loads return in order, and an id behind the values of
    // the block before would have the keys wait for those)
    int k_id = 0, v_id = 0, k_next = 0, v_next = 0;
    auto load_ids = [&](int t0) {
      k_next = row_pages[run_of(t0 + k_in) >> P.t.shift];
      v_next = row_pages[run_of(t0 + v_in) >> P.t.shift];
    };
    auto page_at = [&](int id) {
      const bool in = id >= 0 && id < P.t.n_pages;
      bad |= !in;
      return static_cast<int64_t>(in ? id : 0) * P.p.page_stride;
    };
    uint4 kf[BF ? 2 : 1][QC];
    uint32_t vr[TOK][VW];
    const uint32_t token_stride = static_cast<uint32_t>(P.p.token_stride);  // (a page's tokens lie within 2^31 bytes)
    auto load_keys = [&](int t0) {
      const int run = run_of(t0 + k_in);
      const char* src = kb + page_at(k_id) + (g * 16);
#pragma unroll
      for (int s = 0; s < (BF ? 2 : 1); ++s) {
        int tok = BF ? run + (c & 3) + 4 * s : run + (c & 7);
        tok = tok < last ? tok : last;
        const char* at = src + static_cast<uint32_t>(tok & mask) * token_stride;
        if (D == DP) {
#pragma unroll
          for (int e = 0; e < QC; ++e) kf[s][e] = *reinterpret_cast<const uint4*>(at + e * 64);
        } else {
#pragma unroll
          for (int e = 0; e < QC; ++e)
            kf[s][e] = e * 64 + g * 16 < D * static_cast<int>(sizeof(T)) ? *reinterpret_cast<const uint4*>(at + e * 64)
                                                                         : uint4{0, 0, 0, 0};
        }
      }
    };
    auto load_values = [&](int t0) {
      const int run = run_of(t0 + v_in);
      const char* src = vb + page_at(v_id);
#pragma unroll
      for (int e = 0; e < TOK; ++e) {
        int tok = run + (BF ? 0 : v_in & 7) + e;
        tok = tok < last ? tok : last;
        const char* at = src + static_cast<uint32_t>(tok & mask) * token_stride;
#pragma unroll
        for (int w = 0; w < VC; ++w) {
          // (elements from D on make rows of O that are not kept: any values will do)
          const int d = c * NT + w * VE < D ? c * NT + w * VE : 0;
          const VPiece x = *reinterpret_cast<const VPiece*>(at + d * sizeof(T));
          __builtin_memcpy(&vr[e][w * sizeof(VPiece) / 4], &x, sizeof(x));
        }
      }
    };
    // The next block's keys are loaded once this block's are multiplied, and its values
    // once this block's are: both are under way while the rest of a block is computed.
    int i = from + wave;
    if (i < to) {
      load_ids(token_of(i));
      k_id = k_next;
      v_id = v_next;
      load_keys(token_of(i));
      if (i + KV_ATT_WAVES < to) load_ids(token_of(i + KV_ATT_WAVES));
      load_values(token_of(i));
    }
    if constexpr (!Q_LDS)
      if (P.zero)  // (here, where the first keys are under way)
#pragma unroll
        for (int e = 0; e < QC; ++e) qf[0][e] = kv_zero_query<T>(qf[0][e]);
    while (i < to) {
      const int t0 = token_of(i), vt0 = t0 + v_in;
      const int next = i + KV_ATT_WAVES;
      const int t_next = token_of(next);
      // scores
      f32x4 s[R][BF ? 2 : 1];
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int u = 0; u < (BF ? 2 : 1); ++u) {
          f32x4 x{0, 0, 0, 0};
#pragma unroll
          for (int e = 0; e < QC; ++e) {
            // (four products of 32 cycles each; in bf16 one of 16.  The branches also keep the loads of Q from
            // LDS apart, all of which at once would not fit the registers)
            if (!BF && DP <= 128 && e * 16 >= D) break;
            const uint4 q = Q_LDS ? q_lds[Q_LDS ? r * QC + e : 0][lane] : qf[Q_LDS ? 0 : r][e];
            if constexpr (BF) {
              x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf[u][e]),
                                                          __builtin_bit_cast(bf16x8, q), x, 0, 0, 0);
            } else {
              const f32x4 a = __builtin_bit_cast(f32x4, kf[u][e]), z = __builtin_bit_cast(f32x4, q);
#pragma unroll
              for (int w = 0; w < 4; ++w) x = __builtin_amdgcn_mfma_f32_16x16x4f32(a[w], z[w], x, 0, 0, 0);
            }
          }
          s[r][u] = x;
        }
      if (next < to) {
        k_id = k_next;
        v_id = v_next;
        load_keys(t_next);
        if (next + KV_ATT_WAVES < to) load_ids(token_of(next + KV_ATT_WAVES));
      }
      // whole block visible to every row of the tile?
      const bool whole = t0 + BLK - 1 <= p0 && (P.window <= 0 || t0 > p1 - 1 - P.window || t0 + BLK <= P.sinks);
      if (!whole)
#pragma unroll
        for (int r = 0; r < R; ++r) kv_mask(s[r], vt0, pos[r], P.window, P.sinks);
#pragma unroll
      for (int r = 0; r < R; ++r)
        kv_soften(s[r], acc[r], &m[r], &l[r], P.scale2);
      // A value that is not finite would reach rows that do not see its token (0 times infinity):
      // in blocks where that can be, such values are taken out, and how much weight lies on
      // +infinity or NaN, and on -infinity or NaN, is multiplied by itself.
      bool odd = false;
      constexpr int PER_WORD = 4 / sizeof(T), MARKS = (TOK * VW * PER_WORD + 31) / 32;
      uint32_t up[MARKS], down[MARKS];
      if (!whole) {
        bool mine = false;
        uint32_t largest = 0;
#pragma unroll
        for (int e = 0; e < TOK; ++e)
#pragma unroll
          for (int w = 0; w < VW; ++w) {
            if constexpr (BF)
              largest = kv_largest(largest, vr[e][w]);
            else
              mine |= (vr[e][w] & 0x7f800000u) == 0x7f800000u;
          }
        odd = __any(mine || kv_not_finite(largest));
        if (odd) {
#pragma unroll
          for (int i = 0; i < MARKS; ++i) up[i] = down[i] = 0;
#pragma unroll
          for (int e = 0; e < TOK; ++e)
#pragma unroll
            for (int w = 0; w < VW; ++w) {
              const int at = (e * VW + w) * PER_WORD;
              const uint32_t u = kv_select<T, 1>(vr[e][w]), d = kv_select<T, -1>(vr[e][w]);
#pragma unroll
              for (int k = 0; k < PER_WORD; ++k) {
                up[(at + k) / 32] |= (u >> (16 * k) & 0xffffu || (PER_WORD == 1 && u) ? 1u : 0u) << (at + k) % 32;
                down[(at + k) / 32] |= (d >> (16 * k) & 0xffffu || (PER_WORD == 1 && d) ? 1u : 0u) << (at + k) % 32;
              }
              vr[e][w] = kv_select<T, 0>(vr[e][w]);
            }
        }
      }
      bf16x8 pf[R], pl[R];
      if constexpr (HALVES) {
#pragma unroll
        for (int r = 0; r < R; ++r) kv_halves(s[r], &pf[r], &pl[r]);
      } else if constexpr (BF) {
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int e = 0; e < 8; ++e) pf[r][e] = static_cast<__bf16>(s[r][e >> 2][e & 3]);
      }
      // x += V^T P^T, tile t of the values
      auto multiply = [&](int t, f32x4(&x)[R]) {
        if constexpr (BF) {
          uint32_t w[4];  // element t of the lane's eight value rows
#pragma unroll
          for (int e = 0; e < 4; ++e)
            w[e] = __builtin_amdgcn_perm(vr[2 * e + 1][t >> 1], vr[2 * e][t >> 1], t & 1 ? 0x07060302u : 0x05040100u);
          const bf16x8 a = __builtin_bit_cast(bf16x8, uint4{w[0], w[1], w[2], w[3]});
#pragma unroll
          for (int r = 0; r < R; ++r) x[r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, pf[r], x[r], 0, 0, 0);
          if constexpr (HALVES)
#pragma unroll
            for (int r = 0; r < R; ++r) x[r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, pl[r], x[r], 0, 0, 0);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int r = 0; r < R; ++r)
              x[r] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vr[e][t]), s[r][0][e], x[r], 0, 0, 0);
        }
      };
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        f32x4 x[R];
#pragma unroll
        for (int r = 0; r < R; ++r) x[r] = acc[r][t];
        multiply(t, x);
#pragma unroll
        for (int r = 0; r < R; ++r) acc[r][t] = x[r];
      }
      if (odd) {
        constexpr uint32_t ONE = BF ? 0x3f80u : 0x3f800000u;
#pragma unroll 1
        for (int sign = 0; sign < 2; ++sign) {
          const float inf = sign ? -INFINITY : INFINITY;
#pragma unroll
          for (int e = 0; e < TOK; ++e)
#pragma unroll
            for (int w = 0; w < VW; ++w) {
              const int at = (e * VW + w) * PER_WORD;
              const uint32_t bits = (sign ? down[at / 32] : up[at / 32]) >> at % 32;
              vr[e][w] = (bits & 1 ? ONE : 0u) | (PER_WORD == 2 && bits & 2 ? ONE << 16 : 0u);
            }
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            f32x4 x[R];
#pragma unroll
            for (int r = 0; r < R; ++r) x[r] = f32x4{0, 0, 0, 0};
            multiply(t, x);
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
              for (int e = 0; e < 4; ++e) acc[r][t][e] += x[r][e] > 0.0f ? inf : 0.0f;
          }
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
      const int j = map.token(row), head = it.head * G + map.member(row, j);
      T* dst = reinterpret_cast<T*>(P.out.data + (it.first + j) * P.out.token + head * P.out.head);
      kv_put_row(dst + jc * NT, o, sum, D - jc * NT);
      if (P.lse && jc == 0)
        P.lse[static_cast<int64_t>(it.first + j) * P.n_q_heads + head] = (ref + log2f(sum)) * KV_LN2;
    }
  }
}

// Joins the partial sums of the split units, of which there are no more than items aimed at
// (each has more blocks than an item takes).  A workgroup takes JR rows of a unit at a time;
// 16 threads hold a row's elements, and the splits are dealt to the 16 / JR groups of them.  What
// bounds it: latency.  A launch that finds nothing to join takes 4 us, 128 units of 16 drafts 8.
template <typename T, int DP, int ROWS, int JR>
__global__ __launch_bounds__(KV_ATT_NT) void kv_join_kernel(KvAttnParams P) {
  constexpr int NT = DP / 16, PER = ROWS / JR, GROUPS = 16 / JR;
  __shared__ float sum_o[KV_ATT_NT][NT + 1];
  __shared__ float sum_m[16], sum_l[16];
  const int tid = threadIdx.x, jc = tid & 15, jr = (tid >> 4) % JR, grp = (tid >> 4) / JR;
  const int D = P.p.dim, G = P.group;
  const int n = *P.n_split * PER;
  for (int work = blockIdx.x; work < n; work += gridDim.x) {
    const KvItem it = kv_uniform(P.split[work / PER]);
    const int row0 = it.tile * ROWS, rows = it.count * G;
    const KvRowMap map(row0, G);
    const int row = work % PER * JR + jr;
    // (token ranges that overlap, which are not allowed, can make more items than were launched, and entries that
    // none of them wrote: what does not fit is left out)
    const bool fits = it.slot >= 0 && it.splits > 0 && it.splits <= P.slots - it.slot && it.first >= 0 && it.count > 0 &&
                      it.count <= P.n.n_tokens - it.first && it.head >= 0 && it.head < P.p.n_heads && it.tile >= 0 &&
                      it.tile <= it.count * G / ROWS;
    const bool real = fits && row0 + row < rows;
    float m = -INFINITY, l = 0.0f, o[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) o[t] = 0.0f;
    if (real) {
      const float* ml = P.part_ml + (static_cast<int64_t>(it.slot) * ROWS + row) * 2;
      const float* po = P.part + (static_cast<int64_t>(it.slot) * ROWS + row) * DP + jc * NT;
      // one pass, four splits' loads at a time
      for (int s0 = grp; s0 < it.splits; s0 += 4 * GROUPS) {
        float sm[4], sl[4];
        f32x4 so[4][NT / 4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int64_t s = s0 + i * GROUPS < it.splits ? s0 + i * GROUPS : s0;
          sm[i] = s0 + i * GROUPS < it.splits ? ml[s * ROWS * 2] : -INFINITY;
          sl[i] = ml[s * ROWS * 2 + 1];
#pragma unroll
          for (int t = 0; t < NT / 4; ++t) so[i][t] = *reinterpret_cast<const f32x4*>(po + s * ROWS * DP + 4 * t);
        }
        const float to = fmaxf(fmaxf(fmaxf(sm[0], sm[1]), fmaxf(sm[2], sm[3])), m);
        const float ref = to == -INFINITY ? 0.0f : to;
        const float old = __builtin_amdgcn_exp2f(m - ref);
        m = to;
        l *= old;
#pragma unroll
        for (int t = 0; t < NT; ++t) o[t] *= old;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (s0 + i * GROUPS >= it.splits) break;
          const float f = __builtin_amdgcn_exp2f(sm[i] - ref);
          l += f * sl[i];
#pragma unroll
          for (int t = 0; t < NT; ++t) o[t] += f * so[i][t / 4][t % 4];
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
    if (grp == 0 && real) {
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
      const int j = map.token(row), head = it.head * G + map.member(row, j);
      T* dst = reinterpret_cast<T*>(P.out.data + (it.first + j) * P.out.token + head * P.out.head);
      kv_put_row(dst + jc * NT, o, sum, D - jc * NT);
      if (P.lse && jc == 0)
        P.lse[static_cast<int64_t>(it.first + j) * P.n_q_heads + head] = (ref + log2f(sum)) * KV_LN2;
    }
    __syncthreads();  // before the sums are written again
  }
}

// Prompts: many rows a sequence.  Each of the four waves takes 32 rows of the item's 128, and
// all of them the same keys and values, 64 tokens at a time, through LDS, into which the
// memory pipeline writes them without a detour through registers; the next 64 tokens are under
// way while these are multiplied (two buffers, one barrier).  A token's row lies there as
// in memory, but its 16-byte pieces are permuted: piece p of a row is at p ^ kv_swizzle(row), so
// that the 16 rows which a read touches lie in 16 different banks.  The values are transposed
// by the read (ds_read_b64_tr_b16: 16 lanes read 4 tokens of 16 elements, and each gets
// one element's 4 tokens).  The banks differ for the reads of keys; of values, four lanes read two neighbouring pieces of a
// row, and two rows' pieces each lie in the same banks: a two-way conflict on every read (9.5e6 of the 29.4e6 cycles
// in which the LDS is active, 16 ragged prompts).
// What bounds it: three pipes that a wave uses in turn and two waves a SIMD overlap in part: matrix products (a
// third of the time), vector instructions (2.4 for a product: exponentials, their sums, the running
// maximum) and LDS (16 KB for 32 products), and the wait for the next tokens.  One sequence of
// 16,384 tokens, 8 key heads, 16 query heads: 1,276 us, 862 TFLOP/s; 16 ragged ones of 1 to 2,500 tokens
// 197 us, 717, with the start of a workgroup, some 5 us, and the last ones to end.
template <int DP>
struct KvPromptShared {
  alignas(1024) uint16_t k[2][64 * DP];
  alignas(1024) uint16_t v[2][64 * DP];
};

// Rows that differ here are read together: 8 a + 4 u + b for a, b in 0 .. 3 (keys), and
// 8 a + b (values).
template <int DP>
__device__ __forceinline__ int kv_swizzle(int row) {
  const int f = (row & 3) | (row >> 1 & 12);
  return DP == 128 ? f : f >> 1;  // (two rows of 64 elements fill the banks)
}

// The same address in all lanes, which the compiler does not always see.
__device__ __forceinline__ uint64_t kv_scalar(const char* p) {
  const uint64_t f = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(f)),
                 hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(f >> 32));
  return static_cast<uint64_t>(hi) << 32 | lo;
}

// 16 bytes a lane from memory at `from` + lane_offset to LDS at `lds` + 16 lane, twice.  Nothing waits for them but
// kv_lds_wait (the compiler, which is not told, would have every LDS read wait); they
// write no vector register.  m0, which holds the LDS address, is the compiler's (it takes no clobber of it) and is put
// back.  Nor does the compiler look into the statement for hazards: a transfer must come one wait state after the
// write to m0, and five after a vector instruction that wrote its base's scalar registers.  The scalar copy of the
// base is that wait state, and what the transfer reads is then written by a scalar instruction.  (One sequence of
// 16,384 tokens: 1,264 us without copies and without m0 put back, 1,276 with, 1,303 with s_nop 4.)
__device__ __forceinline__ void kv_to_lds(uint32_t lds, const char* from, uint32_t lds2, const char* from2, uint32_t lane_offset) {
  uint32_t m0;
  uint64_t base;
  asm volatile(
      "s_mov_b32 %0, m0\n\t"
      "s_mov_b32 m0, %2\n\ts_mov_b64 %1, %3\n\tglobal_load_lds_dwordx4 %6, %1\n\t"
      "s_mov_b32 m0, %4\n\ts_mov_b64 %1, %5\n\tglobal_load_lds_dwordx4 %6, %1\n\t"
      "s_mov_b32 m0, %0"
      : "=&s"(m0), "=&s"(base)
      : "s"(__builtin_amdgcn_readfirstlane(lds)), "s"(kv_scalar(from)), "s"(__builtin_amdgcn_readfirstlane(lds2)),
        "s"(kv_scalar(from2)), "v"(lane_offset)
      : "memory");
}
__device__ __forceinline__ void kv_lds_wait() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// WHOLE: the heads have DP elements (without the branches a block's transfers are one piece of code, and what
// the scalar registers do not hold is fetched once for all of them; one sequence of 16,384 tokens 1,690 ->
// 1,413 us, together with kv_largest).
template <int DP, bool WHOLE>
__global__ __launch_bounds__(KV_ATT_NT, 2) void kv_prompt_kernel(KvAttnParams P) {
  constexpr int R = 2, BLK = 64, ROWS = KV_PROMPT_ROWS;
  constexpr int NT = DP / 16, QC = DP / 32;
  __shared__ KvPromptShared<DP> sh;
  KvItem it;
  if (!kv_find_item<ROWS, BLK, KV_ITEMS<uint16_t, DP, ROWS>>(P, &it)) return;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / KV_WAVE), lane = tid & (KV_WAVE - 1);
  const int c = lane & 15, g = lane >> 4;
  const int D = WHOLE ? DP : P.p.dim, G = P.group;
  const int row0 = it.tile * ROWS, rows = it.count * G;
  const int n_rows = rows - row0 < ROWS ? rows - row0 : ROWS;
  const KvRowMap map(row0, G);
  const int p0 = it.start + map.j0, p1 = it.start + map.token(n_rows - 1) + 1;
  // this wave's rows and the positions of their tokens
  const int w0 = wave * 32 < n_rows ? wave * 32 : n_rows - 1, w1 = w0 + 31 < n_rows ? w0 + 31 : n_rows - 1;
  const int wp0 = it.start + map.token(w0), wp1 = it.start + map.token(w1);
  const bool idle = wave * 32 >= n_rows;
  bool bad = !it.fine;

  int pos[R];
  uint4 qf[R][QC];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int row = wave * 32 + 16 * r + c;
    const int in = row < n_rows ? row : n_rows - 1, j = map.token(in), head = it.head * G + map.member(in, j);
    pos[r] = it.start + j;
    const char* src = P.q.data + (it.first + j) * P.q.token + head * P.q.head;
#pragma unroll
    for (int e = 0; e < QC; ++e)
      qf[r][e] = kv_flip(e * 32 + g * 8 < D ? *reinterpret_cast<const uint4*>(src + e * 64 + g * 16) : uint4{0, 0, 0, 0}, P.flip);
  }
  if (P.zero) {
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int e = 0; e < QC; ++e) qf[r][e] = kv_zero_query<uint16_t>(qf[r][e]);
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
    const int from = kv_split_at(span.blocks, it.splits, it.split), to = kv_split_at(span.blocks, it.splits, it.split + 1);
    const int32_t* row_pages = P.t.pages + static_cast<int64_t>(it.b) * P.t.max_pages;
    const int mask = (1 << P.t.shift) - 1, last = p1 - 1;
    const char* kb = P.p.k + it.head * P.p.head_stride;
    const char* vb = P.p.v + it.head * P.p.head_stride;
    const uint32_t token_stride = static_cast<uint32_t>(P.p.token_stride);  // (a page's tokens lie within 2^31 bytes)
    auto token_of = [&](int i) { return i < span.sinks ? i * BLK : span.lo + (i - span.sinks) * BLK; };
    auto page_at = [&](int id) {
      const bool in = id >= 0 && id < P.t.n_pages;
      bad |= !in;
      return static_cast<int64_t>(in ? id : 0) * P.p.page_stride;
    };
    // A wave's share of 64 tokens: 16 of them, J times RPI whole rows of keys and of values.  RPI tokens lie
    // in one page, so a transfer's base is the same for the wave, and a lane's offset from it the same for
    // every block: a block costs a lookup and a product, which lane j makes for transfer j, and scalar sums
    // (all of it in scalar registers took 139 instructions a block: 16,384 tokens 1,410 us, now 1,306)
    constexpr int PIECES = DP / 8, J = DP / 32, RPI = 64 / PIECES;
    const uint32_t lds_k = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(
                       (__attribute__((address_space(3))) uint16_t*)&sh.k[0][0])),
                   lds_v = lds_k + static_cast<uint32_t>(offsetof(KvPromptShared<DP>, v));
    const int row_in = lane / PIECES;
    int piece[J];
    uint32_t off_whole[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
      piece[j] = lane % PIECES ^ kv_swizzle<DP>(wave * 16 + j * RPI + row_in);
      off_whole[j] = static_cast<uint32_t>(row_in) * token_stride + piece[j] * 16;
    }
    // first token of transfer j (behind the last token: the run of rows that holds that one)
    auto run_of = [&](int t0, int j) {
      const int tok = t0 + wave * 16 + j * RPI;
      return tok <= last ? tok : last & ~(RPI - 1);
    };
    int ids = 0;
    auto load_ids = [&](int t0) __attribute__((always_inline)) { ids = row_pages[run_of(t0, lane % J) >> P.t.shift]; };
    auto load_tokens = [&](int buf, int t0) __attribute__((always_inline)) {
      const int64_t own = page_at(ids) + static_cast<uint32_t>(run_of(t0, lane % J) & mask) * token_stride;
      uint32_t off[J];
#pragma unroll
      for (int j = 0; j < J; ++j) off[j] = off_whole[j];
      if (t0 + BLK - 1 > last)  // no row behind the last token is read
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const int left = last - run_of(t0, j);
          off[j] = static_cast<uint32_t>(row_in < left ? row_in : left) * token_stride + piece[j] * 16;
        }
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const uint32_t lo = __builtin_amdgcn_readlane(static_cast<int>(own), j),
                       hi = __builtin_amdgcn_readlane(static_cast<int>(own >> 32), j);
        const int64_t at = static_cast<int64_t>(static_cast<uint64_t>(hi) << 32 | lo);
        const uint32_t to = buf * 64 * DP * 2 + (wave * J + j) * 1024;
        if (WHOLE || piece[j] * 8 < D) kv_to_lds(lds_k + to, kb + at, lds_v + to, vb + at, off[j]);
      }
    };
    // whether every token at first .. end sees the n tokens from t0 on
    auto whole_for = [&](int t0, int n, int first, int end) {
      return t0 + n - 1 <= first && (P.window <= 0 || t0 > end - P.window || t0 + n <= P.sinks);
    };
    // this lane's places in 32 tokens: of the keys' row 8 (c / 4) + c % 4 (+ 4 u) piece 4 e + g, and of the
    // values' row 8 g + c / 4 (+ 4 q) elements 16 t + 4 (c % 4) on
    const int k_row = (c >> 2) * 8 + (c & 3), v_row = g * 8 + (c >> 2);
    int k_at[QC], v_at[NT];
#pragma unroll
    for (int e = 0; e < QC; ++e) k_at[e] = k_row * DP + ((4 * e + g) ^ kv_swizzle<DP>(k_row)) * 8;
#pragma unroll
    for (int t = 0; t < NT; ++t) v_at[t] = v_row * DP + ((2 * t + (c >> 1 & 1)) ^ kv_swizzle<DP>(v_row)) * 8 + (c & 1) * 4;
    // element 16 t + c of tokens 8 g .. 8 g + 7
    auto values = [&](const uint16_t* base, int t) __attribute__((always_inline)) {
      const uint16_t* at = base + v_at[t];
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at);
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 4 * DP));
      uint4 r;
      __builtin_memcpy(&r.x, &lo, 8);
      __builtin_memcpy(&r.z, &hi, 8);
      return r;
    };
    // the 32 tokens from t0 on, whose keys and values start at kt and vt
    auto multiply = [&](const uint16_t* kt, const uint16_t* vt, int t0) __attribute__((always_inline)) {
      const bool whole = whole_for(t0, 32, wp0, wp1);
      f32x4 s[R][2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        uint4 kf[QC];
#pragma unroll
        for (int e = 0; e < QC; ++e) kf[e] = *reinterpret_cast<const uint4*>(kt + k_at[e] + u * 4 * DP);
#pragma unroll
        for (int r = 0; r < R; ++r) s[r][u] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < QC; ++e)
#pragma unroll
          for (int r = 0; r < R; ++r)
            s[r][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf[e]),
                                                              __builtin_bit_cast(bf16x8, qf[r][e]), s[r][u], 0, 0, 0);
      }
      // (the values' reads are under way while the weights are computed)
      uint4 a[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t) a[t] = values(vt, t);
      bool odd = false;  // as in kv_attention_kernel
      if (!whole) {
#pragma unroll
        for (int r = 0; r < R; ++r) kv_mask(s[r], t0 + g * 8, pos[r], P.window, P.sinks);
        uint32_t largest = 0;
#pragma unroll
        for (int t = 0; t < NT; ++t)
          for (const uint32_t x : {a[t].x, a[t].y, a[t].z, a[t].w}) largest = kv_largest(largest, x);
        odd = __any(kv_not_finite(largest));
        if (odd)
#pragma unroll
          for (int t = 0; t < NT; ++t) a[t] = kv_part<0>(a[t]);
      }
      // (weights as one bf16 number: two cost 29% here, 16,384 tokens 1,260 us -> 1,625; the rounding, 2^-9 of a weight,
      // takes the error of 16 ragged prompts from 1.6e-3, the output's own, to 1.9e-3)
      bf16x8 pf[R];
#pragma unroll
      for (int r = 0; r < R; ++r) {
        kv_soften(s[r], acc[r], &m[r], &l[r], P.scale2);
#pragma unroll
        for (int e = 0; e < 8; ++e) pf[r][e] = static_cast<__bf16>(s[r][e >> 2][e & 3]);
      }
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < R; ++r)
          acc[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a[t]), pf[r], acc[r][t], 0, 0, 0);
      if (odd) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const uint4 x = values(vt, t), up = kv_part<1>(x), down = kv_part<-1>(x);
#pragma unroll
          for (int r = 0; r < R; ++r) {
            const f32x4 zero{0, 0, 0, 0};
            const f32x4 y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, up), pf[r], zero, 0, 0, 0);
            const f32x4 z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, down), pf[r], zero, 0, 0, 0);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[r][t][e] += (y[e] > 0.0f ? INFINITY : 0.0f) - (z[e] > 0.0f ? INFINITY : 0.0f);
          }
        }
      }
    };
    if (!WHOLE) {  // elements from D on are zero in Q, and here, whatever the LDS held
      for (int e = tid; e < 2 * 64 * DP / 8; e += KV_ATT_NT) reinterpret_cast<uint4*>(&sh.k[0][0])[e] = uint4{0, 0, 0, 0};
      __syncthreads();
    }
    int i = from;
    if (i < to) {
      load_ids(token_of(i));
      load_tokens(0, token_of(i));
      if (i + 1 < to) load_ids(token_of(i + 1));
    }
    kv_lds_wait();
    __syncthreads();
    // block i, in buffer BUF
    auto step = [&](auto buf) __attribute__((always_inline)) {
      constexpr int BUF = decltype(buf)::value;
      const int t0 = token_of(i);
      // (the other buffer was read before the last barrier)
      if (i + 1 < to) load_tokens(BUF ^ 1, token_of(i + 1));
      if (i + 2 < to) load_ids(token_of(i + 2));
      if (!idle) {
        if (t0 <= wp1) multiply(&sh.k[BUF][0], &sh.v[BUF][0], t0);
        if (t0 + 32 <= wp1) multiply(&sh.k[BUF][32 * DP], &sh.v[BUF][32 * DP], t0 + 32);
      }
      kv_lds_wait();
      __syncthreads();
    };
    while (i < to) {
      step(std::integral_constant<int, 0>{});
      if (++i >= to) break;
      step(std::integral_constant<int, 1>{});
      ++i;
    }
  }

  const bool any_bad = __syncthreads_or(bad);
#pragma unroll
  for (int r = 0; r < R; ++r) {
    l[r] += __shfl_xor(l[r], 16);
    l[r] += __shfl_xor(l[r], 32);
    if (any_bad) l[r] = __builtin_nanf("");
  }
  if (it.splits > 1) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int row = wave * 32 + 16 * r + c;
      if (row >= n_rows || it.slot < 0 || it.slot >= P.slots) continue;
      float* dst = P.part + (static_cast<int64_t>(it.slot) * ROWS + row) * DP + g * 4;
#pragma unroll
      for (int t = 0; t < NT; ++t) *reinterpret_cast<f32x4*>(dst + 16 * t) = acc[r][t];
      if (g == 0) {
        float* ml = P.part_ml + (static_cast<int64_t>(it.slot) * ROWS + row) * 2;
        ml[0] = m[r];
        ml[1] = l[r];
      }
    }
    return;
  }
  // The wave's rows through LDS (the workgroup is past its last read of the keys), so that DP / 8
  // lanes write a row's consecutive bytes: a lane's own 8 bytes of 16 rows each took 4 us a workgroup.
  uint16_t* own = &sh.k[0][0] + wave * 32 * DP;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const bool none = l[r] == 0.0f;  // (as in kv_put_row)
    const float inv = 1.0f / l[r];
    // (pieces of 8 bytes, permuted as the keys' of 16)
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      uint16_t y[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = kv_to_bf16(none ? 0.0f : acc[r][t][e] * inv);
      __builtin_memcpy(__builtin_assume_aligned(own + (16 * r + c) * DP + ((4 * t + g) ^ (c & 7) << 1) * 4, 8), y, 8);
    }
    const int row = wave * 32 + 16 * r + c;
    if (P.lse && g == 0 && row < n_rows) {
      const int j = map.token(row), head = it.head * G + map.member(row, j);
      P.lse[static_cast<int64_t>(it.first + j) * P.n_q_heads + head] =
          ((m[r] == -INFINITY ? 0.0f : m[r]) + log2f(l[r])) * KV_LN2;
    }
  }
  constexpr int PIECES = DP / 8, PER = KV_WAVE / PIECES;
  const int piece = lane % PIECES;
#pragma unroll
  for (int i = 0; i < 32; i += PER) {
    const int in = i + lane / PIECES, row = wave * 32 + in;
    if (row >= n_rows || piece * 8 >= D) continue;
    const uint4 x = *reinterpret_cast<const uint4*>(own + in * DP + ((2 * piece) ^ (in & 7) << 1) * 4);
    const int j = map.token(row), head = it.head * G + map.member(row, j);
    *reinterpret_cast<uint4*>(P.out.data + (it.first + j) * P.out.token + head * P.out.head + piece * 16) = x;
  }
}

// Most tiles of 16 rows that a workgroup takes: what the registers of its waves hold
// (O and Q of each row tile beside a block's keys and values).
template <typename T>
constexpr int kv_row_tiles(int dp) {
  return sizeof(T) == 2 ? (dp <= 64 ? 4 : dp <= 128 ? 2 : 1) : (dp <= 128 ? 2 : 1);
}

// Launches for heads of up to DP elements, `row_tiles` of 16 rows a workgroup (8: the
// kernel for prompts); `units` bounds the units of the call.
template <typename T, int DP>
hipError_t launch_kv_attention(const KvAttnParams& P, int row_tiles, int64_t units, bool join, hipStream_t st);

}  // namespace saki
