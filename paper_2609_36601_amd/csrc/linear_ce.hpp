// Cross entropy from hidden states: the products, and what stands around them.
//
// With logits L = X W^T (X [n, D], W [V, D]), log-sum-exp lse_r and target y_r of row r, weight w_r:
//   loss_r = -w_r (L[r, y_r] - lse_r),   dL[r, v] = w_r (exp(L[r, v] - lse_r) - [v = y_r]),
//   dX = dL W,   dW = dL^T X.
// Four products, 8 n V D operations: L is computed for the loss, whose epilogue keeps a maximum and a sum for each row
// and wave, and again, a piece of the vocabulary at a time, for dL, which is a bf16 array of the piece that both
// gradients read.  Where L fits into the workspace (KEEP_BYTES) it is kept instead, and there are three, 6 n V D.
// What bounds them: with many rows the matrix pipes at the clock that the power allows (8,192 x 151,936 x 4,096: 7.2 to
// 7.8 ms for L, 1,310 to 1,420 TFLOP/s, where a library product of this size reaches 1,435 to 1,509); with few the reading of
// W (8 rows of 2,048, 32,000 tokens, 131 MB: 23 us with the launch).
//
// One kernel does all four (ce_gemm_kernel), C[p, q] = sum_k P(p, k) Q(q, k):
//   CE_LSE  P = W   (tokens; k contiguous)   Q = X   (rows; k contiguous)    epilogue: maximum and sum over p
//   CE_DL   P = W                            Q = X                           epilogue: dL
//   CE_DX   P = W^T (elements of D; p contiguous)   Q = dL (rows; k contiguous)   epilogue: 32-bit sums
//   CE_DW   P = X^T (elements of D; p contiguous)   Q = dL^T (tokens; q contiguous)   epilogue: the gradient
// p is the side of the result that a lane holds four consecutive entries of, so that a row's maximum
// and sum are mostly in a lane's registers, and stores are 8 or 16 bytes.  Tiles of 64 k are written into
// LDS by the memory pipeline without a detour through registers, NS - 1 tiles ahead of the matrix
// instructions.  Their 16-byte pieces are permuted so that a read's rows lie in different banks.  An
// operand whose k is not contiguous is transposed by the read (ds_read_b64_tr_b16).
//
// 32 bits: a number is the sum of three bf16 numbers (24 bits, the exponent range of f32), and a product of two the
// six products of parts that are not below 2^-24 of it, which makes six times as many tiles of k for the same
// kernel: 6 / 16 of bf16's rate against the 1 / 16 of the f32 matrix instructions.
#pragma once

#include "common.hpp"
#include "../../include/saki_distill.h"

namespace saki {

typedef __attribute__((ext_vector_type(8))) __bf16 ce_bf16x8;
typedef float ce_f32x4 __attribute__((ext_vector_type(4)));
typedef short ce_s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) ce_s16x4 ce_lds_s16x4;

enum CeKind { CE_LSE, CE_DL, CE_DX, CE_DW };

constexpr int CE_BK = 64;   // k of a tile
constexpr int64_t CE_MOST_THREADS = (int64_t{1} << 32) - 1;  // of a launch
constexpr int CE_PAD = 256;  // rows and pieces of the vocabulary are padded to it: the largest tile

// What a row's gradient is made of.
struct CeRow {
  float lse_hi, lse_lo;  // log-sum-exp / ln 2, in two floats
  float weight;
  int token;
  float rest;            // 1 - p at the token, from the other tokens' sum
};

struct CeGemm {
  const void* p;               // bf16, or (ce_direct_kernel) f32
  const uint16_t* q;
  int64_t ldp, ldq;            // elements between rows in memory
  int64_t p_plane, q_plane;    // elements between the three parts of numbers of 32 bits
  int n_p, n_q, n_k;           // extents; rows of X and dL are at most *count where there is a count
  const int* count;            // rows that take part, or NULL: all
  int planes;                  // 1 or 3
  int p_tiles, q_tiles;
  int k_split;                 // CE_DX, CE_DW: tiles of k of a split
  // CE_LSE
  float2* stats;               // [rows, slots] maximum in units of log2, and sum without the row's token
  int slots, slot0;
  const int32_t* token;        // the call's; of the rows that take part, source[row] where there is a count
  const int* source;
  float* target;               // [rows] the token's logit in units of log2
  float* logits;               // [rows, ld_logits] kept for the gradient, or NULL
  int64_t ld_logits;           // at least p_tiles whole tiles
  // CE_DL
  const CeRow* rows;
  uint16_t* dl;                // [rows, ld_dl] (planes: dl_plane apart)
  int64_t ld_dl, dl_plane;
  int v0;                      // the piece's first token
  // CE_DX, and CE_DW where it has splits (else NULL)
  float* sums;                 // [splits, q, ld_sums]
  int64_t ld_sums, split_stride;
  int add;                     // to the sums of the pieces before
  // CE_DW
  void* grad;
  int64_t ld_grad;
  float scale;
};

// Parts of P and Q in the products of numbers of 32 bits, largest first.
__device__ __forceinline__ int ce_part_p(int seg) { return (0x102100 >> (4 * seg)) & 3; }  // 0 0 1 2 0 1
__device__ __forceinline__ int ce_part_q(int seg) { return (0x120010 >> (4 * seg)) & 3; }  // 0 1 0 0 2 1

// 16 bytes a lane from `from` + off to LDS at `lds` + 16 lane.  m0 holds the LDS address; it is the compiler's, which
// takes no clobber of it, and is put back.  A transfer must come one wait state after a write to m0, and five after a
// vector instruction that wrote its base: the scalar copy of the base is that wait state, and what the transfer reads is
// then written by a scalar instruction.  The compiler is not told of the transfers (every LDS read would wait for them):
// ce_wait does.
__device__ __forceinline__ void ce_to_lds(uint32_t lds, uint64_t from, uint32_t off) {
  uint32_t m0;
  uint64_t base;
  asm volatile(
      "s_mov_b32 %0, m0\n\t"
      "s_mov_b32 m0, %2\n\ts_mov_b64 %1, %3\n\tglobal_load_lds_dwordx4 %4, %1\n\t"
      "s_mov_b32 m0, %0"
      : "=&s"(m0), "=&s"(base)
      : "s"(lds), "s"(from), "v"(off)
      : "memory");
}

// All but the N youngest transfers of this wave are done, its LDS reads are, and all waves are here.
template <int N>
__device__ __forceinline__ void ce_wait() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

__device__ __forceinline__ uint64_t ce_scalar(const void* p) {
  const uint64_t f = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(f)),
                 hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(f >> 32));
  return static_cast<uint64_t>(hi) << 32 | lo;
}

// One operand's side of a workgroup: EXT entries of p (or q) and 64 of k a tile.  KC: k is
// contiguous in memory, and a tile lies in LDS as [EXT][64], piece j of row r at j ^ (r & 7).  Otherwise
// as [64][EXT], piece j of row r at j ^ 2 (r & 3) ^ (r & 8): the 32 bytes of four rows that 16 lanes of a transposing
// read take, and those of the next 16 lanes, eight rows on, lie in different banks (where two rows fill the banks,
// without the last).
// SIZE: bytes of an element; of 4, as [EXT][64] with piece j of row r at j ^ (r & 15), or [64][EXT] with piece j of row r at
// j ^ 4 (r / 8 & 3) (EXT = 64: the 16 entries that each 16 lanes read, 8 rows apart, lie in different banks).
template <bool KC, int EXT, int WAVES, int SIZE = 2>
struct CeSide {
  static constexpr int BYTES = EXT * CE_BK * SIZE;
  static constexpr int LOADS = BYTES / 1024 / WAVES;  // transfers of a wave and tile
  static_assert(LOADS * WAVES * 1024 == BYTES, "whole transfers");
  static constexpr int PER = 16 / SIZE, PIECES = (KC ? CE_BK : EXT) / PER;  // entries of a piece, pieces of a row in LDS
  static constexpr int ROWS_PER = 64 / PIECES;

  uint64_t base;       // of the tile that is transferred next (the same in all lanes)
  int64_t ld;
  uint32_t off[LOADS], off_last[LOADS];  // of this lane's parts; in the last tile of k

  // row in the tile and piece in memory of this lane's part of transfer i
  __device__ __forceinline__ static int row_of(int i, int wave, int lane) { return (i * WAVES + wave) * ROWS_PER + lane / PIECES; }
  __device__ __forceinline__ static int piece_of(int row, int lane) {
    const int at = lane % PIECES;
    if (SIZE == 4) return KC ? at ^ (row & 15) : at ^ ((row >> 3 & 3) << 2);
    return KC ? at ^ (row & 7) : at ^ ((row & 3) << 1) ^ (EXT >= 128 ? row & 8 : 0);
  }

  // first: the tile's first entry of p (q), of `extent`; n_k: how many k there are, whole tiles or not
  __device__ __forceinline__ void init(const void* data, int64_t ld_, int first, int extent, int n_k, int wave, int lane) {
    ld = ld_;
    const int left = extent - first, k_left = n_k % CE_BK == 0 ? CE_BK : n_k % CE_BK;
    base = ce_scalar(static_cast<const char*>(data) + (KC ? static_cast<int64_t>(first) * ld : static_cast<int64_t>(first)) * SIZE);
    const uint32_t pitch = static_cast<uint32_t>(ld * SIZE);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int row = row_of(i, wave, lane), piece = piece_of(row, lane);
      // behind the last row (entry): the last (the tile's first); k behind the last: one that exists
      if (KC) {
        off[i] = static_cast<uint32_t>(min(row, left - 1)) * pitch + piece * 16;
        off_last[i] = off[i] - (piece * PER < k_left ? 0 : piece * 16);
      } else {
        const uint32_t at = piece * PER < left ? piece * 16 : 0;
        off[i] = static_cast<uint32_t>(row) * pitch + at;
        off_last[i] = static_cast<uint32_t>(min(row, k_left - 1)) * pitch + at;
      }
    }
  }
  // This wave's i-th transfer of the tile of k at `base`.
  __device__ __forceinline__ void transfer(int i, uint32_t lds, bool last, int wave) const {
    ce_to_lds(__builtin_amdgcn_readfirstlane(lds + (i * WAVES + wave) * 1024), base, last ? off_last[i] : off[i]);
  }
  __device__ __forceinline__ uint64_t step() const { return static_cast<uint64_t>(KC ? CE_BK : ld * CE_BK) * SIZE; }
};

// This lane's places in an operand's tile: the fragment of 16 entries from `from` + 16 f on (f < N), k 32 kk + 8 g .. + 7.
template <bool KC, int EXT, int N>
struct CeFrag {
  const char* at[KC ? 2 : N];
  __device__ __forceinline__ void init(const char* tiles, int from, int lane) {
    const int c = lane & 15, g = lane >> 4;
    if constexpr (KC) {
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) at[kk] = tiles + (from + c) * 128 + ((kk * 4 + g) ^ (c & 7)) * 16;
    } else {
      const int row = 8 * g + (c >> 2);
#pragma unroll
      for (int f = 0; f < N; ++f) {
        const int piece = ((from >> 4) + f) * 2 + (c >> 1 & 1);
        at[f] = tiles + row * (EXT * 2) + (piece ^ ((row & 3) << 1) ^ (EXT >= 128 ? row & 8 : 0)) * 16 + (c & 1) * 8;
      }
    }
  }
  __device__ __forceinline__ ce_bf16x8 read(int tile, int f, int kk) const {
    if constexpr (KC) {
      return *reinterpret_cast<const ce_bf16x8*>(at[kk] + tile + f * 2048);
    } else {
      const char* a = at[f] + tile + kk * 32 * EXT * 2;
      const ce_s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ce_lds_s16x4*)a);
      const ce_s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ce_lds_s16x4*)(a + 4 * EXT * 2));
      ce_bf16x8 r;
      __builtin_memcpy(&r, &lo, 8);
      __builtin_memcpy(reinterpret_cast<char*>(&r) + 8, &hi, 8);
      return r;
    }
  }
};

// x as a sum of three bf16 numbers, the largest first.
__device__ __forceinline__ void ce_parts(float x, uint32_t (&h)[3]) {
  h[0] = f32_to_bf16_bits(x);
  const float a = x - __uint_as_float(h[0] << 16);
  h[1] = f32_to_bf16_bits(a);
  h[2] = f32_to_bf16_bits(a - __uint_as_float(h[1] << 16));
}

// PT x QT: the tile; WP x WQ waves; NS tiles of k in LDS.
template <int PT_, int QT_, int WP_, int WQ_, int NS_>
struct CeTile {
  static constexpr int PT = PT_, QT = QT_, WP = WP_, WQ = WQ_, NS = NS_;
  static constexpr int WAVES = WP * WQ, NT = WAVES * WAVE;
  static constexpr int TP = PT / WP / 16, TQ = QT / WQ / 16;  // fragments of a wave
  static constexpr int LDS = NS * (PT + QT) * CE_BK * 2;
  static constexpr int PER_SIMD = (LDS > 81920 ? 1 : 2) * WAVES / 4 > 0 ? (LDS > 81920 ? 1 : 2) * WAVES / 4 : 1;
};
using CeLarge = CeTile<256, 256, 2, 4, 2>;
using CeMiddle = CeTile<128, 128, 2, 2, 2>;
using CeFew = CeTile<64, 64, 4, 1, 4>;

// Which tile and split a workgroup takes.  Workgroups go round the eight dies: each die gets a run of tiles, splits one after
// the other (whose slices of both operands its L2 then holds), in columns of eight q, so that those at work on it at a
// time (32) share 4 + 8 tiles.  With a mask the runs are those of all the call's rows: tiles behind the last row that takes
// part end at once, and where there are several columns of rows the last dies have little else (3,001 rows, 2,011 of them
// taking part: 294 tiles of L on five dies, 98 on one, none on two).
__device__ __forceinline__ void ce_place(const CeGemm& A, int* p_tile, int* q_tile, int* split) {
  const int tiles = A.p_tiles * A.q_tiles, n = gridDim.x, die = blockIdx.x & 7, i = blockIdx.x >> 3;
  const int each = n >> 3, more = n & 7;
  int t = die * each + min(die, more) + i;
  *split = t / tiles;
  t -= *split * tiles;
  const int column = 8 * A.p_tiles, c0 = t / column * 8, wide = min(8, A.q_tiles - c0), in = t - c0 * A.p_tiles;
  *p_tile = in / wide;
  *q_tile = c0 + in % wide;
}

// A logit in units of log2: rounded, so that a difference of two is that of the numbers the sum is made of.
__device__ __forceinline__ float ce_log2(float logit) {
#pragma clang fp contract(off)
  return logit * LOG2E;
}

// A logit's gradient, as the products take it: the row's weight times p, and at the token p - 1, which is not taken from p: of a
// row that is certain of its token the difference would be rounding alone (1,000 tokens, 1 - p = 5e-7: off by 150%, 30% of
// the rows with the wrong sign).  bf16 heads round it to bf16, by 2^-8 of itself at most, since both products that
// read it multiply bf16 numbers; two parts would make them twice as long.  It shows in the gradients' distance from 64 bits: 1.84e-3 of
// their size instead of the 1.65e-3 that the rounding of the result alone makes (8,192 x 4,096 x 151,936).
template <bool THREE>
__device__ __forceinline__ void ce_share(const CeRow& R, float logit, bool hot, bool there, uint32_t (&h)[3]) {
  float x = R.weight * (hot ? -R.rest : fexp2((ce_log2(logit) - R.lse_hi) - R.lse_lo));
  if (!there) x = 0.0f;
  if constexpr (THREE) ce_parts(x, h);
  else h[0] = f32_to_bf16_bits(x);
}

__device__ __forceinline__ uint2 ce_bits(ce_f32x4 x) {
  return make_uint2(f32_to_bf16_bits(x[0]) | f32_to_bf16_bits(x[1]) << 16, f32_to_bf16_bits(x[2]) | f32_to_bf16_bits(x[3]) << 16);
}
// Two lanes with 4 entries each of two runs of 16 exchange halves: 8 entries of one run each, `at` from the lane's place in the first.
__device__ __forceinline__ uint4 ce_pair(uint2 a, uint2 b, int lane, int* at) {
  const bool odd = (lane & 16) != 0;
  const uint2 give = odd ? a : b;
  const uint2 got = make_uint2(__shfl_xor(give.x, 16), __shfl_xor(give.y, 16));
  *at = odd ? 12 : 0;
  return odd ? make_uint4(got.x, got.y, b.x, b.y) : make_uint4(a.x, a.y, got.x, got.y);
}

// What a wave does with its products: entry (p, q) of acc[i][j][e] is p = pw + 16 i + e, q = qw + 16 j.
template <int KIND, typename TILE, bool THREE>
__device__ __forceinline__ void ce_finish(const CeGemm& A, ce_f32x4 (&acc)[TILE::TP][TILE::TQ], int p_tile, int pw, int qw, int wp,
                                          int split, int n_q, int lane) {
  constexpr int TP = TILE::TP, TQ = TILE::TQ;
  if constexpr (KIND == CE_LSE) {
#pragma unroll
    for (int j = 0; j < TQ; ++j) {
      const int row = qw + 16 * j;
      if (A.logits && row < n_q) {
        float* const to = A.logits + row * A.ld_logits + pw;
#pragma unroll
        for (int i = 0; i < TP; ++i) *reinterpret_cast<ce_f32x4*>(to + 16 * i) = acc[i][j];
      }
      float m = -finf();
#pragma unroll
      for (int i = 0; i < TP; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          acc[i][j][e] = pw + 16 * i + e < A.n_p ? ce_log2(acc[i][j][e]) : -finf();
          m = fmaxf(m, acc[i][j][e]);
        }
      // The token's logit, which the sum leaves out: a row that is certain of its token has a log-probability and a gradient
      // of the size of what the others have, which in a sum with the token's 1 would be rounded at 2^-24.
      int at = -1;  // place of the token among this lane's 4 TP, if it is there
      if (row < n_q) {
        const int v = A.token[A.count ? A.source[row] : row] - A.v0 - pw;
        at = v >= 0 && v < TP * 16 && (v & 12) == 0 ? (v >> 4) * 4 + (v & 3) : -1;
      }
      if (__ballot(at >= 0) != 0ull) {
        float x = 0.0f;
#pragma unroll
        for (int i = 0; i < TP * 4; ++i) x = at == i ? acc[i / 4][j][i % 4] : x;
        if (at >= 0 && pw + (at >> 2) * 16 + (at & 3) < A.n_p) A.target[row] = x;
      }
      m = fmaxf(m, __shfl_xor(m, 16));
      m = fmaxf(m, __shfl_xor(m, 32));
      // (no token here: -infinity and 0)
      const float ref = m == -finf() ? 0.0f : m;
      float s = 0.0f;
#pragma unroll
      for (int i = 0; i < TP; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) s += fexp2(acc[i][j][e] - ref);
      // (the token's term left out afterwards, where there is one: left out above, it costs every tile 2% of L's time)
      if (__ballot(at >= 0) != 0ull) {
        s = 0.0f;
#pragma unroll
        for (int i = 0; i < TP * 4; ++i) s += at == i ? 0.0f : fexp2(acc[i / 4][j][i % 4] - ref);
      }
      s += __shfl_xor(s, 16);
      s += __shfl_xor(s, 32);
      if (lane < 16 && row < n_q)
        A.stats[static_cast<int64_t>(row) * A.slots + A.slot0 + p_tile * TILE::WP + wp] = make_float2(m, s);
    }
  } else if constexpr (KIND == CE_DL) {
#pragma unroll
    for (int j = 0; j < TQ; ++j) {
      const int row = qw + 16 * j;
      CeRow R = {0.0f, 0.0f, 0.0f, -1, 0.0f};
      if (row < n_q) R = A.rows[row];
      const bool there = R.token >= 0;  // (a row without a token adds nothing, whatever its logits are)
      const int hot = R.token - A.v0;
#pragma unroll
      for (int i = 0; i < TP; ++i) {
        uint32_t h[4][3];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int v = pw + 16 * i + e;
          ce_share<THREE>(R, acc[i][j][e], v == hot, there && v < A.n_p, h[e]);
        }
#pragma unroll
        for (int s = 0; s < (THREE ? 3 : 1); ++s) {
          const uint2 w = make_uint2(h[0][s] | h[1][s] << 16, h[2][s] | h[3][s] << 16);
          *reinterpret_cast<uint2*>(A.dl + s * A.dl_plane + row * A.ld_dl + pw + 16 * i) = w;
        }
      }
    }
  } else if constexpr (KIND == CE_DX) {
    float* const sums = A.sums + split * A.split_stride;
#pragma unroll
    for (int j = 0; j < TQ; ++j) {
      const int row = qw + 16 * j;
#pragma unroll
      for (int i = 0; i < TP; ++i) {
        if (row >= n_q || pw + 16 * i >= A.n_p) continue;
        ce_f32x4* const to = reinterpret_cast<ce_f32x4*>(sums + row * A.ld_sums + pw + 16 * i);
        *to = A.add ? *to + acc[i][j] : acc[i][j];
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < TQ; ++j) {
      const int64_t v = qw + 16 * j;
      if constexpr (!THREE && TP % 2 == 0) {
        if (!A.sums) {
#pragma unroll
          for (int i = 0; i < TP; i += 2) {
            int at;
            const uint4 w = ce_pair(ce_bits(acc[i][j] * A.scale), ce_bits(acc[i + 1][j] * A.scale), lane, &at);
            if (v < n_q && pw + 16 * i + at < A.n_p)
              *reinterpret_cast<uint4*>(static_cast<uint16_t*>(A.grad) + v * A.ld_grad + pw + 16 * i + at) = w;
          }
          continue;
        }
      }
#pragma unroll
      for (int i = 0; i < TP; ++i) {
        if (v >= n_q || pw + 16 * i >= A.n_p) continue;
        if (A.sums) {  // (k in splits)
          *reinterpret_cast<ce_f32x4*>(A.sums + split * A.split_stride + v * A.ld_sums + pw + 16 * i) = acc[i][j];
          continue;
        }
        const ce_f32x4 x = acc[i][j] * A.scale;
        if constexpr (THREE) {
          *reinterpret_cast<ce_f32x4*>(static_cast<float*>(A.grad) + v * A.ld_grad + pw + 16 * i) = x;
        } else {
          *reinterpret_cast<uint2*>(static_cast<uint16_t*>(A.grad) + v * A.ld_grad + pw + 16 * i) = ce_bits(x);
        }
      }
    }
  }
}

enum CeChoice { CE_LARGE, CE_MIDDLE, CE_FEW, CE_DIRECT };

// Logits in sums of 256 k: a logit that grows to 50 along k is otherwise rounded, at that size, at each of its products.
// A row that is certain of its token has a log-probability near 0 that is as far off as the difference of two such logits
// (2 rows of 2,880, log-probability 1.0e-5 off relative to itself where the sums were not split).  Few rows have the
// registers for it, and no other rows whose larger losses such an error is small beside.
template <int KIND, typename TILE>
constexpr bool CE_CHUNKS = (KIND == CE_LSE || KIND == CE_DL) && TILE::QT == CeFew::QT;
template <int TQ>
struct CeChunks {
  ce_f32x4 sum[TQ] = {};
  __device__ __forceinline__ void end(ce_f32x4 (&acc)[1][TQ]) const {
#pragma unroll
    for (int j = 0; j < TQ; ++j) acc[0][j] += sum[j];
  }
  __device__ __forceinline__ void add(ce_f32x4 (&acc)[1][TQ], int t) {
    if (t % 4 != 3) return;
#pragma unroll
    for (int j = 0; j < TQ; ++j) {
      sum[j] += acc[0][j];
      acc[0][j] = ce_f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
  }
};

template <int KIND, typename TILE, bool THREE>
__global__ __launch_bounds__(TILE::NT, TILE::PER_SIMD) void ce_gemm_kernel(CeGemm A) {
  constexpr int PT = TILE::PT, QT = TILE::QT, NS = TILE::NS, TP = TILE::TP, TQ = TILE::TQ;
  constexpr bool PKC = KIND == CE_LSE || KIND == CE_DL, QKC = KIND != CE_DW;
  using PSide = CeSide<PKC, PT, TILE::WAVES>;
  using QSide = CeSide<QKC, QT, TILE::WAVES>;
  constexpr int LOADS = PSide::LOADS + QSide::LOADS;
  constexpr int STAGE = PSide::BYTES + QSide::BYTES;
  __shared__ alignas(1024) char tiles[NS * STAGE];
  const int lane = threadIdx.x & (WAVE - 1);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
  const int wp = wave % TILE::WP, wq = wave / TILE::WP;
  int p_tile, q_tile, split;
  ce_place(A, &p_tile, &q_tile, &split);
  const int rows = A.count ? __builtin_amdgcn_readfirstlane(*A.count) : KIND == CE_DW ? A.n_k : A.n_q;
  const int n_q = KIND == CE_DW ? A.n_q : rows, n_k = KIND == CE_DW ? rows : A.n_k;
  const int p0 = p_tile * PT, q0 = q_tile * QT;
  if (q0 >= n_q) return;
  int kt = (n_k + CE_BK - 1) / CE_BK, k_first = 0;
  if (KIND == CE_DX || KIND == CE_DW) {
    k_first = split * A.k_split;
    kt = min(kt - k_first, A.k_split);
  }
  const int steps = THREE ? 6 * kt : kt;

  PSide ps;
  QSide qs;
  ps.init(A.p, A.ldp, p0, A.n_p, n_k, wave, lane);
  // (Q's memory is whole tiles of k, and holds zeros behind the last: what P has there does not matter)
  qs.init(A.q, A.ldq, q0, n_q, 0, wave, lane);
  ps.base += ps.step() * k_first;
  qs.base += qs.step() * k_first;
  const uint64_t p_start = ps.base, q_start = qs.base;
  const uint32_t lds = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char*)tiles));
  const int k_last = (n_k + CE_BK - 1) / CE_BK - 1 - k_first;
  int k_next = 0, seg = 0, stage = 0;
  // The i-th transfer of the next tile of k; the last one done, moves on (behind the last tile: the last again, which
  // nobody reads).
  auto transfer = [&](int i) __attribute__((always_inline)) {
    if (i < PSide::LOADS) ps.transfer(i, lds + stage * STAGE, k_next == k_last, wave);
    else qs.transfer(i - PSide::LOADS, lds + stage * STAGE + PSide::BYTES, false, wave);
  };
  auto transferred = [&]() __attribute__((always_inline)) {
    stage = stage + 1 == NS ? 0 : stage + 1;
    const bool more = k_next + 1 < kt;
    if constexpr (THREE) {
      if (more) {
        ++k_next;
        ps.base += ps.step();
        qs.base += qs.step();
      } else if (seg < 5) {
        ++seg;
        k_next = 0;
        ps.base = p_start + ce_part_p(seg) * A.p_plane * 2;
        qs.base = q_start + ce_part_q(seg) * A.q_plane * 2;
      }
    } else {
      k_next += more ? 1 : 0;
      ps.base += more ? ps.step() : 0;
      qs.base += more ? qs.step() : 0;
    }
  };

  CeFrag<PKC, PT, TP> pf;
  CeFrag<QKC, QT, TQ> qf;
  pf.init(tiles, wp * TP * 16, lane);
  qf.init(tiles + PSide::BYTES, wq * TQ * 16, lane);
  ce_f32x4 acc[TP][TQ];
#pragma unroll
  for (int i = 0; i < TP; ++i)
#pragma unroll
    for (int j = 0; j < TQ; ++j) acc[i][j] = ce_f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  // A tile is two halves of 32 k.  The fragments of one are read while those of the other are multiplied, and the barrier that
  // changes tiles stands between the last read of a tile and its last products, which need nothing from LDS.  What
  // else a wave has to issue, reads and transfers, is spread between the products.
  struct Half {
    ce_bf16x8 p[TP], q[TQ];
  };
  // step i of TP: 4 (TQ) products of `have`, and its share of the reads of `next`
  auto step = [&](int i, const Half& have, Half& next, int at, int kk) __attribute__((always_inline)) {
    if (i == 0) {
#pragma unroll
      for (int j = 0; j < TQ; j += 2) next.q[j] = qf.read(at, j, kk);
    }
    if (i == (TP > 1 ? 1 : 0)) {
#pragma unroll
      for (int j = 1; j < TQ; j += 2) next.q[j] = qf.read(at, j, kk);
    }
    next.p[i] = pf.read(at, i, kk);
#pragma unroll
    for (int j = 0; j < TQ; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(have.p[i], have.q[j], acc[i][j], 0, 0, 0);
  };
  CeChunks<TQ> chunks;
  if (steps > 0) {
    Half a, b;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) transfer(i);
      transferred();
    }
    ce_wait<(NS - 1) * LOADS>();
#pragma unroll
    for (int j = 0; j < TQ; ++j) a.q[j] = qf.read(0, j, 0);
#pragma unroll
    for (int i = 0; i < TP; ++i) a.p[i] = pf.read(0, i, 0);
    int now = 0;
    for (int t = 0; t < steps; ++t) {
#pragma unroll
      for (int i = 0; i < TP; ++i) {
        step(i, a, b, now * STAGE, 1);
        __builtin_amdgcn_sched_barrier(0);
      }
      ce_wait<(NS - 2) * LOADS>();  // the next tile is there, and nobody reads this one any more
      now = now + 1 == NS ? 0 : now + 1;
#pragma unroll
      for (int i = 0; i < TP; ++i) {
        step(i, b, a, now * STAGE, 0);  // (behind the last tile: the last again, unused)
#pragma unroll
        for (int k = i * LOADS / TP; k < (i + 1) * LOADS / TP; ++k) transfer(k);
        __builtin_amdgcn_sched_barrier(0);
      }
      transferred();
      if constexpr (CE_CHUNKS<KIND, TILE>) chunks.add(acc, t);
    }
    ce_wait<0>();  // no transfer is under way when the workgroup ends
    if constexpr (CE_CHUNKS<KIND, TILE>) chunks.end(acc);
  }

  ce_finish<KIND, TILE, THREE>(A, acc, p_tile, p0 + wp * TP * 16 + (lane >> 4) * 4, q0 + wq * TQ * 16 + (lane & 15), wp, split, n_q, lane);
}

// Few rows in 32 bits: memory bounds them, so the weight (P) is read as it is and taken apart where its fragments are
// read from LDS, 44 instructions for 8 numbers, instead of being written as three parts and read six times.  Q lies in
// three parts as above.  120 rows of 3,888, 106,276 tokens, loss and gradients: 9.1 -> 2.8 ms (2.2 with
// the logits kept).  Each workgroup takes the weight
// apart for 64 rows, so many rows go the other way (DIRECT_ROWS).
struct CeSplit {
  ce_bf16x8 part[3];
};
typedef __bf16 ce_bf16x2 __attribute__((ext_vector_type(2)));
typedef float ce_f32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ CeSplit ce_split(const float (&x)[8]) {
  uint32_t h[3][4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float a = x[2 * i], b = x[2 * i + 1];
#pragma unroll
    for (int s = 0; s < 3; ++s) {
      h[s][i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(ce_f32x2{a, b}, ce_bf16x2));
      a -= __uint_as_float(h[s][i] << 16);
      b -= __uint_as_float(h[s][i] & 0xffff0000u);
    }
  }
  CeSplit r;
#pragma unroll
  for (int s = 0; s < 3; ++s) __builtin_memcpy(&r.part[s], h[s], 16);
  return r;
}

using CeDirect = CeTile<64, 64, 4, 1, 2>;

template <int KIND>
__global__ __launch_bounds__(CeDirect::NT, 2) void ce_direct_kernel(CeGemm A) {
  static_assert(KIND != CE_DW, "the weight is not an operand");
  constexpr int PT = CeDirect::PT, QT = CeDirect::QT, NS = CeDirect::NS, TQ = CeDirect::TQ;
  constexpr bool PKC = KIND != CE_DX;
  using PSide = CeSide<PKC, PT, CeDirect::WAVES, 4>;
  using QSide = CeSide<true, QT, CeDirect::WAVES>;
  constexpr int LOADS = PSide::LOADS + 3 * QSide::LOADS, STAGE = PSide::BYTES + 3 * QSide::BYTES;
  __shared__ alignas(1024) char tiles[NS * STAGE];
  const int lane = threadIdx.x & (WAVE - 1), c = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
  int p_tile, q_tile, split;
  ce_place(A, &p_tile, &q_tile, &split);
  const int n_q = A.count ? __builtin_amdgcn_readfirstlane(*A.count) : A.n_q;
  const int p0 = p_tile * PT, q0 = q_tile * QT;
  if (q0 >= n_q) return;
  int kt = (A.n_k + CE_BK - 1) / CE_BK, k_first = 0;
  const int k_last = kt - 1;
  if (KIND == CE_DX) {
    k_first = split * A.k_split;
    kt = min(kt - k_first, A.k_split);
  }
  PSide ps;
  QSide qs;
  ps.init(A.p, A.ldp, p0, A.n_p, A.n_k, wave, lane);
  qs.init(A.q, A.ldq, q0, n_q, 0, wave, lane);
  ps.base += ps.step() * k_first;
  qs.base += qs.step() * k_first;
  const uint32_t lds = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char*)tiles));
  int k_next = 0;
  auto transfer = [&](int stage) __attribute__((always_inline)) {
    const uint32_t to = lds + stage * STAGE;
#pragma unroll
    for (int i = 0; i < PSide::LOADS; ++i) ps.transfer(i, to, k_first + k_next == k_last, wave);
    QSide part = qs;
#pragma unroll
    for (int s = 0; s < 3; ++s) {
#pragma unroll
      for (int i = 0; i < QSide::LOADS; ++i) part.transfer(i, to + PSide::BYTES + s * QSide::BYTES, false, wave);
      part.base += static_cast<uint64_t>(A.q_plane * 2);
    }
    if (k_next + 1 < kt) {  // (behind the last tile: the last again, which nobody reads)
      ++k_next;
      ps.base += ps.step();
      qs.base += qs.step();
    }
  };
  CeFrag<true, QT, TQ> qf;
  qf.init(tiles + PSide::BYTES, 0, lane);
  ce_f32x4 acc[1][TQ];
#pragma unroll
  for (int j = 0; j < TQ; ++j) acc[0][j] = ce_f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  CeChunks<TQ> chunks;
  if (kt > 0) {
#pragma unroll
    for (int s = 0; s < NS - 1; ++s) transfer(s);
    int now = 0;
    for (int t = 0; t < kt; ++t) {
      ce_wait<(NS - 2) * LOADS>();  // this tile is there, and nobody reads the one before it any more
      transfer(now + NS - 1 >= NS ? now - 1 : now + NS - 1);
      const int at = now * STAGE;
      now = now + 1 == NS ? 0 : now + 1;
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        float x[8];
        if constexpr (PKC) {
          const int row = wave * 16 + c, piece = kk * 8 + 2 * g;
#pragma unroll
          for (int h = 0; h < 2; ++h)
            __builtin_memcpy(x + 4 * h, tiles + at + row * (CE_BK * 4) + ((piece + h) ^ (row & 15)) * 16, 16);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int row = kk * 32 + 8 * g + e, p = wave * 16 + c;
            x[e] = *reinterpret_cast<const float*>(tiles + at + row * (PT * 4) + ((p >> 2) ^ (g << 2)) * 16 + (p & 3) * 4);
          }
        }
        const CeSplit p = ce_split(x);
#pragma unroll
        for (int s = 2; s >= 0; --s) {  // q's parts, the smallest first, with those of p that matter beside them
          ce_bf16x8 q[TQ];
#pragma unroll
          for (int j = 0; j < TQ; ++j) q[j] = qf.read(at + s * QSide::BYTES, j, kk);
#pragma unroll
          for (int h = 2 - s; h >= 0; --h)
#pragma unroll
            for (int j = 0; j < TQ; ++j) acc[0][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(p.part[h], q[j], acc[0][j], 0, 0, 0);
        }
      }
      if constexpr (CE_CHUNKS<KIND, CeDirect>) chunks.add(acc, t);
    }
    ce_wait<0>();  // no transfer is under way when the workgroup ends
    if constexpr (CE_CHUNKS<KIND, CeDirect>) chunks.end(acc);
  }
  ce_finish<KIND, CeDirect, true>(A, acc, p_tile, p0 + wave * 16 + g * 4, q0 + c, wave, split, n_q, lane);
}

// ---------------------------------------------------------------------------
// Around the products.
// ---------------------------------------------------------------------------
struct CeRows {
  int64_t n_rows;
  int vocab;
  const int32_t* token;
  const float* row_weight;
  const uint8_t* valid;
  float grad_scale;
  float* row_loss;
  float* logp_token;
  double* scaled_loss;
  uint8_t* row_status;
  // workspace
  int* count;      // rows that take part (with a mask)
  int* source;     // [rows that take part] their place in the call
  int* place;      // [n_rows] the row's place among them, or -1
  CeRow* rows;     // [rows that take part]
  const float2* stats;
  const float* target;
  int slots;
};

// Rows of T as bf16 (T = float: as three parts), 64-element pieces whole: elements behind D are 0.
// source: the rows to take (or NULL: all in order).
template <typename T>
__global__ __launch_bounds__(256) void ce_pack_kernel(const T* x, int64_t stride, int64_t n_rows, int D, const int* source,
                                                      const int* count, uint16_t* to, int64_t ld, int64_t plane) {
  const int64_t rows = count ? *count : n_rows;
  const int pieces = static_cast<int>(ld / 8);
  for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < rows * pieces; i += gridDim.x * 256ll) {
    const int64_t r = i / pieces;
    const int d = static_cast<int>(i - r * pieces) * 8;
    const T* from = x + (source ? static_cast<int64_t>(source[r]) : r) * stride + d;
    uint4* const out = reinterpret_cast<uint4*>(to + r * ld + d);
    if constexpr (sizeof(T) == 2) {
      *out = d < D ? *reinterpret_cast<const uint4*>(from) : make_uint4(0u, 0u, 0u, 0u);
    } else {
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = 0.0f;
      if (d < D) Loader<float>::load8(from, v);
      uint32_t h[8][3];
#pragma unroll
      for (int e = 0; e < 8; ++e) ce_parts(v[e], h[e]);
#pragma unroll
      for (int s = 0; s < 3; ++s)
        out[s * (plane / 8)] = make_uint4(h[0][s] | h[1][s] << 16, h[2][s] | h[3][s] << 16, h[4][s] | h[5][s] << 16, h[6][s] | h[7][s] << 16);
    }
  }
}

// dL where the log-sum-exp's product kept its logits, in whole tiles of k of the products that read it.  A thread takes 8
// tokens.  It reads 4 bytes and writes 2 (three parts: 6) a logit, mostly in the last-level cache.
template <bool THREE>
__global__ __launch_bounds__(256) void ce_share_kernel(CeGemm A) {
  const int rows = A.count ? *A.count : A.n_q;
  const int v = (blockIdx.x * 256 + threadIdx.x) * 8;
  if (v >= (A.n_p + CE_BK - 1) / CE_BK * CE_BK) return;
  for (int row = blockIdx.y; row < (rows + CE_BK - 1) / CE_BK * CE_BK; row += gridDim.y) {
    CeRow R = {0.0f, 0.0f, 0.0f, -1, 0.0f};
    ce_f32x4 x[2] = {};
    if (row < rows) R = A.rows[row];
    const bool there = R.token >= 0;
    if (there) {
      const float* const from = A.logits + row * A.ld_logits + v;
      x[0] = *reinterpret_cast<const ce_f32x4*>(from);
      x[1] = *reinterpret_cast<const ce_f32x4*>(from + 4);
    }
    uint32_t h[8][3];
#pragma unroll
    for (int e = 0; e < 8; ++e) ce_share<THREE>(R, x[e / 4][e % 4], v + e == R.token - A.v0, there && v + e < A.n_p, h[e]);
#pragma unroll
    for (int s = 0; s < (THREE ? 3 : 1); ++s)
      *reinterpret_cast<uint4*>(A.dl + s * A.dl_plane + row * A.ld_dl + v) =
          make_uint4(h[0][s] | h[1][s] << 16, h[2][s] | h[3][s] << 16, h[4][s] | h[5][s] << 16, h[6][s] | h[7][s] << 16);
  }
}

// A gradient from the splits' sums, [splits, rows that take part, ld_sums].  Four of a thread's loads are under way.
struct CeSums {
  const float* sums;
  int64_t ld_sums, split_stride;
  int splits;
  int64_t n_rows;
  int D;
  const int* place;   // each row's place in the sums, -1: none (0); NULL: its own
  const CeRow* rows;  // rows without a token are NaN; NULL: none
  float scale;
  void* grad;
  int64_t stride;
};
template <typename T>
__global__ __launch_bounds__(256) void ce_sums_kernel(CeSums P) {
  const int pieces = P.D / 4;
  for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < P.n_rows * pieces; i += gridDim.x * 256ll) {
    const int64_t r = i / pieces;
    const int d = static_cast<int>(i - r * pieces) * 4;
    const int64_t at = P.place ? P.place[r] : r;
    ce_f32x4 g = {0.0f, 0.0f, 0.0f, 0.0f};
    if (at >= 0) {
      const float* from = P.sums + at * P.ld_sums + d;
      int s = 0;
      for (; s + 4 <= P.splits; s += 4) {
        ce_f32x4 v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = *reinterpret_cast<const ce_f32x4*>(from + (s + e) * P.split_stride);
#pragma unroll
        for (int e = 0; e < 4; ++e) g += v[e];
      }
      for (; s < P.splits; ++s) g += *reinterpret_cast<const ce_f32x4*>(from + s * P.split_stride);
      g *= P.rows && P.rows[at].token < 0 ? nanf_() : P.scale;
    }
    T* const to = static_cast<T*>(P.grad) + r * P.stride + d;
    if constexpr (sizeof(T) == 4) {
      *reinterpret_cast<ce_f32x4*>(to) = g;
    } else {
      *reinterpret_cast<uint2*>(to) = make_uint2(f32_to_bf16_bits(g[0]) | f32_to_bf16_bits(g[1]) << 16,
                                                 f32_to_bf16_bits(g[2]) | f32_to_bf16_bits(g[3]) << 16);
    }
  }
}

// linear_ce.hip, a unit for each part (CeKind)
template <int KIND>
hipError_t launch_ce_part(const CeGemm& A, int tile, bool three, int splits, hipStream_t st);  // tile: CeChoice

}  // namespace saki
