// What the kernels of the paged key-value cache share: the table and the token
// ranges as the device sees them, and block-wide sums.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/saki_kv.h"

namespace saki {

constexpr int KV_WAVE = 64;

// The table and the pool (one layer's bases) as kernels read them.
struct KvTable {
  int32_t* pages;
  int32_t* length;
  int32_t* held;
  int32_t* refs;
  int n_seq, max_pages, n_pages;
  int shift;  // log2(page_size)
};

struct KvPool {
  char* k;
  char* v;
  int64_t layer_stride, page_stride, head_stride, token_stride;  // bytes
  int n_layers, n_heads, dim;
};

struct KvTokens {
  const int32_t* offsets;
  int n_tokens, n_new, shift;
};

// The token rows of sequence b: first row and count (0 for a range out of order).
__device__ __forceinline__ void kv_rows(const KvTokens& T, int b, int* first, int* count) {
  if (T.offsets) {
    const int a = T.offsets[b], z = T.offsets[b + 1];
    const bool fine = a >= 0 && a < z && z <= T.n_tokens;
    *first = fine ? a : 0;
    *count = fine ? z - a : 0;
  } else {
    *first = b * T.n_new;
    *count = T.n_new;
  }
}

// Pages a table entry may name as held (the count itself may be damaged).
__device__ __forceinline__ int kv_held(const KvTable& t, int b) {
  const int h = t.held[b];
  return h < 0 ? 0 : h > t.max_pages ? t.max_pages : h;
}

// x of another lane by a data-parallel move, 0 where there is none.
template <int CTRL, int ROWS>
__device__ __forceinline__ int kv_dpp(int x) {
  return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xF, true);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ int64_t kv_dpp(int64_t x) {
  const unsigned lo = static_cast<unsigned>(kv_dpp<CTRL, ROWS>(static_cast<int>(x)));
  const unsigned hi = static_cast<unsigned>(kv_dpp<CTRL, ROWS>(static_cast<int>(x >> 32)));
  return static_cast<int64_t>(static_cast<uint64_t>(hi) << 32 | lo);
}

// Inclusive prefix sum over the lanes of a wave: within the rows of 16 by shifts, then each
// row's last lane to the rows behind it.
template <typename V>
__device__ __forceinline__ V kv_wave_scan(V x) {
  x += kv_dpp<0x111, 0xF>(x);
  x += kv_dpp<0x112, 0xF>(x);
  x += kv_dpp<0x114, 0xF>(x);
  x += kv_dpp<0x118, 0xF>(x);
  x += kv_dpp<0x142, 0xA>(x);
  x += kv_dpp<0x143, 0xC>(x);
  return x;
}

__device__ __forceinline__ int kv_last(int x) { return __builtin_amdgcn_readlane(x, KV_WAVE - 1); }
__device__ __forceinline__ int64_t kv_last(int64_t x) {
  const unsigned lo = static_cast<unsigned>(kv_last(static_cast<int>(x))), hi = static_cast<unsigned>(kv_last(static_cast<int>(x >> 32)));
  return static_cast<int64_t>(static_cast<uint64_t>(hi) << 32 | lo);
}

template <typename V>
__device__ __forceinline__ V kv_wave_sum(V x) {
  return kv_last(kv_wave_scan(x));
}

// Exclusive prefix sum over the workgroup's NT threads and the total; `part` is NT / 64 values
// of LDS, which must not be written to (again) before the workgroup's next barrier.
template <int NT, typename V>
__device__ __forceinline__ V kv_block_scan(V x, V* part, V* total) {
  const int wave = threadIdx.x / KV_WAVE;
  const V in = kv_wave_scan(x);
  if ((threadIdx.x & (KV_WAVE - 1)) == KV_WAVE - 1) part[wave] = in;
  __syncthreads();
  V before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < NT / KV_WAVE; ++w) {
    if (w < wave) before += part[w];
    all += part[w];
  }
  *total = all;
  return before + in - x;
}

}  // namespace saki
