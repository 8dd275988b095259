// The pages of a key-value cache: room for new tokens with copies of shared last
// pages, commit and rollback, forks, compaction.
//
// A page is free iff its reference count is 0; there is no list of free pages.
// Giving pages back is then a decrement and sharing them an increment, whose
// order does not matter, and the pages given out (the lowest free ids, to the
// sequences in order) are a function of the table alone.  Taking pages has to
// find free ones among n_pages counts: one workgroup reads them all.
#pragma once

#include "kv_common.hpp"
#include "kv_count.hpp"

namespace saki {

constexpr int KV_PLAN_NT = 1024;
constexpr int KV_PLAN_WAVES = KV_PLAN_NT / KV_WAVE;

struct KvMove {  // a page to copy: its first `tokens` slots
  int32_t src, dst, tokens;
};

// What reserve keeps of a sequence between its steps.
struct KvWant {
  int32_t slot;   // table column of the page that takes the next token; -1: no copy in question
  int32_t page;   // that page
  int32_t fresh;  // new pages
  int32_t fill;   // length % page_size
};

struct KvReserveParams {
  KvTable t;
  const int32_t* n_new;
  int uniform;
  uint8_t* status;
  KvWant* want;       // [n_seq]
  int32_t* writers;   // [n_pages] sequences of this call that write to a shared page
  int32_t* last;      // [n_pages] the last of them
  int32_t* list;      // [n_pages] free pages, ascending, as many as are taken
  KvMove* moves;      // [n_seq]
  int32_t* n_moves;
};

// Which pages are free, as bits.  A wave reads 256 counts at a time, 4 consecutive ones a lane:
// bit `lane` of word e of a group stands for its page 4 lane + e.  The words of a pool of up to
// KV_BITS_PAGES pages stay in LDS between the count and the search (a search that read the
// counts again took 18 dependent loads a wave for 73,000 pages: 23 us a call, 18 with the
// bits); those of a larger one are formed again.
constexpr int KV_BITS_PAGES = 1 << 19;

struct KvFree {
  const int32_t* refs;
  int n_pages;
  bool vec;                  // refs lies on 16 bytes
  unsigned long long* bits;  // LDS

  __device__ __forceinline__ KvFree(const KvTable& t, unsigned long long* lds)
      : refs(t.refs), n_pages(t.n_pages), vec((reinterpret_cast<uintptr_t>(t.refs) & 15u) == 0), bits(lds) {}

  // pages of each wave: whole groups of 256, in order
  __device__ __forceinline__ int per_wave() const {
    return ((n_pages + KV_PLAN_WAVES * 256 - 1) / (KV_PLAN_WAVES * 256)) * 256;
  }

  __device__ __forceinline__ int4 counts(int first) const {
    const int p = first + 4 * (threadIdx.x & (KV_WAVE - 1));
    if (vec && p + 4 <= n_pages) return *reinterpret_cast<const int4*>(refs + p);
    int4 r{1, 1, 1, 1};
    if (p < n_pages) r.x = refs[p];
    if (p + 1 < n_pages) r.y = refs[p + 1];
    if (p + 2 < n_pages) r.z = refs[p + 2];
    if (p + 3 < n_pages) r.w = refs[p + 3];
    return r;
  }

  static __device__ __forceinline__ void words_of(int4 r, unsigned long long (&w)[4]) {
    w[0] = __ballot(r.x == 0);
    w[1] = __ballot(r.y == 0);
    w[2] = __ballot(r.z == 0);
    w[3] = __ballot(r.w == 0);
  }

  // free pages of this wave's part of the pool
  __device__ __forceinline__ int count() {
    constexpr int DEPTH = 16;
    const int lane = threadIdx.x & (KV_WAVE - 1);
    const int per = per_wave(), first = __builtin_amdgcn_readfirstlane(threadIdx.x / KV_WAVE) * per;
    int n = 0;
    for (int g0 = 0; g0 < per; g0 += DEPTH * 256) {
      int4 r[DEPTH];
#pragma unroll
      for (int d = 0; d < DEPTH; ++d) r[d] = g0 + d * 256 < per ? counts(first + g0 + d * 256) : int4{1, 1, 1, 1};
#pragma unroll
      for (int d = 0; d < DEPTH; ++d) {
        if (g0 + d * 256 >= per) break;
        unsigned long long w[4];
        words_of(r[d], w);
        n += __popcll(w[0]) + __popcll(w[1]) + __popcll(w[2]) + __popcll(w[3]);
        if (n_pages <= KV_BITS_PAGES && lane < 4)
          bits[(first + g0 + d * 256) / 64 + lane] = lane < 2 ? (lane == 0 ? w[0] : w[1]) : (lane == 2 ? w[2] : w[3]);
      }
    }
    return n;
  }

  // words of the group from page `first` on (the same wave's part)
  __device__ __forceinline__ void words(int first, unsigned long long (&w)[4]) const {
    if (n_pages <= KV_BITS_PAGES) {
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = bits[first / 64 + e];
    } else {
      words_of(counts(first), w);
    }
  }

  // free pages of the group before this lane's first
  static __device__ __forceinline__ int before(const unsigned long long (&w)[4]) {
    int n = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      n = __builtin_amdgcn_mbcnt_hi(static_cast<unsigned>(w[e] >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<unsigned>(w[e]), n));
    return n;
  }
  static __device__ __forceinline__ int all(const unsigned long long (&w)[4]) {
    return __popcll(w[0]) + __popcll(w[1]) + __popcll(w[2]) + __popcll(w[3]);
  }
};

// What bounds it: latency, of a chain of dependent loads and barriers in the one workgroup, which
// has to see every count before it may give a page away: 17 us for a wave of 512 sequences over
// 73,000 pages, 11 for 512 copies in a pool of 25,000, where a call that finds nothing to do takes 4.
// More workgroups would share the 290 KB of counts, but need a second launch, some 4 us.  The first 1,024
// sequences' requests stay in their threads' registers and up to KV_LIST_LDS pages in LDS.
constexpr int KV_LIST_LDS = 4096;

__global__ __launch_bounds__(KV_PLAN_NT) void kv_reserve_kernel(KvReserveParams P) {
  const KvTable& t = P.t;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / KV_WAVE), lane = tid & (KV_WAVE - 1);
  const int page_mask = (1 << t.shift) - 1;
  __shared__ int free_of[KV_PLAN_WAVES], list_lds[KV_LIST_LDS], long_from[KV_PLAN_NT];
  __shared__ int64_t part[KV_PLAN_WAVES];
  __shared__ unsigned long long bits[KV_BITS_PAGES / 64];

  // 1. what every sequence asks for (the loads of the first ones are under way while the
  // free pages are counted)
  auto asked_of = [&](int b) { return P.n_new ? P.n_new[b] : P.uniform; };
  int n0 = 0, L0 = 0, H0 = 0;
  if (tid < t.n_seq) {
    n0 = asked_of(tid);
    L0 = t.length[tid];
    H0 = t.held[tid];
  }
  KvFree pool(t, bits);
  const int counted = pool.count();
  if (lane == 0) free_of[wave] = counted;

  bool shares = false;
  KvWant first_want{-1, -1, 0, 0};  // that of sequence tid
  int first_status = SAKI_KV_OK;
  auto want_of = [&](int b) { return b == tid ? first_want : P.want[b]; };
  for (int b = tid; b < t.n_seq; b += KV_PLAN_NT) {
    const bool first = b == tid;
    const int n = first ? n0 : asked_of(b), L = first ? L0 : t.length[b], H = first ? H0 : t.held[b];
    KvWant w{-1, -1, 0, 0};
    int st = SAKI_KV_OK;
    if (n < 0 || L < 0 || H < 0 || H > t.max_pages || static_cast<int64_t>(L) > (static_cast<int64_t>(H) << t.shift)) {
      st = SAKI_KV_BAD;
    } else if (n > 0) {
      const int64_t need = (static_cast<int64_t>(L) + n + page_mask) >> t.shift;
      if (need > t.max_pages) {
        st = SAKI_KV_TOO_LONG;
      } else {
        w.fresh = need > H ? static_cast<int>(need) - H : 0;
        w.fill = L & page_mask;
        if (w.fill) {
          const int slot = L >> t.shift;
          const int p = t.pages[static_cast<int64_t>(b) * t.max_pages + slot];
          if (p < 0 || p >= t.n_pages) {
            st = SAKI_KV_BAD;
            w.fresh = 0;
          } else if (t.refs[p] > 1) {
            w.slot = slot;
            w.page = p;
            P.writers[p] = 0;
            P.last[p] = -1;
            shares = true;
          }
        }
      }
    }
    if (first) {
      first_want = w;
      first_status = st;
    } else {
      P.want[b] = w;
      if (P.status) P.status[b] = static_cast<uint8_t>(st);
    }
  }
  // 2. of a shared page's writers, the last keeps it if all its holders write
  if (__syncthreads_or(shares)) {
    for (int b = tid; b < t.n_seq; b += KV_PLAN_NT) {
      const KvWant w = want_of(b);
      if (w.slot < 0) continue;
      atomicAdd(&P.writers[w.page], 1);
      atomicMax(&P.last[w.page], b);
    }
    __syncthreads();
    for (int b = tid; b < t.n_seq; b += KV_PLAN_NT) {
      const KvWant w = want_of(b);
      // (atomic reads: the counts were changed in the L2)
      if (w.slot >= 0 && __hip_atomic_load(&P.writers[w.page], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == t.refs[w.page] &&
          __hip_atomic_load(&P.last[w.page], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == b) {
        if (b == tid)
          first_want.slot = -1;
        else
          P.want[b].slot = -1;
      }
    }
  }
  // 3. how much that is: the call takes all of it or nothing (pages and copies in one sum: kv_count)
  auto sum_of = [&](const KvWant& w) { return kv_count(w.slot >= 0, w.fresh); };
  const bool one = t.n_seq <= KV_PLAN_NT;  // each sequence has a thread
  int64_t all = 0, at0 = 0;
  if (one) {
    at0 = kv_block_scan<KV_PLAN_NT, int64_t>(sum_of(first_want), part, &all);
  } else {
    int64_t mine = 0;
    for (int b = tid; b < t.n_seq; b += KV_PLAN_NT) mine += sum_of(want_of(b));
    kv_block_scan<KV_PLAN_NT, int64_t>(mine, part, &all);
  }
  int before = 0, n_free = 0;
  for (int w = 0; w < KV_PLAN_WAVES; ++w) {
    if (w < wave) before += free_of[w];
    n_free += free_of[w];
  }
  const bool enough = kv_count_pages(all) <= n_free;
  if (P.status) {
    if (tid < t.n_seq)
      P.status[tid] = static_cast<uint8_t>(!enough && n0 > 0 && first_status == SAKI_KV_OK ? SAKI_KV_NO_PAGES : first_status);
    if (!enough)
      for (int b = tid + KV_PLAN_NT; b < t.n_seq; b += KV_PLAN_NT)
        if (asked_of(b) > 0 && P.status[b] == SAKI_KV_OK) P.status[b] = SAKI_KV_NO_PAGES;
  }
  const int total = enough ? static_cast<int>(kv_count_pages(all)) : 0;
  if (tid == 0) *P.n_moves = enough ? static_cast<int>(kv_count_copies(all)) : 0;
  if (total == 0) return;
  // 4. the lowest `total` free pages, ascending
  const bool in_lds = total <= KV_LIST_LDS;
  {
    const int per = pool.per_wave();
    const int first = wave * per;
    int rank = before;
    for (int g = 0; g < per && rank < total; g += 256) {
      unsigned long long w[4];
      pool.words(first + g, w);
      int at = rank + KvFree::before(w);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if ((w[e] >> lane) & 1) {
          if (at < total) {
            if (in_lds)
              list_lds[at] = first + g + 4 * lane + e;
            else
              P.list[at] = first + g + 4 * lane + e;
          }
          ++at;
        }
      rank += KvFree::all(w);
    }
  }
  __syncthreads();
  auto taken = [&](int i) { return in_lds ? list_lds[i] : P.list[i]; };
  // 5. each sequence its share, in order; long shares by whole waves
  int64_t done = 0;
  for (int b0 = 0; b0 < t.n_seq; b0 += KV_PLAN_NT) {
    const int b = b0 + tid;
    const KvWant w = b < t.n_seq ? want_of(b) : KvWant{-1, -1, 0, 0};
    const bool copy = w.slot >= 0;
    int64_t sum = 0;
    const int64_t at = done + (one ? at0 : kv_block_scan<KV_PLAN_NT, int64_t>(sum_of(w), part, &sum));
    done += sum;
    int from = static_cast<int>(kv_count_pages(at));
    const int64_t row = static_cast<int64_t>(b) * t.max_pages;
    if (copy) {
      const int to = taken(from);
      P.moves[kv_count_copies(at)] = KvMove{w.page, to, w.fill};
      t.pages[row + w.slot] = to;
      t.refs[to] = 1;
      atomicSub(&t.refs[w.page], 1);
      ++from;
    }
    const bool is_long = w.fresh > 8;
    const int H = w.fresh > 0 ? (b == tid ? H0 : t.held[b]) : 0;
    if (!is_long)
      for (int i = 0; i < w.fresh; ++i) {
        const int id = taken(from + i);
        t.pages[row + H + i] = id;
        t.refs[id] = 1;
      }
    if (w.fresh > 0) t.held[b] = H + w.fresh;
    if (__syncthreads_or(is_long)) {
      __shared__ int long_held[KV_PLAN_NT], long_n[KV_PLAN_NT];
      long_from[tid] = is_long ? from : -1;
      long_held[tid] = H;
      long_n[tid] = w.fresh;
      __syncthreads();
      for (int s = wave; s < KV_PLAN_NT && b0 + s < t.n_seq; s += KV_PLAN_WAVES) {
        const int f = long_from[s];
        if (f < 0) continue;
        for (int i = lane; i < long_n[s]; i += KV_WAVE) {
          const int id = taken(f + i);
          t.pages[static_cast<int64_t>(b0 + s) * t.max_pages + long_held[s] + i] = id;
          t.refs[id] = 1;
        }
      }
      __syncthreads();
    }
  }
}

// Copies pages: a unit is the slots of one head of one page of one layer, of the
// keys or the values; workgroups take units in turn.  What bounds it: memory (512 shared pages of 4
// layers copied in 31 us, 7.2 TB/s read and written, much of it from the caches, since
// eight copies have one source; compaction's moves of whole pages 5.1 TB/s).
struct KvCopyParams {
  KvPool p;
  const KvMove* moves;
  const int32_t* n_moves;
  int row_chunks;  // 16-byte pieces of a token's row
};

constexpr int KV_COPY_NT = 256;

__device__ __forceinline__ void kv_copy_units(const KvCopyParams& P, int64_t unit, int64_t step) {
  const int64_t n = static_cast<int64_t>(*P.n_moves) * P.p.n_layers * 2 * P.p.n_heads;
  for (; unit < n; unit += step) {
    int64_t u = unit;
    const int h = static_cast<int>(u % P.p.n_heads);
    u /= P.p.n_heads;
    char* base = (u & 1) ? P.p.v : P.p.k;
    u >>= 1;
    const int64_t layer = u % P.p.n_layers;
    const KvMove mv = P.moves[u / P.p.n_layers];
    base += layer * P.p.layer_stride + h * P.p.head_stride;
    const char* src = base + mv.src * P.p.page_stride;
    char* dst = base + mv.dst * P.p.page_stride;
    const int pieces = mv.tokens * P.row_chunks;
    for (int i = threadIdx.x; i < pieces; i += KV_COPY_NT) {
      const int tok = i / P.row_chunks, c = i - tok * P.row_chunks;
      const int64_t off = tok * P.p.token_stride + c * 16;
      *reinterpret_cast<uint4*>(dst + off) = *reinterpret_cast<const uint4*>(src + off);
    }
  }
}

__global__ __launch_bounds__(KV_COPY_NT) void kv_copy_kernel(KvCopyParams P) {
  kv_copy_units(P, blockIdx.x, gridDim.x);
}

// One wave per sequence: the new length, and the pages behind it given back.  What bounds it: the
// launch and three dependent accesses (512 sequences 4 us).
struct KvCommitParams {
  KvTable t;
  const int32_t* delta;
  const uint8_t* done;
  uint8_t* status;
};

__global__ __launch_bounds__(256) void kv_commit_kernel(KvCommitParams P) {
  const KvTable& t = P.t;
  const int b = blockIdx.x * (256 / KV_WAVE) + threadIdx.x / KV_WAVE, lane = threadIdx.x & (KV_WAVE - 1);
  if (b >= t.n_seq) return;
  const int L = t.length[b], H = t.held[b];
  const bool over = P.done && P.done[b] != 0;
  const int64_t to = over ? 0 : static_cast<int64_t>(L) + (P.delta ? P.delta[b] : 0);
  const bool fine = H >= 0 && H <= t.max_pages && L >= 0 && to >= 0 && to <= (static_cast<int64_t>(H) << t.shift);
  if (fine) {
    const int keep = static_cast<int>((to + (1 << t.shift) - 1) >> t.shift);
    int32_t* row = t.pages + static_cast<int64_t>(b) * t.max_pages;
    for (int i = keep + lane; i < H; i += KV_WAVE) {
      const int p = row[i];
      row[i] = -1;
      if (p >= 0 && p < t.n_pages) atomicSub(&t.refs[p], 1);
    }
    if (lane == 0) {
      t.length[b] = static_cast<int>(to);
      if (keep != H) t.held[b] = keep;
    }
  }
  if (P.status && lane == 0) P.status[b] = fine ? SAKI_KV_OK : SAKI_KV_BAD;
}

// One wave per pair.  Whether a pair is allowed is decided from the lists and
// from entries that no allowed pair changes: dst of an allowed pair is changed
// by its own wave alone, and no allowed pair's src is any pair's dst.  What bounds it: as the commit
// (448 pairs 5 us; comparing the pairs with each other outgrows that from some 10,000 on).
struct KvForkParams {
  KvTable t;
  const int32_t* src;
  const int32_t* dst;
  uint8_t* status;
  int n;
};

__global__ __launch_bounds__(256) void kv_fork_kernel(KvForkParams P) {
  const KvTable& t = P.t;
  const int i = blockIdx.x * (256 / KV_WAVE) + threadIdx.x / KV_WAVE, lane = threadIdx.x & (KV_WAVE - 1);
  if (i >= P.n) return;
  const int s = P.src[i], d = P.dst[i];
  bool fine = s >= 0 && s < t.n_seq && d >= 0 && d < t.n_seq;
  bool clash = false;
  for (int j = lane; j < P.n; j += KV_WAVE) {
    const int o = P.dst[j];
    clash |= (o == d && j < i) || P.src[j] == d;
  }
  fine = fine && !__any(clash);
  int L = 0, H = 0;
  if (fine) {
    L = t.length[s];
    H = t.held[s];
    fine = t.length[d] == 0 && t.held[d] == 0 && L >= 0 && H >= 0 && H <= t.max_pages &&
           static_cast<int64_t>(L) <= (static_cast<int64_t>(H) << t.shift);
  }
  if (fine) {
    const int n = (L + (1 << t.shift) - 1) >> t.shift;
    const int32_t* from = t.pages + static_cast<int64_t>(s) * t.max_pages;
    int32_t* to = t.pages + static_cast<int64_t>(d) * t.max_pages;
    for (int j = lane; j < n; j += KV_WAVE) {
      const int p = from[j];
      to[j] = p;
      if (p >= 0 && p < t.n_pages) atomicAdd(&t.refs[p], 1);
    }
    if (lane == 0) {
      t.length[d] = L;
      t.held[d] = n;
    }
  }
  if (P.status && lane == 0) P.status[i] = fine ? SAKI_KV_OK : SAKI_KV_BAD;
}

// Compaction's plan: the holes below n_live and the live pages from there on, both
// ascending, are paired; counts move with the pages.  One workgroup, as reserve, and bound alike
// (25,000 pages 8.5 us, of a compaction's 380).
struct KvCompactParams {
  KvTable t;
  int32_t* n_live;  // in the workspace
  int32_t* n_live_out;
  int32_t* to;  // [n_pages] where a live page >= n_live goes; -1: a free one
  int32_t* holes;
  int32_t* live;
  KvMove* moves;
  int32_t* n_moves;
};

__global__ __launch_bounds__(KV_PLAN_NT) void kv_compact_kernel(KvCompactParams P) {
  const KvTable& t = P.t;
  const int tid = threadIdx.x, wave = tid / KV_WAVE, lane = tid & (KV_WAVE - 1);
  __shared__ int free_of[KV_PLAN_WAVES], holes_of[KV_PLAN_WAVES];
  __shared__ unsigned long long bits[KV_BITS_PAGES / 64];
  KvFree pool(t, bits);
  const int counted = pool.count();
  if (lane == 0) free_of[wave] = counted;
  __syncthreads();
  int free_before = 0, n_free = 0;
  for (int w = 0; w < KV_PLAN_WAVES; ++w) {
    if (w < wave) free_before += free_of[w];
    n_free += free_of[w];
  }
  const int n_live = t.n_pages - n_free;
  const int per = pool.per_wave();
  const int first = wave * per;
  // ranks among all free and all live pages; of those, the holes are the free
  // pages below n_live, which are the first ones, and the moving pages the last
  int holes = 0;
  int rank = free_before;
  for (int g = 0; g < per; g += 256) {
    unsigned long long w[4];
    pool.words(first + g, w);
    int f = rank + KvFree::before(w);  // free pages before this lane's first
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int p = first + g + 4 * lane + e;
      if (p >= t.n_pages) break;
      if ((w[e] >> lane) & 1) {
        if (p < n_live) {
          P.holes[f] = p;
          ++holes;
        } else {
          P.to[p] = -1;
        }
        ++f;
      } else if (p >= n_live) {
        // live pages before p: p - f; counted from the end, since how many live
        // pages lie below n_live is not known yet
        P.live[n_live - 1 - (p - f)] = p;
      }
    }
    rank += KvFree::all(w);
  }
  holes = kv_wave_sum(holes);
  if (lane == 0) holes_of[wave] = holes;
  __syncthreads();
  int n = 0;
  for (int w = 0; w < KV_PLAN_WAVES; ++w) n += holes_of[w];
  // as many live pages lie from n_live on as holes below it
  for (int i = tid; i < n; i += KV_PLAN_NT) {
    const int src = P.live[n - 1 - i], dst = P.holes[i];
    P.to[src] = dst;
    P.moves[i] = KvMove{src, dst, 1 << t.shift};
    t.refs[dst] = t.refs[src];
    t.refs[src] = 0;
  }
  if (tid == 0) {
    *P.n_moves = n;
    *P.n_live = n_live;
    if (P.n_live_out) *P.n_live_out = n_live;
  }
}

// The moves, and the table's entries after them: the first workgroups take a
// sequence a wave, the others copy.
struct KvMoveParams {
  KvCopyParams c;
  KvTable t;
  const int32_t* n_live;
  const int32_t* to;
  int table_groups;
};

__global__ __launch_bounds__(KV_COPY_NT) void kv_move_kernel(KvMoveParams P) {
  if (static_cast<int>(blockIdx.x) >= P.table_groups) {
    kv_copy_units(P.c, blockIdx.x - P.table_groups, gridDim.x - P.table_groups);
    return;
  }
  if (*P.c.n_moves == 0) return;
  const int wave = threadIdx.x / KV_WAVE, lane = threadIdx.x & (KV_WAVE - 1);
  const int n_live = *P.n_live;
  for (int b = blockIdx.x * (KV_COPY_NT / KV_WAVE) + wave; b < P.t.n_seq; b += P.table_groups * (KV_COPY_NT / KV_WAVE)) {
    const int H = kv_held(P.t, b);
    int32_t* row = P.t.pages + static_cast<int64_t>(b) * P.t.max_pages;
    for (int i = lane; i < H; i += KV_WAVE) {
      const int p = row[i];
      if (p >= n_live && p < P.t.n_pages) {
        const int to = P.to[p];
        if (to >= 0) row[i] = to;
      }
    }
  }
}

}  // namespace saki
