// The entry points of the paged key-value cache: argument checks and launches.
#include <algorithm>

#include "abi.hpp"
#include "kv_attention.hpp"
#include "kv_pages.hpp"

namespace saki {

namespace {

constexpr int64_t MAX_TOKENS = int64_t{1} << 30;  // of a sequence's pages, and of `shift`
constexpr int64_t MAX_FORKS = int64_t{1} << 20;   // pairs of a call: each is compared with all others
constexpr int64_t MAX_THREADS = int64_t{1} << 32;  // a launch has fewer

int64_t up16(int64_t b) { return (b + 15) & ~int64_t{15}; }
int elem_bytes(int32_t dtype) { return dtype == SAKI_BF16 ? 2 : 4; }
bool off(const void* p, unsigned align) { return (reinterpret_cast<uintptr_t>(p) & (align - 1)) != 0; }

saki_status check_table(const saki_kv_table* t) {
  if (!t) return abi_fail(SAKI_E_NULLPTR, "table descriptor is NULL");
  if (t->reserved != 0) return abi_fail(SAKI_E_VALUE, "saki_kv_table.reserved must be 0");
  if (t->n_seq < 0 || t->n_seq > KV_MAX_SEQ) return abi_fail(SAKI_E_SHAPE, "n_seq outside [0, 2^24]");
  if (t->n_pages < 1 || t->n_pages > MAX_TOKENS) return abi_fail(SAKI_E_SHAPE, "n_pages outside [1, 2^30]");
  if (t->page_size < 8 || t->page_size > 1024 || (t->page_size & (t->page_size - 1)) != 0)
    return abi_fail(SAKI_E_SHAPE, "page_size must be a power of two, 8 .. 1024");
  if (t->max_pages < 1 || t->max_pages > MAX_TOKENS / t->page_size)
    return abi_fail(SAKI_E_SHAPE, "max_pages < 1, or max_pages * page_size > 2^30");
  // (n_seq <= 2^24 and max_pages <= 2^27)
  if (t->n_seq * t->max_pages >= KV_MAX_ENTRIES) return abi_fail(SAKI_E_SHAPE, "n_seq * max_pages must be below 2^38");
  if (t->n_seq == 0) return SAKI_OK;
  if (!t->pages || !t->length || !t->held || !t->refs)
    return abi_fail(SAKI_E_NULLPTR, "pages, length, held and refs are required");
  if (off(t->pages, 4) || off(t->length, 4) || off(t->held, 4) || off(t->refs, 4))
    return abi_fail(SAKI_E_ALIGN, "table arrays must be 4-byte aligned");
  return SAKI_OK;
}

// Whether an array of rows of `dim` elements with these extents and strides (in
// elements) has rows that overlap, strides off 16 bytes or an extent past 2^62
// bytes.  Strides along an extent of 1 do not matter.
struct Axis {
  int64_t extent, stride;
};
const char* bad_layout(Axis* axes, int n, int64_t dim, int elem) {
  std::sort(axes, axes + n, [](const Axis& a, const Axis& b) { return a.stride < b.stride; });
  __int128 span = dim;
  for (int i = 0; i < n; ++i) {
    if (axes[i].extent <= 1) continue;
    if (axes[i].stride < 0 || (axes[i].stride * static_cast<__int128>(elem)) % 16 != 0) return "strides must be multiples of 16 bytes, >= 0";
    if (axes[i].stride < span) return "rows overlap";
    span += static_cast<__int128>(axes[i].stride) * (axes[i].extent - 1);
    if (span * elem > (static_cast<__int128>(1) << 62)) return "strides too large";
  }
  return nullptr;
}

saki_status check_pool(const saki_kv_pool* p, const saki_kv_table* t) {
  if (!p) return abi_fail(SAKI_E_NULLPTR, "pool descriptor is NULL");
  if (p->dtype != SAKI_F32 && p->dtype != SAKI_BF16) return abi_fail(SAKI_E_DTYPE, "unknown pool dtype");
  if (p->reserved != 0) return abi_fail(SAKI_E_VALUE, "saki_kv_pool.reserved must be 0");
  if (p->n_kv_heads < 1 || p->n_kv_heads > 1024) return abi_fail(SAKI_E_SHAPE, "n_kv_heads outside [1, 1024]");
  if (p->head_dim < 8 || p->head_dim > 256 || p->head_dim % 8 != 0)
    return abi_fail(SAKI_E_SHAPE, "head_dim must be a multiple of 8, 8 .. 256");
  if (p->n_layers < 1 || p->n_layers > 65536) return abi_fail(SAKI_E_SHAPE, "n_layers outside [1, 65536]");
  if (!p->k || !p->v) return abi_fail(SAKI_E_NULLPTR, "pool k and v are required");
  if (off(p->k, 16) || off(p->v, 16)) return abi_fail(SAKI_E_ALIGN, "pool bases must be 16-byte aligned");
  Axis axes[4] = {{p->n_layers, p->layer_stride},
                  {t->n_pages, p->page_stride},
                  {p->n_kv_heads, p->head_stride},
                  {t->page_size, p->token_stride}};
  if (const char* why = bad_layout(axes, 4, p->head_dim, elem_bytes(p->dtype)))
    return abi_fail(why[0] == 's' ? SAKI_E_ALIGN : SAKI_E_SHAPE, why);
  if (p->token_stride * elem_bytes(p->dtype) > INT32_MAX / t->page_size)
    return abi_fail(SAKI_E_SHAPE, "page_size * token_stride must be below 2^31 bytes");
  return SAKI_OK;
}

saki_status check_tokens(const saki_kv_tokens* n, const saki_kv_table* t) {
  if (!n) return abi_fail(SAKI_E_NULLPTR, "tokens descriptor is NULL");
  if (n->n_tokens < 0 || n->n_tokens > INT32_MAX) return abi_fail(SAKI_E_SHAPE, "n_tokens outside [0, 2^31 - 1]");
  if (n->shift < 0 || n->shift > MAX_TOKENS) return abi_fail(SAKI_E_VALUE, "shift outside [0, 2^30]");
  if (n->offsets) {
    if (off(n->offsets, 4)) return abi_fail(SAKI_E_ALIGN, "offsets must be 4-byte aligned");
  } else if (n->n_new < 0 || n->n_tokens != t->n_seq * n->n_new) {
    return abi_fail(SAKI_E_SHAPE, "without offsets, n_tokens must be n_seq * n_new, n_new >= 0");
  }
  return SAKI_OK;
}

saki_status check_heads(const saki_kv_heads* x, int64_t n_tokens, int64_t heads, const saki_kv_pool* p, bool out,
                        const char* name) {
  (void)name;
  if (!x || !x->data) return abi_fail(SAKI_E_NULLPTR, "q, q_out, k, v, out: data is required");
  if (off(x->data, 16)) return abi_fail(SAKI_E_ALIGN, "token arrays must be 16-byte aligned");
  const int e = elem_bytes(p->dtype);
  const int64_t lim = int64_t{1} << 56;
  if ((n_tokens > 1 && (x->token_stride < 0 || x->token_stride > lim / n_tokens || x->token_stride * e % 16 != 0)) ||
      (heads > 1 && (x->head_stride < 0 || x->head_stride > lim / heads || x->head_stride * e % 16 != 0)))
    return abi_fail(SAKI_E_ALIGN, "token array strides must be multiples of 16 bytes, >= 0");
  if (out) {
    Axis axes[2] = {{n_tokens, x->token_stride}, {heads, x->head_stride}};
    if (const char* why = bad_layout(axes, 2, p->head_dim, e)) return abi_fail(SAKI_E_SHAPE, why);
  }
  return SAKI_OK;
}

saki_status check_ws(const void* ws, size_t have, int op, int64_t n, int64_t m) {
  if (!ws) return abi_fail(SAKI_E_WORKSPACE, "workspace is NULL");
  if (have < kv_workspace_bytes(op, n, m)) return abi_fail(SAKI_E_WORKSPACE, "workspace too small");
  if (off(ws, 16)) return abi_fail(SAKI_E_ALIGN, "workspace must be 16-byte aligned");
  return SAKI_OK;
}

KvTable device_table(const saki_kv_table* t) {
  return KvTable{t->pages, t->length, t->held, t->refs, static_cast<int>(t->n_seq), static_cast<int>(t->max_pages),
                 static_cast<int>(t->n_pages), __builtin_ctz(static_cast<unsigned>(t->page_size))};
}

KvPool device_pool(const saki_kv_pool* p, int64_t layer) {
  const int64_t e = elem_bytes(p->dtype);
  const int64_t base = p->n_layers > 1 ? layer * p->layer_stride * e : 0;
  return KvPool{static_cast<char*>(p->k) + base,
                static_cast<char*>(p->v) + base,
                p->n_layers > 1 ? p->layer_stride * e : 0,
                p->page_stride * e,
                p->n_kv_heads > 1 ? p->head_stride * e : 0,
                p->token_stride * e,
                static_cast<int>(p->n_layers),
                p->n_kv_heads,
                p->head_dim};
}

KvTokens device_tokens(const saki_kv_tokens* n) {
  return KvTokens{n->offsets, static_cast<int>(n->n_tokens), n->n_new, n->shift};
}

KvStrides device_heads(const saki_kv_heads* x, const saki_kv_pool* p) {
  const int64_t e = elem_bytes(p->dtype);
  return x ? KvStrides{static_cast<char*>(x->data), x->token_stride * e, x->head_stride * e} : KvStrides{nullptr, 0, 0};
}

int pow2_dim(int64_t d) { return d <= 64 ? 64 : d <= 128 ? 128 : 256; }

// Workspace of an attention call with tiles of ROWS rows: the split units, and slots for the
// partial sums of their items, at most twice the items aimed at (a unit of more than one
// item fills at least half of each).
struct AttentionWs {
  int64_t split, part, slots, part_ml, bytes;
};
template <typename T, int DP, int ROWS>
AttentionWs attention_ws_of() {
  AttentionWs w{};
  constexpr int64_t ITEMS = KV_ITEMS<T, DP, ROWS>;
  w.split = 16;  // after their number
  w.part = w.split + up16(ITEMS * static_cast<int64_t>(sizeof(KvItem)));
  w.slots = 2 * ITEMS;
  w.part_ml = w.part + w.slots * ROWS * DP * 4;
  w.bytes = w.part_ml + w.slots * ROWS * 8;
  return w;
}
template <typename T, int DP>
AttentionWs attention_ws_rows(int rows) {
  if (rows == KV_PROMPT_ROWS) return attention_ws_of<T, DP, KV_PROMPT_ROWS>();
  return rows == 64 ? attention_ws_of<T, DP, 64>() : rows == 32 ? attention_ws_of<T, DP, 32>() : attention_ws_of<T, DP, 16>();
}
AttentionWs attention_ws(bool bf, int dp, int rows) {
  if (bf)
    return dp == 64    ? attention_ws_rows<uint16_t, 64>(rows)
           : dp == 128 ? attention_ws_rows<uint16_t, 128>(rows)
                       : attention_ws_rows<uint16_t, 256>(rows);
  return dp == 64    ? attention_ws_rows<float, 64>(rows)
         : dp == 128 ? attention_ws_rows<float, 128>(rows)
                     : attention_ws_rows<float, 256>(rows);
}

// Row tiles a workgroup takes in a call of `mean` rows a sequence and key head: those
// of a sequence of mean length; past 64, and past what a tile takes where the sequences alone fill the
// card (`full`), the kernel for prompts.  64 sequences, 2,000 keys, 8 key heads, us:
//   rows                16   32   48   64   96  128    (heads of 128 elements)
//   tiles of 16        100  129  170  212  296  384
//   tiles of 32        116  120  142  142  192  239
//   for prompts                  122  122  128  128
//   rows                16   32   48   64   96  128    (64)
//   tiles of 16         65   76   98  124  173  223
//   tiles of 64         66   69   70   74  112  113
//   for prompts                   76   76   82   81
// Where they do not fill it, half-empty workgroups gain nothing (4 sequences, 8,000 keys, 64 rows of 128
// elements: 45 to 60 us in tiles of 32, 56 to 61 in the kernel for prompts).
int attention_tiles(bool bf, int dp, int64_t mean, bool full) {
  const int most = bf ? kv_row_tiles<uint16_t>(dp) : kv_row_tiles<float>(dp);
  if (bf && dp <= 128 && (mean > 64 || (full && mean > 16 * most))) return KV_PROMPT_ROWS / 16;
  return std::min(most, mean <= 16 ? 1 : mean <= 32 ? 2 : 4);
}

struct ReserveWs {
  int64_t want, moves, n_moves, writers, last, list, bytes;
};
ReserveWs reserve_ws(int64_t n_seq, int64_t n_pages) {
  ReserveWs w{};
  w.want = 16;  // after the count of moves
  w.moves = w.want + up16(n_seq * static_cast<int64_t>(sizeof(KvWant)));
  w.writers = w.moves + up16(n_seq * static_cast<int64_t>(sizeof(KvMove)));
  w.last = w.writers + up16(n_pages * 4);
  w.list = w.last + up16(n_pages * 4);
  w.bytes = w.list + up16(n_pages * 4);
  return w;
}

struct CompactWs {
  int64_t to, holes, live, moves, bytes;
};
CompactWs compact_ws(int64_t n_pages) {
  CompactWs w{};
  w.to = 16;  // after n_live and the count of moves
  w.holes = w.to + up16(n_pages * 4);
  w.live = w.holes + up16(n_pages * 4);
  w.moves = w.live + up16(n_pages * 4);
  w.bytes = w.moves + up16((n_pages / 2 + 1) * static_cast<int64_t>(sizeof(KvMove)));
  return w;
}

KvCopyParams copy_params(const saki_kv_pool* pool, const KvMove* moves, const int32_t* n_moves) {
  KvCopyParams c{};
  c.p = device_pool(pool, 0);
  c.moves = moves;
  c.n_moves = n_moves;
  c.row_chunks = pool->head_dim * elem_bytes(pool->dtype) / 16;
  return c;
}

// Workgroups that copy: what keeps the memory busy, and no more than units.
int copy_groups(int64_t most_moves, const saki_kv_pool* pool, int cus) {
  const int64_t most = 8 * static_cast<int64_t>(cus);
  const int64_t per_page = 2 * pool->n_layers * pool->n_kv_heads;
  return static_cast<int>(most_moves < most / per_page + 1 ? std::min(most, most_moves * per_page) : most);
}

template <typename T>
void launch_append(const KvAppendParams& P, bool interleaved, bool vec, hipStream_t st) {
  const auto f = interleaved ? (vec ? kv_append_kernel<T, true, true> : kv_append_kernel<T, true, false>)
                             : (vec ? kv_append_kernel<T, false, true> : kv_append_kernel<T, false, false>);
  hipLaunchKernelGGL(f, dim3(static_cast<unsigned>(P.n.n_tokens)), dim3(KV_APPEND_NT), 0, st, P);
}

}  // namespace

size_t kv_workspace_bytes(int op, int64_t n, int64_t m) {
  if (n <= 0 || m <= 0) return 0;
  switch (op) {
    case SAKI_OP_KV_RESERVE:
      return n > KV_MAX_SEQ || m > MAX_TOKENS ? 0 : static_cast<size_t>(reserve_ws(n, m).bytes);
    case SAKI_OP_KV_COMPACT:
      return m > MAX_TOKENS ? 0 : static_cast<size_t>(compact_ws(m).bytes);
    case SAKI_OP_KV_ATTENTION: {
      // (a call's rows are at least those of a sequence of mean length, its tile's rows)
      int64_t most = 0;
      for (const int64_t rows : {1, 17, 33, 65})
        if (rows <= n)
          for (const bool bf : {false, true})
            for (const bool full : {false, true})
              most = std::max(most, attention_ws(bf, pow2_dim(m), 16 * attention_tiles(bf, pow2_dim(m), rows, full)).bytes);
      return static_cast<size_t>(most);
    }
    default:
      return 0;
  }
}

}  // namespace saki

using namespace saki;

extern "C" {

saki_status saki_kv_reserve(const saki_kv_table* table, const saki_kv_pool* pool, const int32_t* n_new,
                            int32_t uniform, uint8_t* status, void* ws, size_t ws_bytes, saki_stream_t stream) {
  saki_status st = check_table(table);
  if (st != SAKI_OK) return st;
  st = check_pool(pool, table);
  if (st != SAKI_OK) return st;
  if (!n_new && uniform < 0) return abi_fail(SAKI_E_VALUE, "uniform < 0");
  if (off(n_new, 4)) return abi_fail(SAKI_E_ALIGN, "n_new must be 4-byte aligned");
  if (table->n_seq == 0) return abi_ok();
  st = check_ws(ws, ws_bytes, SAKI_OP_KV_RESERVE, table->n_seq, table->n_pages);
  if (st != SAKI_OK) return st;
  int cus = 0;
  st = abi_cus(&cus);
  if (st != SAKI_OK) return st;
  char* w = static_cast<char*>(ws);
  const ReserveWs at = reserve_ws(table->n_seq, table->n_pages);
  KvReserveParams P{};
  P.t = device_table(table);
  P.n_new = n_new;
  P.uniform = uniform;
  P.status = status;
  P.want = reinterpret_cast<KvWant*>(w + at.want);
  P.writers = reinterpret_cast<int32_t*>(w + at.writers);
  P.last = reinterpret_cast<int32_t*>(w + at.last);
  P.list = reinterpret_cast<int32_t*>(w + at.list);
  P.moves = reinterpret_cast<KvMove*>(w + at.moves);
  P.n_moves = reinterpret_cast<int32_t*>(w);
  hipStream_t hs = static_cast<hipStream_t>(stream);
  hipLaunchKernelGGL(kv_reserve_kernel, dim3(1), dim3(KV_PLAN_NT), 0, hs, P);
  st = abi_launched(hipGetLastError(), "kv_reserve_kernel");
  if (st != SAKI_OK) return st;
  hipLaunchKernelGGL(kv_copy_kernel, dim3(copy_groups(table->n_seq, pool, cus)), dim3(KV_COPY_NT), 0, hs,
                     copy_params(pool, P.moves, P.n_moves));
  st = abi_launched(hipGetLastError(), "kv_copy_kernel");
  return st != SAKI_OK ? st : abi_ok();
}

saki_status saki_kv_commit(const saki_kv_table* table, const int32_t* delta, const uint8_t* done, uint8_t* status,
                           saki_stream_t stream) {
  saki_status st = check_table(table);
  if (st != SAKI_OK) return st;
  if (!delta && !done) return abi_fail(SAKI_E_NULLPTR, "delta or done is required");
  if (off(delta, 4)) return abi_fail(SAKI_E_ALIGN, "delta must be 4-byte aligned");
  if (table->n_seq == 0) return abi_ok();
  const KvCommitParams P{device_table(table), delta, done, status};
  constexpr int PER = 256 / KV_WAVE;
  hipLaunchKernelGGL(kv_commit_kernel, dim3(static_cast<unsigned>((table->n_seq + PER - 1) / PER)), dim3(256), 0,
                     static_cast<hipStream_t>(stream), P);
  st = abi_launched(hipGetLastError(), "kv_commit_kernel");
  return st != SAKI_OK ? st : abi_ok();
}

saki_status saki_kv_fork(const saki_kv_table* table, int64_t n, const int32_t* src, const int32_t* dst,
                         uint8_t* status, saki_stream_t stream) {
  saki_status st = check_table(table);
  if (st != SAKI_OK) return st;
  if (n < 0 || n > table->n_seq || n > MAX_FORKS) return abi_fail(SAKI_E_SHAPE, "n outside [0, n_seq], or more than 2^20");
  if (n == 0) return abi_ok();
  if (!src || !dst) return abi_fail(SAKI_E_NULLPTR, "src and dst are required");
  if (off(src, 4) || off(dst, 4)) return abi_fail(SAKI_E_ALIGN, "src and dst must be 4-byte aligned");
  const KvForkParams P{device_table(table), src, dst, status, static_cast<int>(n)};
  constexpr int PER = 256 / KV_WAVE;
  hipLaunchKernelGGL(kv_fork_kernel, dim3(static_cast<unsigned>((n + PER - 1) / PER)), dim3(256), 0,
                     static_cast<hipStream_t>(stream), P);
  st = abi_launched(hipGetLastError(), "kv_fork_kernel");
  return st != SAKI_OK ? st : abi_ok();
}

saki_status saki_kv_compact(const saki_kv_table* table, const saki_kv_pool* pool, int32_t* n_live, void* ws,
                            size_t ws_bytes, saki_stream_t stream) {
  saki_status st = check_table(table);
  if (st != SAKI_OK) return st;
  st = check_pool(pool, table);
  if (st != SAKI_OK) return st;
  if (off(n_live, 4)) return abi_fail(SAKI_E_ALIGN, "n_live must be 4-byte aligned");
  if (table->n_seq == 0) return abi_ok();
  st = check_ws(ws, ws_bytes, SAKI_OP_KV_COMPACT, table->n_seq, table->n_pages);
  if (st != SAKI_OK) return st;
  int cus = 0;
  st = abi_cus(&cus);
  if (st != SAKI_OK) return st;
  char* w = static_cast<char*>(ws);
  const CompactWs at = compact_ws(table->n_pages);
  KvCompactParams P{};
  P.t = device_table(table);
  P.n_moves = reinterpret_cast<int32_t*>(w);
  P.n_live = reinterpret_cast<int32_t*>(w + 4);
  P.n_live_out = n_live;
  P.to = reinterpret_cast<int32_t*>(w + at.to);
  P.holes = reinterpret_cast<int32_t*>(w + at.holes);
  P.live = reinterpret_cast<int32_t*>(w + at.live);
  P.moves = reinterpret_cast<KvMove*>(w + at.moves);
  hipStream_t hs = static_cast<hipStream_t>(stream);
  hipLaunchKernelGGL(kv_compact_kernel, dim3(1), dim3(KV_PLAN_NT), 0, hs, P);
  st = abi_launched(hipGetLastError(), "kv_compact_kernel");
  if (st != SAKI_OK) return st;
  KvMoveParams M{};
  M.c = copy_params(pool, P.moves, P.n_moves);
  M.t = P.t;
  M.n_live = P.n_live;
  M.to = P.to;
  constexpr int PER = KV_COPY_NT / KV_WAVE;
  M.table_groups = static_cast<int>(std::min<int64_t>((table->n_seq + PER - 1) / PER, cus));
  const int grid = M.table_groups + copy_groups(table->n_pages / 2 + 1, pool, cus);
  hipLaunchKernelGGL(kv_move_kernel, dim3(grid), dim3(KV_COPY_NT), 0, hs, M);
  st = abi_launched(hipGetLastError(), "kv_move_kernel");
  return st != SAKI_OK ? st : abi_ok();
}

saki_status saki_kv_append(const saki_kv_table* table, const saki_kv_pool* pool, int64_t layer,
                           const saki_kv_tokens* tokens, const saki_kv_rope* rope, int32_t n_q_heads,
                           const saki_kv_heads* q, const saki_kv_heads* q_out, const saki_kv_heads* k,
                           const saki_kv_heads* v, saki_stream_t stream) {
  saki_status st = check_table(table);
  if (st != SAKI_OK) return st;
  st = check_pool(pool, table);
  if (st != SAKI_OK) return st;
  if (layer < 0 || layer >= pool->n_layers) return abi_fail(SAKI_E_SHAPE, "layer outside [0, n_layers)");
  st = check_tokens(tokens, table);
  if (st != SAKI_OK) return st;
  if (rope) {
    if (rope->rotary_dim < 0 || rope->rotary_dim > pool->head_dim || rope->rotary_dim % 2 != 0)
      return abi_fail(SAKI_E_SHAPE, "rotary_dim must be even, 0 .. head_dim");
    if (rope->interleaved != 0 && rope->interleaved != 1) return abi_fail(SAKI_E_VALUE, "interleaved must be 0 or 1");
    if (!isfinite(rope->amplitude)) return abi_fail(SAKI_E_VALUE, "amplitude is not finite");
    if (rope->rotary_dim > 0 && !rope->freq) return abi_fail(SAKI_E_NULLPTR, "freq is required");
    if (off(rope->freq, 8)) return abi_fail(SAKI_E_ALIGN, "freq must be 8-byte aligned");
  }
  if (n_q_heads < 0 || n_q_heads > 65536) return abi_fail(SAKI_E_SHAPE, "n_q_heads outside [0, 65536]");
  if ((n_q_heads > 0) != (q != nullptr) || (q == nullptr) != (q_out == nullptr))
    return abi_fail(SAKI_E_NULLPTR, "q, q_out and n_q_heads > 0 go together");
  if (table->n_seq == 0 || tokens->n_tokens == 0) return abi_ok();
  const int64_t n = tokens->n_tokens;
  if (q) {
    st = check_heads(q, n, n_q_heads, pool, false, "q");
    if (st != SAKI_OK) return st;
    st = check_heads(q_out, n, n_q_heads, pool, true, "q_out");
    if (st != SAKI_OK) return st;
  }
  st = check_heads(k, n, pool->n_kv_heads, pool, false, "k");
  if (st != SAKI_OK) return st;
  st = check_heads(v, n, pool->n_kv_heads, pool, false, "v");
  if (st != SAKI_OK) return st;
  if (n >= MAX_THREADS / KV_APPEND_NT) return abi_fail(SAKI_E_SHAPE, "too many tokens in one call");
  KvAppendParams P{};
  P.t = device_table(table);
  P.p = device_pool(pool, layer);
  P.n = device_tokens(tokens);
  P.freq = rope ? rope->freq : nullptr;
  P.pairs = rope ? rope->rotary_dim / 2 : 0;
  P.amplitude = rope ? rope->amplitude : 1.0f;
  P.n_q_heads = n_q_heads;
  P.q = device_heads(q, pool);
  P.q_out = device_heads(q_out, pool);
  P.k = device_heads(k, pool);
  P.v = device_heads(v, pool);
  const bool inter = P.pairs > 0 && rope->interleaved != 0;
  const bool vec = P.pairs % (inter ? 4 : 8) == 0;
  hipStream_t hs = static_cast<hipStream_t>(stream);
  if (pool->dtype == SAKI_BF16)
    launch_append<uint16_t>(P, inter, vec, hs);
  else
    launch_append<float>(P, inter, vec, hs);
  st = abi_launched(hipGetLastError(), "kv_append_kernel");
  return st != SAKI_OK ? st : abi_ok();
}

saki_status saki_kv_attention(const saki_kv_table* table, const saki_kv_pool* pool, int64_t layer,
                              const saki_kv_tokens* tokens, int32_t n_q_heads, const saki_kv_heads* q,
                              const saki_kv_heads* out, float* lse, float scale, int32_t window, int32_t sinks,
                              void* ws, size_t ws_bytes, saki_stream_t stream) {
  saki_status st = check_table(table);
  if (st != SAKI_OK) return st;
  st = check_pool(pool, table);
  if (st != SAKI_OK) return st;
  if (layer < 0 || layer >= pool->n_layers) return abi_fail(SAKI_E_SHAPE, "layer outside [0, n_layers)");
  st = check_tokens(tokens, table);
  if (st != SAKI_OK) return st;
  if (n_q_heads < 1 || n_q_heads > 65536 || n_q_heads % pool->n_kv_heads != 0)
    return abi_fail(SAKI_E_SHAPE, "n_q_heads must be a multiple of n_kv_heads, at most 65536");
  // (a larger one times log2 e would be infinite in 32 bits)
  if (!(fabsf(scale) <= 0x1p127f)) return abi_fail(SAKI_E_VALUE, "scale must be within -2^127 .. 2^127");
  if (window < 0 || sinks < 0) return abi_fail(SAKI_E_VALUE, "window < 0 or sinks < 0");
  if (off(lse, 4)) return abi_fail(SAKI_E_ALIGN, "lse must be 4-byte aligned");
  if (table->n_seq == 0 || tokens->n_tokens == 0) return abi_ok();
  const int64_t n = tokens->n_tokens;
  st = check_heads(q, n, n_q_heads, pool, false, "q");
  if (st != SAKI_OK) return st;
  st = check_heads(out, n, n_q_heads, pool, true, "out");
  if (st != SAKI_OK) return st;
  st = check_ws(ws, ws_bytes, SAKI_OP_KV_ATTENTION, n * n_q_heads, pool->head_dim);
  if (st != SAKI_OK) return st;

  const bool bf = pool->dtype == SAKI_BF16;
  const int dp = pow2_dim(pool->head_dim);
  const int group = n_q_heads / pool->n_kv_heads;
  const bool full = table->n_seq * pool->n_kv_heads >= KV_ITEMS<uint16_t, 128, KV_PROMPT_ROWS>;
  const int tiles = attention_tiles(bf, dp, n * group / table->n_seq, full), rows = 16 * tiles;
  int64_t units = tokens->offsets ? n * group / rows + std::min<int64_t>(table->n_seq, n)
                                  : table->n_seq * ((static_cast<int64_t>(tokens->n_new) * group + rows - 1) / rows);
  units *= pool->n_kv_heads;
  if (n * group > INT32_MAX - 256 || units >= MAX_THREADS / KV_ATT_NT - 8192)
    return abi_fail(SAKI_E_SHAPE, "too many query rows in one call");
  KvAttnParams P{};
  P.t = device_table(table);
  P.p = device_pool(pool, layer);
  P.n = device_tokens(tokens);
  P.q = device_heads(q, pool);
  P.out = device_heads(out, pool);
  P.lse = lse;
  P.n_q_heads = n_q_heads;
  P.group = group;
  // (not 0: a hidden score is -infinity, which 0 would make a NaN)
  P.zero = scale == 0.0f;
  P.scale2 = P.zero ? 1.0f : fabsf(scale) * KV_LOG2E;
  P.flip = scale < 0.0f ? (bf ? 0x80008000u : 0x80000000u) : 0u;
  P.window = window;
  P.sinks = sinks;
  const AttentionWs at = attention_ws(bf, dp, rows);
  char* w = static_cast<char*>(ws);
  P.n_split = reinterpret_cast<int*>(w);
  P.split = reinterpret_cast<KvItem*>(w + at.split);
  P.part = reinterpret_cast<float*>(w + at.part);
  P.part_ml = reinterpret_cast<float*>(w + at.part_ml);
  P.slots = static_cast<int>(at.slots);
  // An item's share of the blocks of all units; a unit's items are rounded up, by half of one on
  // average, which calls of few units have to leave room for.  (A little more than that: the
  // slots are counted on no item being smaller.)
  const int items = static_cast<int>(at.slots / 2);
  const double aim = units < items ? items - static_cast<double>(units) / 2 : items;
  P.share = static_cast<float>(pool->n_kv_heads / aim * 1.00001);
  P.per_tile = static_cast<float>(static_cast<double>(pool->n_kv_heads) / static_cast<double>(units));
  P.span = (rows + group - 2) / group + 1;
  hipStream_t hs = static_cast<hipStream_t>(stream);
  // without more than 8 blocks of keys in any sequence nothing is split
  const bool join = table->max_pages * table->page_size > 8 * (bf ? 32 : 16);
  hipError_t e;
  if (bf)
    e = dp == 64    ? launch_kv_attention<uint16_t, 64>(P, tiles, units, join, hs)
        : dp == 128 ? launch_kv_attention<uint16_t, 128>(P, tiles, units, join, hs)
                    : launch_kv_attention<uint16_t, 256>(P, tiles, units, join, hs);
  else
    e = dp == 64    ? launch_kv_attention<float, 64>(P, tiles, units, join, hs)
        : dp == 128 ? launch_kv_attention<float, 128>(P, tiles, units, join, hs)
                    : launch_kv_attention<float, 256>(P, tiles, units, join, hs);
  st = abi_launched(e, "kv_attention_kernel");
  return st != SAKI_OK ? st : abi_ok();
}

}  // extern "C"
