/*
 * saki_kv.h -- the paged key-value caches behind the logits of a speculative rollout: room for a
 * wave's tokens, the commit and rollback of their pages, responses forked from one prompt,
 * rotary positions, and attention of the new tokens  (App. I, steps 1-2, 7).
 *
 * Part of libsaki.so; saki.h's conventions (streams, status codes, saki_last_error) hold.
 */
#ifndef SAKI_KV_H
#define SAKI_KV_H

#include "saki.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Ops of saki_workspace_bytes: for SAKI_OP_KV_RESERVE and SAKI_OP_KV_COMPACT n_rows is n_seq
 * and vocab is n_pages; for SAKI_OP_KV_ATTENTION it is n_tokens * n_q_heads and vocab is head_dim. */
#define SAKI_OP_KV_RESERVE 4
#define SAKI_OP_KV_COMPACT 5
#define SAKI_OP_KV_ATTENTION 6

/* ---------------------------------------------------------------------------
 * Paged key-value caches (App. I: the student's and teacher's caches of a
 * rollout, committed and rolled back with the trajectories).
 *
 * A cache is a pool of pages, each page_size tokens of every layer, and a table
 * that says which pages each sequence holds.  Token i of sequence b lies in
 * page pages[b][i / page_size] at slot i % page_size.  refs[p] counts the
 * sequences that hold page p; a page is free iff refs[p] = 0, and there is no
 * other list of free pages.  Sequences may share pages (saki_kv_fork); only
 * pages in front of a sequence's next token are shared, and saki_kv_reserve
 * gives a sequence a page of its own before the next token is written.
 *
 * Tables are device state that calls on one stream update in order.  Calls of
 * other streams on the same table need the caller's events between them.  All
 * table arrays are 4-byte aligned.  Entries that contradict each other (a
 * length beyond the pages held, a page id outside the pool) never lead to an
 * access outside the arrays; the sequence's status or outputs say so.
 * ------------------------------------------------------------------------- */
typedef struct {
  int64_t n_seq;     /* sequences, 0 .. 2^24                                              */
  int64_t max_pages; /* pages a sequence can hold (the width of `pages`), >= 1; max_pages *
                        page_size <= 2^30, n_seq * max_pages < 2^38                       */
  int64_t n_pages;   /* pages of the pool, 1 .. 2^30                                      */
  int32_t page_size; /* tokens per page: a power of two, 8 .. 1024                        */
  int32_t reserved;  /* must be 0                                                         */
  int32_t *pages;    /* [n_seq, max_pages] page ids; entries from held[b] on are -1       */
  int32_t *length;   /* [n_seq] tokens committed                                          */
  int32_t *held;     /* [n_seq] pages held                                                */
  int32_t *refs;     /* [n_pages] sequences that hold the page                            */
} saki_kv_table;     /* an empty table: pages -1, everything else 0                       */

/* The pool: element d of token slot t, head h, page p, layer l is at
 * base[l * layer_stride + p * page_stride + h * head_stride + t * token_stride + d].
 * Keys and values have the same type, shape and strides (in elements).  Both
 * bases are 16-byte aligned and every stride is a multiple of 16 bytes; the axes
 * may be in any order, nothing may overlap, and page_size * token_stride is
 * below 2^31 bytes. */
typedef struct {
  void *k, *v;
  int32_t dtype;      /* saki_dtype                                                       */
  int32_t n_kv_heads; /* 1 .. 1024                                                        */
  int32_t head_dim;   /* a multiple of 8, 8 .. 256                                        */
  int32_t reserved;   /* must be 0                                                        */
  int64_t n_layers;   /* 1 .. 65536                                                       */
  int64_t layer_stride, page_stride, head_stride, token_stride;
} saki_kv_pool;

/* Per-sequence status of a table call. */
#define SAKI_KV_OK 0
#define SAKI_KV_NO_PAGES 1 /* the pool has too few free pages for the call               */
#define SAKI_KV_TOO_LONG 2 /* the sequence would hold more than max_pages pages          */
#define SAKI_KV_BAD 3      /* an argument or the table's state is invalid for it         */

/* Room for n_new[b] more tokens behind length[b] (n_new: device [n_seq], >= 0;
 * or NULL and `uniform` tokens for every sequence).  A sequence that lacks
 * pages gets new ones.  If its next token falls into a partly filled page that
 * other sequences hold too, it gets a copy of that page's first length %
 * page_size slots (in every layer); only if all who hold the page write to it
 * in this call, the last of them keeps it.  length does not change; a sequence with no new
 * tokens is left as it is.  Free pages are given lowest id first to the
 * sequences in order (a sequence's copy before its new pages).  If the pool has
 * fewer free pages than the call needs, nothing changes and every sequence with
 * new tokens gets SAKI_KV_NO_PAGES; a sequence that gets SAKI_KV_TOO_LONG or
 * SAKI_KV_BAD is left out and does not hinder the others.
 *   pool    pool->k, v hold table->n_pages pages
 *   status  [n_seq] SAKI_KV_*, or NULL
 *   ws      saki_workspace_bytes(SAKI_OP_KV_RESERVE, n_seq, n_pages) bytes, 16-byte aligned */
saki_status saki_kv_reserve(const saki_kv_table *table, const saki_kv_pool *pool, const int32_t *n_new,
                            int32_t uniform, uint8_t *status, void *ws, size_t ws_bytes,
                            saki_stream_t stream);

/* length[b] += delta[b] (device [n_seq]; a negative delta drops tokens), or
 * length[b] = 0 where done[b] is non-zero (done: device uint8 [n_seq], e.g.
 * saki_traj.done, or NULL).  delta may be NULL if done is not (0 then).  Pages
 * behind the new length are given back.  A new length outside [0, held[b] *
 * page_size] leaves the sequence as it is, with SAKI_KV_BAD.  With delta =
 * saki_commit's n_commit this is the commit and rollback of a wave: the pages
 * of rejected drafts return to the pool.
 *   status  [n_seq] SAKI_KV_*, or NULL */
saki_status saki_kv_commit(const saki_kv_table *table, const int32_t *delta, const uint8_t *done,
                           uint8_t *status, saki_stream_t stream);

/* Sequence dst[i] becomes a copy of sequence src[i], i < n (device int32
 * arrays), by sharing its pages.  dst[i] must hold nothing, may be no pair's src
 * and no earlier pair's dst: such a pair, or one with an index outside [0, n_seq), is left out
 * with SAKI_KV_BAD.  n <= n_seq, at most 2^20.
 *   status  [n] SAKI_KV_*, or NULL */
saki_status saki_kv_fork(const saki_kv_table *table, int64_t n, const int32_t *src, const int32_t *dst,
                         uint8_t *status, saki_stream_t stream);

/* Moves pages so that the live ones are 0 .. n_live - 1: the i-th live page
 * with an id >= n_live moves to the i-th free id below n_live, whole, in every
 * layer; the table's entries follow.
 *   n_live  device int32 [1], or NULL
 *   ws      saki_workspace_bytes(SAKI_OP_KV_COMPACT, n_seq, n_pages) bytes, 16-byte aligned */
saki_status saki_kv_compact(const saki_kv_table *table, const saki_kv_pool *pool, int32_t *n_live, void *ws,
                            size_t ws_bytes, saki_stream_t stream);

/* Which token rows belong to which sequence: rows offsets[b] .. offsets[b+1] - 1
 * (device int32 [n_seq + 1], non-decreasing, in [0, n_tokens]), or with offsets =
 * NULL rows b * n_new .. b * n_new + n_new - 1 (n_tokens = n_seq * n_new).  The
 * j-th of them is the token at position length[b] + shift + j.  Rows of no sequence
 * are left as they are.  A range that is not in order within
 * [0, n_tokens] is taken as empty; ranges may not overlap. */
typedef struct {
  const int32_t *offsets;
  int64_t n_tokens; /* rows of the token arrays, 0 .. 2^31 - 1                            */
  int32_t n_new;    /* tokens per sequence when offsets is NULL, >= 0                     */
  int32_t shift;    /* 0 .. 2^30                                                          */
} saki_kv_tokens;

/* [n_tokens, heads, head_dim] of the pool's dtype: element (i, h, d) is at
 * data[i * token_stride + h * head_stride + d].  data is 16-byte aligned, the
 * strides are multiples of 16 bytes (e.g. a slice of a fused projection), >= 0. */
typedef struct {
  void *data;
  int64_t token_stride, head_stride;
} saki_kv_heads;

/* Rotary positions: with r = rotary_dim, pair i < r / 2 of a head is elements
 * (i, i + r / 2), or (2 i, 2 i + 1) if interleaved, and turns by
 * 2 pi * position * freq[i]:  (a, b) -> amplitude * (a cos - b sin, b cos + a sin).
 * Elements from r on are left as they are.  freq (device double [r / 2], in turns per
 * position) carries the base and any scaling for long contexts.  The angle is
 * formed and reduced in 64 bits. */
typedef struct {
  const double *freq;
  int32_t rotary_dim;  /* even, 0 (no rotation) .. head_dim                               */
  int32_t interleaved; /* 0 or 1                                                          */
  float amplitude;     /* finite                                                          */
} saki_kv_rope;

/* Rotates q into q_out and k, and writes k and v to the pages of their
 * positions in `layer`.  A token whose position is outside its sequence's pages,
 * or on a page that other sequences hold too, is not written, and its q_out row is
 * NaN: saki_kv_reserve first, again after a saki_kv_fork.
 *   rope   NULL: no rotation
 *   tokens fewer than 2^24 rows
 *   q      NULL (with q_out NULL, n_q_heads 0): keys and values only
 *   q_out  may be q itself; other overlaps between q_out and inputs are not allowed. */
saki_status saki_kv_append(const saki_kv_table *table, const saki_kv_pool *pool, int64_t layer,
                           const saki_kv_tokens *tokens, const saki_kv_rope *rope, int32_t n_q_heads,
                           const saki_kv_heads *q, const saki_kv_heads *q_out, const saki_kv_heads *k,
                           const saki_kv_heads *v, saki_stream_t stream);

/* Attention of the new tokens over their sequences' pages, which hold them
 * already (saki_kv_append).  Query head h reads key head h / (n_q_heads /
 * n_kv_heads).  The token at position i sees the keys at positions j <= i and,
 * with window > 0, of those only j > i - window and j < sinks:
 *   out = sum_j softmax_j(scale q . k_j) v_j,   lse = ln sum_j exp(scale q . k_j).
 * Keys and values at positions that a token does not see have no influence on
 * it, whatever they hold.  A token whose every score is -infinity gets out = 0,
 * lse = -infinity, whatever the values hold; one with a score of NaN or +infinity gets NaN.
 * Where a token gives a key that it sees no weight in 32 bits (a score of -infinity beside
 * finite ones, or some 85 below the largest), it is open whether a value there that is not
 * finite makes the element NaN or has no influence.  Tokens of a sequence that lacks pages
 * for them get NaN.
 * Products and softmax are accumulated in 32 bits.  With bf16 the weights are rounded for
 * their product with the values: to 2^-17 of a weight in calls of up to 32 rows (new
 * tokens times the query heads of a key head) a sequence on average, and with heads of
 * more than 128 elements; to bf16, 2^-9, in others.
 *   n_q_heads  a multiple of pool->n_kv_heads, at most 65536; n_tokens * n_q_heads / 16
 *              + n_seq * n_kv_heads below 2^24 - 8192 (more may be SAKI_E_SHAPE)
 *   out        as q; may be q itself.  lse: float [n_tokens, n_q_heads] or NULL
 *   scale      -2^127 .. 2^127;  window >= 0 (0: none);  sinks >= 0
 *   ws         saki_workspace_bytes(SAKI_OP_KV_ATTENTION, n_tokens * n_q_heads, head_dim)
 *              bytes, 16-byte aligned; calls that may run at the same time need
 *              separate workspaces */
saki_status saki_kv_attention(const saki_kv_table *table, const saki_kv_pool *pool, int64_t layer,
                              const saki_kv_tokens *tokens, int32_t n_q_heads, const saki_kv_heads *q,
                              const saki_kv_heads *out, float *lse, float scale, int32_t window,
                              int32_t sinks, void *ws, size_t ws_bytes, saki_stream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* SAKI_KV_H */
